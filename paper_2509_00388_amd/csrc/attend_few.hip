// Attention of sequences with few new rows (at most 32 stacked query rows a key-value head: one token of up to 32 query
// heads, eight drafted tokens of four): bound by the read of the keys and values.
//
// The tiles of all (sequence, head) pairs are cut into equal stretches, one a workgroup, whatever the lengths (attend.hpp).
// A tile's keys are dealt to the four waves; a wave brings its 32 NB keys and values through LDS of its own, with coalesced
// 16-byte loads of the next tile in flight while this one is multiplied, and keeps its own running maximum, sum and O^T:
// no barrier until the stretch of a pair ends and the waves' parts are joined.  A pair that one workgroup holds whole is
// finished there; the parts of others go to scratch memory and are joined by a second launch.
//
// Measured (bf16 rows, d = 128, eight key heads of four): one token over 131072 keys 97 us, 5.5 TB/s (reading alone is faster than the 4.6 of
// a copy); 64 tokens over 400 to 5000 keys each in fp8 pages 93 us, 4.2 TB/s, where decode and the LDS share the time; one token
// over 2048 keys 8.3 us, a chain of look-ups, loads, two products and the join of the waves with a tile a workgroup.  Slower: three workgroups
// a compute unit, 768 or 1024 of them in all, 64 keys a wave.
#include "attend_tile.hpp"
#include "kernels.hpp"

namespace gkv {

namespace {

// A wave's place in the LDS: KEYS rows of keys, then of values, and the scales of both.
template <typename T, int FORM, int D, int NB> struct WavePlace {
    static constexpr int kPitch = Tile<T, FORM, D, 32 * NB, 64>::kKeyPitch, kRows = 32 * NB * kPitch;
    static constexpr int kBytes = kRows + (FORM == kPagesPlain ? 0 : 2 * 32 * NB * 4);
};

template <typename T, int FORM, int D, int NB>
__global__ __launch_bounds__(256, D * sizeof(T) > 256 ? 1 : 2) void attend_few_kernel(AttendArgs a, FewPlan pl)
{
    constexpr int KEYS = 32 * NB, DB = D / 32;
    using L = Tile<T, FORM, D, KEYS, 64>;
    using P = WavePlace<T, FORM, D, NB>;
    constexpr uint64_t kAllKeys = KEYS == 64 ? ~0ull : (1ull << KEYS) - 1;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint32_t part[20];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hh = lane >> 5;
    unsigned char *kv = smem + wv * P::kBytes, *qt = smem + 4 * P::kBytes;
    float *ks = reinterpret_cast<float *>(kv + P::kRows), *vs = ks + KEYS;
    const PagedBatch &b = a.b;

    uint32_t total, before;
    int n_wg = 0;
    int s = find_share<4>(b.n_seqs, total, before, part, [&](int i) { return few_tiles(seq_rows(b, i), a, pl) * b.H; },
                       [&](uint32_t all) {
                           n_wg = (int)min((uint32_t)pl.join.n_wg, all);
                           if (tid == 0) pl.join.records[blockIdx.x].parts = 0;
                           return (int)blockIdx.x < n_wg ? (int64_t)stretch_first(all, blockIdx.x, n_wg) : -1;
                       });
    if (s < 0) return;
    uint32_t tile = stretch_first(total, blockIdx.x, n_wg);
    const uint32_t last = stretch_first(total, blockIdx.x + 1, n_wg), mine = tile;
    const int pieces = b.d * L::kCached / 16, my_piece = lane % L::kPieces, my_row = lane / L::kPieces;
    const int load_piece = min(my_piece, pieces - 1);

    while (tile < last && s < b.n_seqs) {
        const SeqRows sq = seq_rows(b, s);
        const uint32_t per_head = few_tiles(sq, a, pl);
        if (per_head == 0 || tile >= before + per_head * b.H) {   // the next sequence
            before += per_head * b.H;
            ++s;
            continue;
        }
        const int h = (int)((tile - before) / per_head);
        const int t0 = (int)((tile - before) % per_head), t1 = (int)min(per_head, t0 + (last - tile));
        const int rows = sq.n * a.G;

        // Where the wave's keys of a tile lie: lane j looks key j up (lanes beyond KEYS repeat them).
        const int my_key = wv * KEYS + (lane & (KEYS - 1));
        auto entry = [&](int t) {   // page of the lane's key in tile t, -1: none
            const int pos = t * pl.tile_keys + my_key;
            return t < t1 && pos < sq.len ? raw_page(b, s, pos) : -1;
        };
        auto place = [&](int page, int t) { return !is_page(b, page) ? 0 : pool_row(b, page, h, t * pl.tile_keys + my_key); };
        uint4 kr[L::kPer], vr[L::kPer];
        float ksr = 0.f, vsr = 0.f;
        auto load = [&](const void *pages, int at, uint4 (&r)[L::kPer]) {
#pragma unroll
            for (int u = 0; u < L::kPer; ++u) {
                const int row = __builtin_amdgcn_ds_bpermute(4 * my_row + 4 * u * L::kRowStep, at);   // of lane my_row + u * kRowStep
                r[u] = reinterpret_cast<const uint4 *>(pages)[(long)row * pieces + load_piece];
            }
        };
        int page = entry(t0), at = place(page, t0);
        uint64_t vis = __ballot(is_page(b, page)) & kAllKeys;
        load(a.Kpages, at, kr);
        if (FORM != kPagesPlain) { ksr = a.Kscale[at]; vsr = a.Vscale[at]; }
        load(a.Vpages, at, vr);
        int page1 = entry(t0 + 1);

        // The query rows, in the LDS for all four waves (in registers they would be 32 of a wave's 256, and the loop spills).
        for (int i = tid; i < 32 * P::kPitch / 16; i += 256) {
            const int r = i / (P::kPitch / 16), c = i % (P::kPitch / 16) * (16 / (int)sizeof(T));
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < rows && c < b.d)
                v = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(a.Q) + (sq.row0 + r / a.G) * a.q_row + (h * a.G + r % a.G) * a.q_head + c);
            reinterpret_cast<uint4 *>(qt)[i] = v;
        }
        __syncthreads();
        const int sees = sq.len - sq.n + l32 / a.G;   // last position that the lane's query, stacked row l32, sees

        uint64_t odd_of[2] = {0, 0};   // of the first tile that not all rows see all of, and the next: values with infinities or NaN
        const int hidden = max(0, sq.len - sq.n + 1) / pl.tile_keys;

        float m = -INFINITY, l = 0.f;
        f32x16 o[DB];
#pragma unroll
        for (int x = 0; x < DB; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[x][i] = 0.f;
        if (pieces < L::kPieces)   // columns that d does not reach stay zero
            for (int i = lane; i < P::kRows / 16; i += kWave) reinterpret_cast<uint4 *>(kv)[i] = make_uint4(0, 0, 0, 0);

        for (int t = t0; t < t1; ++t) {   // in the registers: vis, at, page, kr, vr
            const int page2 = entry(t + 2), at1 = place(page1, t + 1);
            const uint64_t vis1 = __ballot(is_page(b, page1)) & kAllKeys;
            const int first = t * pl.tile_keys + wv * KEYS;
            const bool all = vis == kAllKeys && first + KEYS - 1 <= sq.len - sq.n;   // every row sees every key
            auto store = [&](const uint4 (&r)[L::kPer], uint64_t seen) {
                if (my_piece < pieces) {
#pragma unroll
                    for (int u = 0; u < L::kPer; ++u)   // (places that hold no key of the sequence may hold anything: zeros instead)
                        L::put(kv + my_row * P::kPitch + my_piece * L::kDecoded + u * L::kRowStep * P::kPitch,
                               L::only(r[u], (seen >> (u * L::kRowStep)) & 1));
                }
            };
            store(kr, vis >> my_row);
            if (FORM != kPagesPlain) {
                if (lane < KEYS) {   // (a scale without a key may be anything too)
                    ks[lane] = is_page(b, page) ? ksr * a.c : 0.f;
                    vs[lane] = is_page(b, page) ? vsr : 0.f;
                }
                ksr = a.Kscale[at1];
                vsr = a.Vscale[at1];
            }
            load(a.Kpages, at1, kr);
            wave_sync();
            f32x16 x[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[n][i] = 0.f;
#pragma unroll
                for (int st = 0; st < L::kSteps; ++st)
                    add_block(*reinterpret_cast<const uint4 *>(kv + (32 * n + l32) * P::kPitch + 32 * st + 16 * hh),
                              *reinterpret_cast<const uint4 *>(qt + l32 * P::kPitch + 32 * st + 16 * hh), x[n], T{});
            }
            wave_sync();
            uint64_t odd = 0;
            if (first + KEYS - 1 > sq.len - sq.n) {   // (no more than two of a wave's tiles)
                odd = L::odd_rows(vr, 0) & vis;
                odd_of[t > hidden] = odd;
            }
            store(vr, (vis & ~odd) >> my_row);
            load(a.Vpages, at1, vr);
            float p[NB][16];
            const uint64_t seen = seen_keys(vis, sees - first, hh);
            softmax_tile<FORM, NB, DB>(x, ks, a.c, all, seen, hh, m, l, o, p);
            if constexpr (FORM != kPagesPlain) scale_weights<NB>(vs, all, seen, hh, p);
            wave_sync();
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const unsigned char *vt = kv + 32 * n * P::kPitch;
                if constexpr (sizeof(T) == 2 && FORM == kPagesPlain) add_values_twice<D, P::kPitch>(vt, p[n], lane, o);
                else add_values<D, P::kPitch>(vt, p[n], lane, o, T{});
            }
            wave_sync();
            vis = vis1;
            at = at1;
            page = page1;
            page1 = page2;
        }

        // ---- the four waves' parts joined --------------------------------------------------------
        l = other_half_sum(l);
        int G = a.G;
        asm volatile("" : "+s"(G));   // (what was computed from it before the loop is not kept through it)
        __syncthreads();
        float *ml = reinterpret_cast<float *>(smem), *parts = ml + 256;   // [4][32][2], [4][rows][D + 4]
        if (hh == 0) { ml[(wv * 32 + l32) * 2] = m; ml[(wv * 32 + l32) * 2 + 1] = l; }
        __syncthreads();
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[(w * 32 + l32) * 2]);
        const float shift = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            sum += ml[(w * 32 + l32) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(w * 32 + l32) * 2] - shift);
        if (l32 < rows) {
            const float f = __builtin_amdgcn_exp2f(m - shift);
            float *to = parts + (wv * rows + l32) * (D + 4) + 4 * hh;
#pragma unroll
            for (int x = 0; x < DB; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<float4 *>(to + 32 * x + 8 * j) =
                        make_float4(o[x][4 * j] * f, o[x][4 * j + 1] * f, o[x][4 * j + 2] * f, o[x][4 * j + 3] * f);
        }
        if (FORM != kPagesInt8 && (odd_of[0] | odd_of[1])) {
            // Values with infinities or NaN at positions that only some rows see went through the products as zeros (0 x inf would reach
            // the other rows too): what they add to the rows that see them is added here.
            wave_sync();
            for (int k = 0; k < 2; ++k)
                for (uint64_t odd = k ? odd_of[1] : odd_of[0]; odd; odd &= odd - 1) {
                    const int at_pos = (hidden + k) * pl.tile_keys + wv * KEYS + __ffsll((unsigned long long)odd) - 1;
                    const int at_page = page_of(b, s, at_pos);
                    if (at_page < 0) continue;
                    const long row = pool_row(b, at_page, h, at_pos);
                    for (int r = max(0, at_pos - (sq.len - sq.n)) * G; r < rows; ++r) {   // the rows from that position on
                        const T *qr = reinterpret_cast<const T *>(a.Q) + (sq.row0 + r / G) * a.q_row + (h * G + r % G) * a.q_head;
                        float x = 0.f;
                        for (int c = lane; c < b.d; c += kWave) x = fmaf(to_float(qr[c]), cached_value<T, FORM>(a.Kpages, row * b.d + c), x);
                        x = wave_sum(x) * a.c;
                        if (FORM != kPagesPlain) x *= a.Kscale[row];
                        float w = __builtin_amdgcn_exp2f(x - __shfl(shift, r, kWave));
                        if (FORM != kPagesPlain) w *= a.Vscale[row];
                        for (int c = lane; c < b.d; c += kWave)
                            parts[(wv * rows + r) * (D + 4) + c] += w * cached_value<T, FORM>(a.Vpages, row * b.d + c);
                    }
                }
        }
        const bool whole = t0 == 0 && t1 == (int)per_head;
        const int slot_at = 2 * blockIdx.x + (tile == mine ? 0 : 1);
        if (tid == 0 && t0 == 0 && !whole)
            pl.join.records[blockIdx.x] = {stretch_owner(total, tile + per_head - 1, n_wg) - (int)blockIdx.x + 1, slot_at, sq.row0, h, 0, rows};
        float *slot = pl.join.slots + (size_t)slot_at * pl.join.slot_floats;
        float *stat = slot + pl.join.slot_rows * D;
        float *sums = ml + 256 + 4 * rows * (D + 4);   // [rows]
        if (wv == 0 && hh == 0 && l32 < rows) {
            sums[l32] = sum;
            if (!whole) { stat[2 * l32] = top; stat[2 * l32 + 1] = sum; }
            else if (a.lse) a.lse[(long)(sq.row0 + l32 / G) * b.H * G + h * G + l32 % G] = lse_of(top, sum);
        }
        __syncthreads();
        for (int e = tid; e < rows * (D / 4); e += 256) {
            const int r = e / (D / 4), c4 = 4 * (e % (D / 4));
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float4 y = *reinterpret_cast<const float4 *>(parts + (w * rows + r) * (D + 4) + c4);
                v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w;
            }
            if (!whole) {
                *reinterpret_cast<float4 *>(slot + r * D + c4) = v;
            } else if (c4 < b.d) {
                const float f = inverse_of(sums[r]);
                T *to = reinterpret_cast<T *>(a.out) + (sq.row0 + r / G) * a.o_row + (h * G + r % G) * a.o_head + c4;
                if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(to) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
                else *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(v.x * f, v.y * f), pack_bf16(v.z * f, v.w * f));
            }
        }
        __syncthreads();
        tile += t1 - t0;
    }
}

// 32-key blocks of a wave's share of a tile: as many as put 8 KiB of keys in flight.  (fp32 rows of 64, us, two blocks, which leave one workgroup a compute
// unit for their registers, / one: a token over 65536 keys 89 / 73, 64 tokens over 1000 to 5000 231 / 176.)
constexpr int few_blocks(int D, bool wide_rows) { return D <= 64 && !wide_rows ? 2 : 1; }   // wide_rows: cached in 32 bits
template <typename T, int FORM, int D> constexpr int blocks_of() { return few_blocks(D, FORM == kPagesPlain && sizeof(T) == 4); }

template <typename T, int FORM, int D>
hipError_t go_few(const AttendArgs &a, const FewPlan &pl, hipStream_t st)
{
    constexpr int NB = blocks_of<T, FORM, D>();
    using P = WavePlace<T, FORM, D, NB>;
    const int tiles = 4 * P::kBytes + 32 * P::kPitch;
    const int joined = (256 + 4 * pl.join.slot_rows * (D + 4) + pl.join.slot_rows) * 4;
    const int lds = tiles > joined ? tiles : joined;
    auto kernel = attend_few_kernel<T, FORM, D, NB>;
    if (lds > 64 * 1024 && !allow_big_lds(reinterpret_cast<const void *>(kernel))) return hipErrorInvalidValue;
    kernel<<<pl.join.n_wg, 256, lds, st>>>(a, pl);
    return hipGetLastError();
}

template <typename T, int FORM> hipError_t go_few_d(const AttendArgs &a, const FewPlan &pl, hipStream_t st)
{
    if (a.b.d <= 64) return go_few<T, FORM, 64>(a, pl, st);
    if constexpr (sizeof(T) == 2)
        if (a.b.d > 128) return go_few<T, FORM, 256>(a, pl, st);
    return go_few<T, FORM, 128>(a, pl, st);
}

}  // namespace

bool attend_mfma_applies(int dtype, int d) { return d <= (dtype == 0 ? 128 : 256); }   // (32-bit rows of 256 would fill the LDS)

FewPlan few_plan(const PagedBatch &b, int dtype, int form, int G)
{
    const int D = attend_width(b.d);
    FewPlan p{};
    p.tile_keys = 4 * 32 * few_blocks(D, form == kPagesPlain && dtype == 0);
    const long rows = (long)b.max_rows * G;
    p.join.slot_rows = rows < kFewRows ? (int)rows : kFewRows;
    p.join.slot_floats = (p.join.slot_rows * (D + 2) + 3) & ~3;
    p.join.rows_per_wg = 1;
    const long cap = (((long)b.table_pages << b.page_shift) + p.tile_keys - 1) / p.tile_keys * b.H * b.n_seqs;
    p.join.n_wg = cap < kMostFewWorkgroups ? (int)cap : kMostFewWorkgroups;
    return p;
}

hipError_t launch_attend_few(const AttendArgs &a, const FewPlan &pl, int dtype, int form, hipStream_t st)
{
    if (dtype == 0)
        return form == kPagesPlain ? go_few_d<float, kPagesPlain>(a, pl, st)
             : form == kPagesFp8   ? go_few_d<float, kPagesFp8>(a, pl, st) : go_few_d<float, kPagesInt8>(a, pl, st);
    return form == kPagesPlain ? go_few_d<uint16_t, kPagesPlain>(a, pl, st)
         : form == kPagesFp8   ? go_few_d<uint16_t, kPagesFp8>(a, pl, st) : go_few_d<uint16_t, kPagesInt8>(a, pl, st);
}

}  // namespace gkv
