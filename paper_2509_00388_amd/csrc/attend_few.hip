// Attention of sequences with few new rows (at most 32 stacked query rows a key-value head: one token of up to 32 query
// heads, eight drafted tokens of four): bound by the read of the keys and values.
//
// The tiles of all (sequence, head) pairs are cut into equal stretches, one a workgroup, whatever the lengths (attend.hpp).
// A tile's keys are dealt to the four waves; a wave brings its 32 NB keys and values through LDS of its own, with coalesced
// 16-byte loads of the next tile in flight while this one is multiplied, and keeps its own running maximum, sum and O^T:
// no barrier until the stretch of a pair ends and the waves' parts are joined.  A pair that one workgroup holds whole is
// finished there; the parts of others go to scratch memory and are joined by a second launch.
#include "attend_tile.hpp"
#include "kernels.hpp"

namespace gkv {

namespace {

template <typename T, int FORM, int D, int NB>
__global__ __launch_bounds__(256, (sizeof(T) == 4 || D > 128) ? 1 : 2) void attend_few_kernel(AttendArgs a, FewPlan pl)
{
    constexpr int KEYS = 32 * NB, DB = D / 32;
    using L = Tile<T, FORM, D, KEYS, 64>;
    constexpr int REGION = KEYS * (L::kKeyPitch > L::kValPitch ? L::kKeyPitch : L::kValPitch);   // keys, then values
    constexpr int WAVE = REGION + (FORM == kPagesPlain ? 0 : 2 * KEYS * 4);
    constexpr uint64_t kAllKeys = KEYS == 64 ? ~0ull : (1ull << KEYS) - 1;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint32_t part[16];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hh = lane >> 5;
    unsigned char *kv = smem + wv * WAVE;
    float *ks = reinterpret_cast<float *>(kv + REGION), *vs = ks + KEYS;
    const PagedBatch &b = a.b;

    auto weight = [&](int i) { return few_tiles(seq_rows(b, i), a, pl) * b.H; };
    uint32_t before;
    const uint32_t total = weigh(b.n_seqs, 0, before, part, weight);
    const int n_wg = (int)min((uint32_t)pl.n_wg, total);
    if ((int)blockIdx.x >= n_wg) return;
    uint32_t tile = few_first(total, blockIdx.x, n_wg);
    const uint32_t last = few_first(total, blockIdx.x + 1, n_wg);
    int s = find_unit(b.n_seqs, tile, before, part, weight);
    const uint32_t mine = tile;
    const int pieces = b.d * L::kCached / 16, my_piece = lane % L::kPieces, my_row = lane / L::kPieces;
    const int load_piece = min(my_piece, pieces - 1);
    const bool pad = my_piece >= pieces;

    while (tile < last) {
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

        // this lane's query: stacked row l32
        const int token = l32 / a.G, head = h * a.G + l32 % a.G;
        const T *qrow = l32 < rows ? reinterpret_cast<const T *>(a.Q) + (sq.row0 + token) * a.q_row + head * a.q_head : nullptr;
        uint4 q[L::kSteps];
        load_query<T>(qrow, b.d, hh, q);
        const int sees = sq.len - sq.n + token;   // last position it sees

        float m = -INFINITY, l = 0.f;
        f32x16 o[DB];
#pragma unroll
        for (int x = 0; x < DB; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[x][i] = 0.f;

        // Where the wave's keys of a tile lie: lane j looks key j up (lanes beyond KEYS repeat them).
        const int my_key = wv * KEYS + (lane & (KEYS - 1));
        auto entry = [&](int t) {   // page of the lane's key in tile t, -1: none
            const int pos = t * pl.tile_keys + my_key;
            return t < t1 && pos < sq.len ? page_of(b, s, pos) : -1;
        };
        auto place = [&](int page, int t) { return page < 0 ? 0 : pool_row(b, page, h, t * pl.tile_keys + my_key); };
        uint4 kr[L::kPer], vr[L::kPer];
        float ksr = 0.f, vsr = 0.f;
        auto load = [&](const void *pages, int at, uint4 (&r)[L::kPer]) {
#pragma unroll
            for (int u = 0; u < L::kPer; ++u) {
                const int row = __shfl(at, my_row + u * L::kRowStep, kWave);
                r[u] = reinterpret_cast<const uint4 *>(pages)[(long)row * pieces + load_piece];
            }
        };
        auto store = [&](const uint4 (&r)[L::kPer], int pitch, uint64_t vis) {
#pragma unroll
            for (int u = 0; u < L::kPer; ++u) {
                const int row = my_row + u * L::kRowStep;
                // (places that hold no key of the sequence may hold anything: zeros instead)
                L::put(kv + row * pitch + my_piece * (16 / L::kCached) * (int)sizeof(T), r[u],
                       pad || (vis != kAllKeys && !((vis >> row) & 1)));
            }
        };
        int page = entry(t0), at = place(page, t0);
        uint64_t vis = __ballot(page >= 0) & kAllKeys;
        load(a.Kpages, at, kr);
        if (FORM != kPagesPlain) { ksr = a.Kscale[at]; vsr = a.Vscale[at]; }
        load(a.Vpages, at, vr);
        int page1 = entry(t0 + 1);

        for (int t = t0; t < t1; ++t) {
            const int page2 = entry(t + 2), at1 = place(page1, t + 1);
            const uint64_t vis1 = __ballot(page1 >= 0) & kAllKeys;
            const int first = t * pl.tile_keys + wv * KEYS;
            const bool all = vis == kAllKeys && first + KEYS - 1 <= sq.len - sq.n;   // every row sees every key
            store(kr, L::kKeyPitch, vis);
            if (FORM != kPagesPlain) {
                if (lane < KEYS) {   // (a scale without a key may be anything too)
                    ks[lane] = page >= 0 ? ksr * a.c : 0.f;
                    vs[lane] = page >= 0 ? vsr : 0.f;
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
                    add_block(*reinterpret_cast<const uint4 *>(kv + (32 * n + l32) * L::kKeyPitch + 32 * st + 16 * hh), q[st], x[n], T{});
            }
            wave_sync();
            const uint64_t odd = all ? 0 : L::odd_rows(vr, 0) & vis;
            store(vr, L::kValPitch, vis & ~odd);
            load(a.Vpages, at1, vr);
            float p[NB][16];
            softmax_tile<FORM, NB, DB>(x, ks, a.c, all, vis, sees - first, hh, m, l, o, p);
            if constexpr (FORM != kPagesPlain) scale_weights<NB>(vs, all, sees - first, hh, p);
            wave_sync();
#pragma unroll
            for (int n = 0; n < NB; ++n) add_values<D, L::kValPitch>(kv + 32 * n * L::kValPitch, p[n], lane, o, T{});
            if (odd) add_odd_rows<T, FORM, NB, DB>(a.Vpages, odd, at, b.d, p, sees - first, lane, o);
            wave_sync();
            vis = vis1;
            at = at1;
            page = page1;
            page1 = page2;
        }

        // ---- the four waves' parts joined --------------------------------------------------------
        l = other_half_sum(l);
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
        const bool whole = t0 == 0 && t1 == (int)per_head;
        float *slot = pl.slots + (size_t)(2 * blockIdx.x + (tile == mine ? 0 : 1)) * pl.slot_floats;
        float *stat = slot + pl.slot_rows * D;
        float *sums = ml + 256 + 4 * rows * (D + 4);   // [rows]
        if (wv == 0 && hh == 0 && l32 < rows) {
            sums[l32] = sum;
            if (!whole) { stat[2 * l32] = top; stat[2 * l32 + 1] = sum; }
            else if (a.lse) a.lse[(long)(sq.row0 + token) * b.H * a.G + head] = lse_of(top, sum);
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
                T *to = reinterpret_cast<T *>(a.out) + (sq.row0 + r / a.G) * a.o_row + (h * a.G + r % a.G) * a.o_head + c4;
                if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(to) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
                else *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(v.x * f, v.y * f), pack_bf16(v.z * f, v.w * f));
            }
        }
        __syncthreads();
        tile += t1 - t0;
    }
}

// The parts of pairs that several workgroups held: a workgroup a (row, key-value head).
template <typename T, int D>
__global__ __launch_bounds__(256) void attend_join_few_kernel(AttendArgs a, FewPlan pl)
{
    __shared__ uint32_t part[16];
    const PagedBatch &b = a.b;
    const int row = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
    const int s = seq_of_row(b, row, tid & 63);
    if (s >= b.n_seqs) return;
    const SeqRows sq = seq_rows(b, s);
    if (row < sq.row0 || row >= sq.row0 + sq.n) return;
    const uint32_t per_head = few_tiles(sq, a, pl);
    if (per_head == 0) return;
    uint32_t before;
    const uint32_t total = weigh(b.n_seqs, s, before, part, [&](int i) { return few_tiles(seq_rows(b, i), a, pl) * b.H; });
    const int n_wg = (int)min((uint32_t)pl.n_wg, total);
    const uint32_t first = before + h * per_head, end = first + per_head;
    const int w0 = few_owner(total, first, n_wg), w1 = few_owner(total, end - 1, n_wg);
    if (w0 == w1) return;   // finished where it was computed
    for (int e = tid; e < a.G * (D / 4); e += 256) {
        const int g = e / (D / 4), c4 = 4 * (e % (D / 4)), r = (row - sq.row0) * a.G + g;
        // (a workgroup that starts within this pair holds it in its first stretch, one that came from another pair in its last)
        auto slot_of = [&](int w) {
            return pl.slots + (size_t)(2 * w + (few_first(total, w, n_wg) >= first ? 0 : 1)) * pl.slot_floats;
        };
        float top = -INFINITY;
        for (int w = w0; w <= w1; ++w) top = fmaxf(top, slot_of(w)[pl.slot_rows * D + 2 * r]);
        const float shift = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = w0; w <= w1; ++w) {
            const float *p = slot_of(w);
            const float f = __builtin_amdgcn_exp2f(p[pl.slot_rows * D + 2 * r] - shift);
            const float4 y = *reinterpret_cast<const float4 *>(p + r * D + c4);
            sum = fmaf(p[pl.slot_rows * D + 2 * r + 1], f, sum);
            v.x = fmaf(y.x, f, v.x); v.y = fmaf(y.y, f, v.y); v.z = fmaf(y.z, f, v.z); v.w = fmaf(y.w, f, v.w);
        }
        if (a.lse && c4 == 0) a.lse[(long)row * b.H * a.G + h * a.G + g] = lse_of(top, sum);
        if (c4 >= b.d) continue;
        const float f = inverse_of(sum);
        T *to = reinterpret_cast<T *>(a.out) + row * a.o_row + (h * a.G + g) * a.o_head + c4;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(to) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
        else *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(v.x * f, v.y * f), pack_bf16(v.z * f, v.w * f));
    }
}

// 32-key blocks of a wave's share of a tile: as many as put 8 KiB of keys in flight.
template <typename T, int FORM, int D> constexpr int blocks_of() { return D * Tile<T, FORM, 64, 64, 64>::kCached <= 128 ? 2 : 1; }

template <typename T, int FORM, int D>
hipError_t go_few(const AttendArgs &a, const FewPlan &pl, hipStream_t st)
{
    constexpr int NB = blocks_of<T, FORM, D>(), KEYS = 32 * NB;
    using L = Tile<T, FORM, D, KEYS, 64>;
    const int wave = KEYS * (L::kKeyPitch > L::kValPitch ? L::kKeyPitch : L::kValPitch) + (FORM == kPagesPlain ? 0 : 8 * KEYS);
    const int joined = (256 + 4 * pl.slot_rows * (D + 4) + pl.slot_rows) * 4;
    const int lds = 4 * wave > joined ? 4 * wave : joined;
    auto kernel = attend_few_kernel<T, FORM, D, NB>;
    if (lds > 64 * 1024 && !allow_big_lds(reinterpret_cast<const void *>(kernel))) return hipErrorInvalidValue;
    kernel<<<pl.n_wg, 256, lds, st>>>(a, pl);
    return hipGetLastError();
}

template <typename T, int FORM> hipError_t go_few_d(const AttendArgs &a, const FewPlan &pl, hipStream_t st)
{
    return a.b.d <= 64 ? go_few<T, FORM, 64>(a, pl, st) : a.b.d <= 128 ? go_few<T, FORM, 128>(a, pl, st) : go_few<T, FORM, 256>(a, pl, st);
}

}  // namespace

bool attend_mfma_applies(int d) { return d <= 256; }

FewPlan few_plan(const PagedBatch &b, int dtype, int form, int G)
{
    const int D = attend_width(b.d), cached = form != kPagesPlain ? 1 : dtype == 0 ? 4 : 2;
    FewPlan p{};
    p.tile_keys = 4 * 32 * (D * cached <= 128 ? 2 : 1);
    const long rows = (long)b.max_rows * G;
    p.slot_rows = rows < kFewRows ? (int)rows : kFewRows;
    p.slot_floats = (p.slot_rows * (D + 2) + 3) & ~3;
    const long cap = (((long)b.table_pages << b.page_shift) + p.tile_keys - 1) / p.tile_keys * b.H * b.n_seqs;
    const int most = 512;   // two workgroups a compute unit
    p.n_wg = cap < most ? (int)cap : most;
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

hipError_t launch_attend_join_few(const AttendArgs &a, const FewPlan &pl, int dtype, hipStream_t st)
{
    const dim3 grid(a.b.n_rows, a.b.H);
    const int D = attend_width(a.b.d);
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(a, pl); return hipGetLastError(); };
    if (dtype == 0)
        return D == 64 ? go(attend_join_few_kernel<float, 64>) : D == 128 ? go(attend_join_few_kernel<float, 128>) : go(attend_join_few_kernel<float, 256>);
    return D == 64 ? go(attend_join_few_kernel<uint16_t, 64>) : D == 128 ? go(attend_join_few_kernel<uint16_t, 128>) : go(attend_join_few_kernel<uint16_t, 256>);
}

}  // namespace gkv
