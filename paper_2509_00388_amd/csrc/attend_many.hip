// Attention of sequences with many new rows (drafts of wide groups, chunks of a prompt): bound by the matrix cores and the
// exponentials, with few blocks of rows by the read of the keys and values.
//
// A workgroup of four waves takes a block of 32 RG stacked query rows of a head, 32 of them a wave in operand registers, and
// streams the keys and values that they see through the LDS in tiles: the next tile's loads are in flight, in registers, while
// this one is multiplied, and go to the other half of the LDS behind it; one barrier a tile.  With RG = 4 every wave
// multiplies the whole tile; with RG = 2, for sequences of at most 64 stacked rows, two waves share a group of rows and take half
// the tile's keys each, and their sums are joined at the end.  Logits stay in registers: each wave turns its 32 x 32 NB of
// them into weights and multiplies them with the values (attend_tile.hpp).  The work is cut into equal stretches, whatever
// the lengths (attend.hpp); parts of blocks that several workgroups hold are joined by a second launch.
//
// Measured: 16 sequences of eight tokens, seven query heads of each of four key heads, 1000 to 9000 keys of 128 in int8: 42 us, 2.9 TB/s, bound by the issue of
// vector instructions (27 a matrix instruction, a third of them decode); with two tiles on their way instead of one the same.  701 fp32 rows of 16 heads of 64
// over 2000 and over 5000 keys 206 us, 97 TFLOP/s of the 153 that a library product of 8192 cubed reaches.
#include "attend_tile.hpp"
#include "kernels.hpp"

namespace gkv {

namespace {

template <typename T, int FORM, int D, int NB, int RG>
__global__ __launch_bounds__(256, D * sizeof(T) > 256 ? 1 : 2) void attend_many_kernel(AttendArgs a, ManyPlan pl)
{
    constexpr int KS = 4 / RG, KEYS = 32 * NB * KS, DB = D / 32, R = 32 * RG;
    using L = Tile<T, FORM, D, KEYS, 256>;
    constexpr int KEYTILE = KEYS * L::kKeyPitch, HALF = KEYTILE + KEYS * L::kValPitch + (FORM == kPagesPlain ? 0 : 2 * KEYS * 4);
    constexpr uint64_t kAllKeys = KEYS == 64 ? ~0ull : (1ull << KEYS) - 1;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint32_t part[20];
    __shared__ unsigned long long odd_of[8];   // of the tiles that some rows do not see all of: values with infinities or NaN
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hh = lane >> 5;
    const int group = wv % RG, stream = wv / RG, key0 = 32 * NB * stream;   // the wave's rows of the block, its first key of a tile
    const PagedBatch &b = a.b;

    uint32_t total, before, pos = 0, last = 0;
    int n_wg = 0, me = 0;
    int s = find_share<4>(b.n_seqs, total, before, part, [&](int i) { return many_seq(seq_rows(b, i), a, pl).per_head * b.H; },
                       [&](uint32_t all) {
                           const int id = blockIdx.x, xcd = id % 8;
                           n_wg = (int)min((uint32_t)pl.join.n_wg, all);
                           // Neighbouring stretches, which read the same keys at about the same time, to one XCD's workgroups.
                           me = id < n_wg ? xcd * (n_wg / 8) + min(xcd, n_wg % 8) + id / 8 : id;
                           if (tid == 0) pl.join.records[me].parts = 0;
                           if (id >= n_wg) return (int64_t)-1;
                           pos = stretch_first(all, me, n_wg);
                           last = stretch_first(all, me + 1, n_wg);
                           return (int64_t)pos;
                       });
    if (s < 0) return;
    const uint32_t mine = pos;

    const int pieces = b.d * L::kCached / 16, my_piece = tid % L::kPieces, my_row = tid / L::kPieces;
    const int wave_row = __builtin_amdgcn_readfirstlane(my_row);
    const int load_piece = min(my_piece, pieces - 1);
    const bool pad = my_piece >= pieces;
    const int my_key = lane & (KEYS - 1);   // lane j of each wave looks key j of a tile up

    ManyPart mp;
    while (next_part(a, pl, pos, last, s, before, mp)) {
        const SeqRows sq = mp.sq;
        const int h = mp.h, rows = mp.rows;
        const uint32_t u0 = mp.u0, u1 = mp.u1, units = mp.units;
        const int row0 = mp.block * R;                                                  // stacked rows of the sequence
        const int row = row0 + 32 * group + l32;
        const int sees = sq.len - sq.n + row / a.G;                                  // last position the lane's row sees
        const int extent = max(0, sq.len - sq.n + (min(row0 + R, rows) - 1) / a.G + 1);   // positions the block sees
        const int first_sees = sq.len - sq.n + row0 / a.G;                           // last position that all its rows see
        const int hidden = max(0, first_sees + 1) / KEYS;                            // the first tile that not all of them see all of
        const int t0 = (int)u0 * pl.step, t1 = min((int)u1 * pl.step, (extent + KEYS - 1) / KEYS);

        auto query = [&](int G) {
            return row < rows ? reinterpret_cast<const T *>(a.Q) + (sq.row0 + row / G) * a.q_row + (h * G + row % G) * a.q_head : nullptr;
        };
        uint4 q[L::kSteps];
        load_query<T>(query(a.G), b.d, hh, q);

        float m = -INFINITY, l = 0.f;
        f32x16 o[DB];
#pragma unroll
        for (int x = 0; x < DB; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[x][i] = 0.f;

        auto entry = [&](int t) {
            const int at = t * KEYS + my_key;
            return t < t1 && at < extent ? raw_page(b, s, at) : -1;
        };
        auto place = [&](int page, int t) { return !is_page(b, page) ? 0 : pool_row(b, page, h, t * KEYS + my_key); };
        uint4 kr[L::kPer], vr[L::kPer];
        float ksr = 0.f, vsr = 0.f;
        auto load = [&](int at) {
#pragma unroll
            for (int u = 0; u < L::kPer; ++u) {
                const long r = __builtin_amdgcn_ds_bpermute(4 * my_row + 4 * u * L::kRowStep, at);   // of lane my_row + u * kRowStep
                kr[u] = reinterpret_cast<const uint4 *>(a.Kpages)[r * pieces + load_piece];
                vr[u] = reinterpret_cast<const uint4 *>(a.Vpages)[r * pieces + load_piece];
            }
            if (FORM != kPagesPlain) { ksr = a.Kscale[at]; vsr = a.Vscale[at]; }
        };
        auto store = [&](int t, int page, uint64_t vis) {
            unsigned char *kt = smem + (t & 1) * HALF + my_row * L::kKeyPitch + my_piece * L::kDecoded;
            unsigned char *vt = smem + (t & 1) * HALF + KEYTILE + my_row * L::kValPitch + my_piece * L::kDecoded;
            uint64_t odd = 0;
            if (t * KEYS + KEYS - 1 > first_sees) {   // some rows do not see all of it
                odd = L::odd_rows(vr, wave_row) & vis;
                if (odd && lane == 0) atomicOr(&odd_of[t - hidden], (unsigned long long)odd);
            }
            // (places that hold no key of the sequence may hold anything: zeros instead)
            const uint64_t kseen = pad ? 0 : vis >> my_row, vseen = pad ? 0 : (vis & ~odd) >> my_row;
#pragma unroll
            for (int u = 0; u < L::kPer; ++u) {
                L::put(kt + u * L::kRowStep * L::kKeyPitch, L::only(kr[u], (kseen >> (u * L::kRowStep)) & 1));
                L::put(vt + u * L::kRowStep * L::kValPitch, L::only(vr[u], (vseen >> (u * L::kRowStep)) & 1));
            }
            if (FORM != kPagesPlain && wv == 0 && lane < KEYS) {
                float *ks = reinterpret_cast<float *>(smem + (t & 1) * HALF + KEYTILE + KEYS * L::kValPitch);
                ks[lane] = is_page(b, page) ? ksr * a.c : 0.f;
                ks[KEYS + lane] = is_page(b, page) ? vsr : 0.f;
            }
        };
        __syncthreads();   // (the part before is done with them)
        if (tid < 8) odd_of[tid] = 0;
        int page = entry(t0), at = place(page, t0), page1 = entry(t0 + 1);
        uint64_t vis = __ballot(is_page(b, page)) & kAllKeys;
        load(at);
        __syncthreads();
        store(t0, page, vis);
        __syncthreads();
        for (int t = t0; t < t1; ++t) {
            const int at1 = place(page1, t + 1), page2 = entry(t + 2);
            const uint64_t vis1 = __ballot(is_page(b, page1)) & kAllKeys;
            load(at1);
            const unsigned char *kt = smem + (t & 1) * HALF + key0 * L::kKeyPitch, *vt = smem + (t & 1) * HALF + KEYTILE + key0 * L::kValPitch;
            const float *ks = reinterpret_cast<const float *>(smem + (t & 1) * HALF + KEYTILE + KEYS * L::kValPitch) + key0;
            const bool all = vis == kAllKeys && t * KEYS + KEYS - 1 <= first_sees;
            f32x16 x[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[n][i] = 0.f;
#pragma unroll
                for (int st = 0; st < L::kSteps; ++st)
                    add_block(*reinterpret_cast<const uint4 *>(kt + (32 * n + l32) * L::kKeyPitch + 32 * st + 16 * hh), q[st], x[n], T{});
            }
            float p[NB][16];
            const int limit = sees - t * KEYS - key0;
            const uint64_t seen = seen_keys(vis >> key0, limit, hh);
            softmax_tile<FORM, NB, DB>(x, ks, a.c, all, seen, hh, m, l, o, p);
            if constexpr (FORM != kPagesPlain) scale_weights<NB>(ks + KEYS, all, seen, hh, p);
#pragma unroll
            for (int n = 0; n < NB; ++n) add_values<D, L::kValPitch>(vt + 32 * n * L::kValPitch, p[n], lane, o, T{});
            store(t + 1, page1, vis1);
            __syncthreads();
            vis = vis1;
            at = at1;
            page1 = page2;
        }

        l = other_half_sum(l);
        int G = a.G;
        asm volatile("" : "+s"(G));   // (what was computed from it before the loop is not kept through it)
        if (FORM != kPagesInt8)
            for (int t = max(t0, hidden); t < t1; ++t)
                if (const uint64_t odd = odd_of[t - hidden] >> key0 & (~0ull >> (64 - 32 * NB)))
                    add_odd_rows<T, FORM, DB>(a, s, h, odd, t * KEYS + key0, query(G), sq.len - sq.n + row / G, m, hh, o);
        if constexpr (KS > 1) {
            // the second stream's sums to the first: [RG][32] maxima and sums, [RG][32][D + 4]
            float *ml = reinterpret_cast<float *>(smem), *sums = ml + 64 * RG + (group * 32 + l32) * (D + 4) + 4 * hh;
            if (stream == 1) {
                if (hh == 0) { ml[2 * (group * 32 + l32)] = m; ml[2 * (group * 32 + l32) + 1] = l; }
#pragma unroll
                for (int x = 0; x < DB; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<float4 *>(sums + 32 * x + 8 * j) =
                            make_float4(o[x][4 * j], o[x][4 * j + 1], o[x][4 * j + 2], o[x][4 * j + 3]);
            }
            __syncthreads();
            if (stream == 0) {
                const float m1 = ml[2 * (group * 32 + l32)], l1 = ml[2 * (group * 32 + l32) + 1], top = fmaxf(m, m1);
                const float shift = top == -INFINITY ? 0.f : top;
                const float f = __builtin_amdgcn_exp2f(m - shift), f1 = __builtin_amdgcn_exp2f(m1 - shift);
                m = top;
                l = l * f + l1 * f1;
#pragma unroll
                for (int x = 0; x < DB; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float4 y = *reinterpret_cast<const float4 *>(sums + 32 * x + 8 * j);
                        o[x][4 * j] = o[x][4 * j] * f + y.x * f1;
                        o[x][4 * j + 1] = o[x][4 * j + 1] * f + y.y * f1;
                        o[x][4 * j + 2] = o[x][4 * j + 2] * f + y.z * f1;
                        o[x][4 * j + 3] = o[x][4 * j + 3] * f + y.w * f1;
                    }
            }
            __syncthreads();   // (the next block's tiles come to this place)
        }
        if (tid == 0 && u0 == 0 && u1 < units)
            pl.join.records[me] = {stretch_owner(total, pos + units - 1, n_wg) - me + 1, 2 * me + (pos == mine ? 0 : 1), sq.row0, h, row0,
                                   min(R, rows - row0)};
        int r = 32 * group + l32;
        asm volatile("" : "+v"(r));   // (nor are the places of its results: fp8 rows of 128 in blocks of 128 rows spilled)
        if (stream == 0 && row0 + r < rows) {
            if (u0 > 0 || u1 < units) {
                float *slot = pl.join.slots + (size_t)(2 * me + (pos == mine ? 0 : 1)) * pl.join.slot_floats;
                if (hh == 0) { slot[R * D + 2 * r] = m; slot[R * D + 2 * r + 1] = l; }
#pragma unroll
                for (int x = 0; x < DB; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<float4 *>(slot + r * D + 32 * x + 8 * j + 4 * hh) =
                            make_float4(o[x][4 * j], o[x][4 * j + 1], o[x][4 * j + 2], o[x][4 * j + 3]);
            } else {
                const int token = (row0 + r) / G, head = h * G + (row0 + r) % G;
                if (a.lse && hh == 0) a.lse[(long)(sq.row0 + token) * b.H * G + head] = lse_of(m, l);
                const float f = inverse_of(l);
                T *to = reinterpret_cast<T *>(a.out) + (sq.row0 + token) * a.o_row + head * a.o_head;
#pragma unroll
                for (int x = 0; x < DB; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int c = 32 * x + 8 * j + 4 * hh;
                        if (c >= b.d) continue;
                        if constexpr (sizeof(T) == 4)
                            *reinterpret_cast<float4 *>(to + c) = make_float4(o[x][4 * j] * f, o[x][4 * j + 1] * f, o[x][4 * j + 2] * f, o[x][4 * j + 3] * f);
                        else
                            *reinterpret_cast<uint2 *>(to + c) = make_uint2(pack_bf16(o[x][4 * j] * f, o[x][4 * j + 1] * f),
                                                                            pack_bf16(o[x][4 * j + 2] * f, o[x][4 * j + 3] * f));
                    }
            }
        }
        pos += u1 - u0;
    }
}

// Keys of a tile: 64, where the LDS holds two such tiles for two workgroups, otherwise 32.
template <typename T, int D> constexpr int many_tile_keys() { return D * (int)sizeof(T) <= 256 ? 64 : 32; }

template <typename T, int FORM, int D, int RG>
hipError_t go_many_rows(const AttendArgs &a, const ManyPlan &pl, hipStream_t st)
{
    constexpr int KEYS = many_tile_keys<T, D>(), NB = KEYS * RG / 128;
    using L = Tile<T, FORM, D, KEYS, 256>;
    const int tiles = 2 * (KEYS * (L::kKeyPitch + L::kValPitch) + (FORM == kPagesPlain ? 0 : 8 * KEYS));
    const int joined = RG == 4 ? 0 : (64 * RG + 32 * RG * (D + 4)) * 4;
    const int lds = tiles > joined ? tiles : joined;
    auto kernel = attend_many_kernel<T, FORM, D, NB, RG>;
    if (lds > 64 * 1024 && !allow_big_lds(reinterpret_cast<const void *>(kernel))) return hipErrorInvalidValue;
    kernel<<<pl.join.n_wg, 256, lds, st>>>(a, pl);
    return hipGetLastError();
}

template <typename T, int FORM, int D>
hipError_t go_many(const AttendArgs &a, const ManyPlan &pl, hipStream_t st)
{
    if constexpr (many_tile_keys<T, D>() == 64)
        if (pl.block_rows == 64) return go_many_rows<T, FORM, D, 2>(a, pl, st);
    return go_many_rows<T, FORM, D, 4>(a, pl, st);
}

template <typename T, int FORM> hipError_t go_many_d(const AttendArgs &a, const ManyPlan &pl, hipStream_t st)
{
    if (a.b.d <= 64) return go_many<T, FORM, 64>(a, pl, st);
    if constexpr (sizeof(T) == 2)
        if (a.b.d > 128) return go_many<T, FORM, 256>(a, pl, st);
    return go_many<T, FORM, 128>(a, pl, st);
}

}  // namespace

ManyPlan many_plan(const PagedBatch &b, int dtype, int G, bool leave_few)
{
    const int D = attend_width(b.d);
    ManyPlan p{};
    p.leave_few = leave_few;
    p.tile_keys = D * (dtype == 0 ? 4 : 2) <= 256 ? 64 : 32;
    // (us, blocks of 256 rows and of 128, one sequence of so many rows of eight key heads of four over 8000 tokens: 160 36.2 / 40.2, 256 39.5 /
    // 42.9, 800 57.2 / 66.1, 2000 102 / 111; 8 sequences of 256 over 4000 72.5 / 103.  Blocks of 64 rows and of 128: 16 sequences of 64 over
    // 8000 tokens 122 / 127.)
    const long most_rows = (long)b.max_rows * G;
    p.wide = dtype != 0 && D <= 128 && most_rows > 128;
    p.block_rows = p.wide ? 256 : p.tile_keys == 64 && most_rows <= 64 ? 64 : 128;
    p.join.slot_rows = p.block_rows;
    p.join.slot_floats = p.block_rows * (D + 2);
    p.join.rows_per_wg = 8;
    const long blocks = (long)b.n_rows * G / p.block_rows + b.n_seqs;   // at least those of all sequences
    // Units of 256 keys with blocks of 64 rows, of 128 with larger ones, of 64 in fp32, whose tiles take longest; more where their
    // number could pass 31 bits.  Shorter units share the work out better, longer ones leave fewer parts to be joined.  (us, units of
    // 256 / 128 keys, eight key heads of four but for the last: 4 sequences of 12 rows over 2000 tokens 23 / 28, 500 rows over 8000 107 / 103, 500 over 500
    // 32 / 29; fp32, 256 / 64 keys: 701 rows over 3000 and over 5000 tokens 962 / 888, 256 rows over 2000 117 / 122, d = 64 and eight
    // heads, 300 over 900 34 / 30.)
    const long cap = (long)b.table_pages << b.page_shift;
    long units = 0;
    const int keys = p.block_rows == 64 ? 256 : dtype == 0 ? 64 : 128;
    for (p.step = keys / p.tile_keys;; p.step *= 2) {
        units = (blocks / 2 + b.n_seqs) * (2 * (cap / ((long)p.tile_keys * p.step) + 1) + 2) * b.H;
        if (units <= INT32_MAX || p.tile_keys * p.step >= 1 << 29) break;
    }
    const int most = p.wide ? 256 : 512;   // one or two workgroups a compute unit
    p.join.n_wg = units > INT32_MAX ? 0 : units < most ? (int)units : most;
    return p;
}

hipError_t launch_attend_many(const AttendArgs &a, const ManyPlan &pl, int dtype, int form, hipStream_t st)
{
    if (dtype == 0)
        return form == kPagesPlain ? go_many_d<float, kPagesPlain>(a, pl, st)
             : form == kPagesFp8   ? go_many_d<float, kPagesFp8>(a, pl, st) : go_many_d<float, kPagesInt8>(a, pl, st);
    return form == kPagesPlain ? go_many_d<uint16_t, kPagesPlain>(a, pl, st)
         : form == kPagesFp8   ? go_many_d<uint16_t, kPagesFp8>(a, pl, st) : go_many_d<uint16_t, kPagesInt8>(a, pl, st);
}

}  // namespace gkv
