// Attention of sequences with more than 128 stacked rows, bf16 rows of up to 128 values: bound by the matrix cores and the
// vector instructions of the softmax, which this kernel keeps busy at the same time.
//
// A workgroup of eight waves, two on a SIMD, takes a block of 256 stacked query rows of a head, 32 a wave, and shares each tile of 64
// keys and values among all of them.  A wave's tile is one stretch of code without a barrier inside: the softmax of tile t, O^T += V^T P^T of
// tile t and S^T = K Q^T of tile t + 1, so that the sums of the softmax run beside the products, whose operands are
// read from the LDS some steps ahead, and the two waves of a SIMD fill one another's gaps.  The LDS holds three tiles: those two and the next,
// which the waves write, from registers, while nobody reads it; one barrier a tile.
// Measured (2048 rows of four query heads a key head over 32768 keys, eight key heads, d = 128, bf16; whole calls with their join of 10 us, one after
// the other): 1020 to 1100 us from card to card, 975 to 1050 TFLOP/s while the kernel runs; on a card where it takes 1095 a library product of 8192
// cubed reaches 1345, the kernel without its softmax took 850 us and without the reads of its operands from the LDS hardly less.  Slower, on one
// card where the kernel took 1060 to 1095: 128 rows a workgroup and two of them 1290; a barrier between softmax and products that keeps the waves of a SIMD
// half a tile apart 1090, with the operands' reads fixed by hand 1130, with tiles that pass the registers by (global_load_lds, pieces permuted
// instead of padded) 1130.
#include "attend_tile.hpp"
#include "kernels.hpp"

#include <type_traits>

namespace gkv {

namespace {

constexpr int kWideRows = 256, kTiles = 3;   // tiles in the LDS

template <int FORM, int D> struct WideTile {
    using L = Tile<uint16_t, FORM, D, 64, 512>;
    static constexpr int kKeys = 64 * L::kKeyPitch, kVals = 64 * L::kValPitch;
    static constexpr int kBytes = kKeys + kVals + (FORM == kPagesPlain ? 0 : 2 * 64 * 4);   // keys, values, their scales
};

template <int FORM, int D>
__global__ __launch_bounds__(512, 2) void attend_wide_kernel(AttendArgs a, ManyPlan pl)
{
    using T = uint16_t;
    using W = WideTile<FORM, D>;
    using L = typename W::L;
    constexpr int KEYS = 64, NB = 2, DB = D / 32, R = kWideRows;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint32_t part[20];
    __shared__ unsigned long long odd_of[8];   // of the tiles that some rows do not see all of: values with infinities or NaN
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hh = lane >> 5;
    const PagedBatch &b = a.b;

    uint32_t total, before, pos = 0, last = 0;
    int n_wg = 0, me = 0;
    int s = find_share<8>(b.n_seqs, total, before, part, [&](int i) { return many_seq(seq_rows(b, i), a, pl).per_head * b.H; },
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
    const int row_bytes = 16 * pieces;
    const bool together = 1 << b.page_shift >= L::kWaveRows;
    const uint32_t offset = (uint32_t)((my_row - wave_row) * row_bytes + 16 * min(my_piece, pieces - 1));
    const bool moves = !L::kSpare || wave_row < KEYS;   // (64 bytes a row: half of the waves have no piece of a tile)
    const int to_keys = my_row * L::kKeyPitch + my_piece * L::kDecoded, to_vals = W::kKeys + my_row * L::kValPitch + my_piece * L::kDecoded;
    if (pieces < L::kPieces) {   // columns that d does not reach stay zero
        for (int i = tid; i < kTiles * W::kBytes / 16; i += 512) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
    }

    ManyPart mp;
    while (next_part(a, pl, pos, last, s, before, mp)) {
        const SeqRows sq = mp.sq;
        const int h = mp.h, rows = mp.rows, row0 = mp.block * R, row = row0 + 32 * wv + l32;   // stacked rows of the sequence
        const int sees = sq.len - sq.n + row / a.G;                                          // last position the lane's row sees
        const int extent = max(0, sq.len - sq.n + (min(row0 + R, rows) - 1) / a.G + 1);      // positions the block sees
        const int first_sees = sq.len - sq.n + row0 / a.G;                                   // last position that all its rows see
        const int hidden = max(0, first_sees + 1) / KEYS;                                    // the first tile that not all of them see all of
        const int t0 = (int)mp.u0 * pl.step, t1 = min((int)mp.u1 * pl.step, (extent + KEYS - 1) / KEYS);

        auto query = [&](int G) {
            return row < rows ? reinterpret_cast<const T *>(a.Q) + (sq.row0 + row / G) * a.q_row + (h * G + row % G) * a.q_head : nullptr;
        };
        uint4 q[L::kSteps];
        load_query<T>(query(a.G), b.d, hh, q);
        float m = -INFINITY, l = 0.f;
        f32x16 o[DB], x[NB];
        Weights w[NB];
#pragma unroll
        for (int y = 0; y < DB; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[y][i] = 0.f;

        // Lane j of each wave looks key j of a tile up.
        auto entry = [&](int t) {
            const int at = t * KEYS + lane;
            return t < t1 && at < extent ? raw_page(b, s, at) : -1;
        };
        uint4 kr[L::kPer], vr[L::kPer];
        float scale = 0.f;   // of the key (wave 0) or value (wave 1) `lane`
        auto load = [&](int t, int page) {
            const int at = !is_page(b, page) ? 0 : pool_row(b, page, h, t * KEYS + lane);
            if (moves) {
                L::ask(a.Kpages, at, together, wave_row, my_row, row_bytes, offset, kr);
                L::ask(a.Vpages, at, together, wave_row, my_row, row_bytes, offset, vr);
            }
            if (FORM != kPagesPlain && wv < 2) scale = (wv == 0 ? a.Kscale : a.Vscale)[at];
        };
        auto store = [&](int t, uint64_t vis) {
            unsigned char *tile = smem + (t % kTiles) * W::kBytes;
            uint64_t odd = 0;
            if (moves && t * KEYS + KEYS - 1 > first_sees) {   // some rows do not see all of it
                odd = L::odd_rows(vr, wave_row) & vis;
                if (odd && lane == 0) atomicOr(&odd_of[t - hidden], (unsigned long long)odd);
            }
            if (vis != ~0ull || odd) {   // (places that hold no key of the sequence may hold anything: zeros instead)
                const uint64_t kseen = vis >> my_row, vseen = (vis & ~odd) >> my_row;
#pragma unroll
                for (int u = 0; u < L::kPer; ++u) {
                    kr[u] = L::only(kr[u], (kseen >> (u * L::kRowStep)) & 1);
                    vr[u] = L::only(vr[u], (vseen >> (u * L::kRowStep)) & 1);
                }
            }
            if (moves && my_piece < pieces) {
#pragma unroll
                for (int u = 0; u < L::kPer; ++u) {
                    L::put(tile + to_keys + u * L::kRowStep * L::kKeyPitch, kr[u]);
                    L::put(tile + to_vals + u * L::kRowStep * L::kValPitch, vr[u]);
                }
            }
            if (FORM != kPagesPlain && wv < 2)   // (a scale without a key may be anything too)
                reinterpret_cast<float *>(tile + W::kKeys + W::kVals)[64 * wv + lane] = (vis >> lane) & 1 ? (wv == 0 ? scale * a.c : scale) : 0.f;
        };
        // Logits of tile `next`, weights of tile `now` times its values, either of them or both.  The groups ask the scheduler for the operands of
        // two steps of each to be on their way while a step is multiplied (1060 -> 1095 us without).
        auto products = [&](auto with_values, int now, auto with_logits, int next) {
            constexpr bool PV = decltype(with_values)::value, QK = decltype(with_logits)::value;
            constexpr int STEPS = D / 8;   // of each: D / 16 steps of two key blocks, four steps of keys for D / 32 blocks of values
            typedef __attribute__((address_space(3))) bf16x4 lds4;
            const unsigned char *kt = smem + (next % kTiles) * W::kBytes + l32 * L::kKeyPitch + 16 * hh;
            const unsigned char *vt = smem + (now % kTiles) * W::kBytes + W::kKeys + (4 * hh + ((lane & 15) >> 2)) * L::kValPitch +
                                      ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
            if (QK) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[n][i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                if (QK) add_block(*reinterpret_cast<const uint4 *>(kt + 32 * (i & 1) * L::kKeyPitch + 32 * (i >> 1)), q[i >> 1], x[i & 1], T{});
                if (PV) {
                    const int key = 16 * (i / DB), n = key >> 5, st = (key >> 4) & 1, y = i % DB;
                    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(vt + key * L::kValPitch + 64 * y));
                    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(vt + (key + 8) * L::kValPitch + 64 * y));
                    o[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), w[n].w[st], o[y], 0, 0, 0);
                }
            }
            constexpr int reads = (QK ? 1 : 0) + (PV ? 2 : 0), each = (QK ? 1 : 0) + (PV ? 1 : 0), ahead = 2;
            __builtin_amdgcn_sched_group_barrier(0x100, ahead * reads, 0);   // (LDS reads)
#pragma unroll
            for (int i = 0; i < STEPS - ahead; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, each, 0);   // (matrix instructions)
                __builtin_amdgcn_sched_group_barrier(0x100, reads, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, ahead * each, 0);
        };
        constexpr std::true_type yes{};
        constexpr std::false_type no{};

        __syncthreads();   // (the tiles of the part before are done with)
        if (tid < 8) odd_of[tid] = 0;
        int page = entry(t0), page1 = entry(t0 + 1), page2 = entry(t0 + 2);
        uint64_t vis = __ballot(is_page(b, page)), vis1 = __ballot(is_page(b, page1)), vis2 = __ballot(is_page(b, page2));
        load(t0, page);
        __syncthreads();
        store(t0, vis);
        load(t0 + 1, page1);
        store(t0 + 1, vis1);
        load(t0 + 2, page2);
        page = entry(t0 + 3);
        __syncthreads();
        if (t0 < t1) {
            products(no, t0, yes, t0);
            for (int t = t0; t < t1; ++t) {
                __syncthreads();
                const uint64_t vis3 = __ballot(is_page(b, page));
                store(t + 2, vis2);
                load(t + 3, page);
                page = entry(t + 4);
                const float *ks = reinterpret_cast<const float *>(smem + (t % kTiles) * W::kBytes + W::kKeys + W::kVals);
                const bool all = vis == ~0ull && t * KEYS + KEYS - 1 <= first_sees;
                const uint64_t seen = seen_keys(vis, sees - t * KEYS, hh);
                float p[NB][16];
                softmax_tile<FORM, NB, DB>(x, ks, a.c, all, seen, hh, m, l, o, p);
                if constexpr (FORM != kPagesPlain) scale_weights<NB>(ks + KEYS, all, seen, hh, p);
#pragma unroll
                for (int n = 0; n < NB; ++n) w[n] = pack_weights(p[n]);
                vis = vis1;
                vis1 = vis2;
                vis2 = vis3;
                products(yes, t, yes, t + 1);   // (behind the last tile lies one of zeros: a way out between the two would cost the sums twice the registers)
            }
        }

        l = other_half_sum(l);
        int G = a.G;
        asm volatile("" : "+s"(G));   // (what was computed from it before the loop is not kept through it)
        if (FORM != kPagesInt8)
            for (int t = max(t0, hidden); t < t1; ++t)
                if (const uint64_t odd = odd_of[t - hidden])
                    add_odd_rows<T, FORM, DB>(a, s, h, odd, t * KEYS, query(G), sq.len - sq.n + row / G, m, hh, o);
        if (tid == 0 && mp.u0 == 0 && mp.u1 < mp.units)
            pl.join.records[me] = {stretch_owner(total, pos + mp.units - 1, n_wg) - me + 1, 2 * me + (pos == mine ? 0 : 1), sq.row0, h, row0,
                                   min(R, rows - row0)};
        const int r = 32 * wv + l32;
        if (row0 + r < rows) {
            if (mp.u0 > 0 || mp.u1 < mp.units) {
                float *slot = pl.join.slots + (size_t)(2 * me + (pos == mine ? 0 : 1)) * pl.join.slot_floats;
                if (hh == 0) { slot[R * D + 2 * r] = m; slot[R * D + 2 * r + 1] = l; }
#pragma unroll
                for (int y = 0; y < DB; ++y)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<float4 *>(slot + r * D + 32 * y + 8 * j + 4 * hh) =
                            make_float4(o[y][4 * j], o[y][4 * j + 1], o[y][4 * j + 2], o[y][4 * j + 3]);
            } else {
                const int token = (row0 + r) / G, head = h * G + (row0 + r) % G;
                if (a.lse && hh == 0) a.lse[(long)(sq.row0 + token) * b.H * G + head] = lse_of(m, l);
                const float f = inverse_of(l);
                T *to = reinterpret_cast<T *>(a.out) + (sq.row0 + token) * a.o_row + head * a.o_head;
#pragma unroll
                for (int y = 0; y < DB; ++y)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int c = 32 * y + 8 * j + 4 * hh;
                        if (c < b.d)
                            *reinterpret_cast<uint2 *>(to + c) = make_uint2(pack_bf16(o[y][4 * j] * f, o[y][4 * j + 1] * f),
                                                                            pack_bf16(o[y][4 * j + 2] * f, o[y][4 * j + 3] * f));
                    }
            }
        }
        pos += mp.u1 - mp.u0;
    }
}

template <int FORM, int D> hipError_t go_wide(const AttendArgs &a, const ManyPlan &pl, hipStream_t st)
{
    constexpr int lds = kTiles * WideTile<FORM, D>::kBytes;
    auto kernel = attend_wide_kernel<FORM, D>;
    if (lds > 64 * 1024 && !allow_big_lds(reinterpret_cast<const void *>(kernel), lds)) return hipErrorInvalidValue;
    kernel<<<pl.join.n_wg, 512, lds, st>>>(a, pl);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_wide(const AttendArgs &a, const ManyPlan &pl, int form, hipStream_t st)
{
    if (a.b.d <= 64)
        return form == kPagesPlain ? go_wide<kPagesPlain, 64>(a, pl, st)
             : form == kPagesFp8   ? go_wide<kPagesFp8, 64>(a, pl, st) : go_wide<kPagesInt8, 64>(a, pl, st);
    return form == kPagesPlain ? go_wide<kPagesPlain, 128>(a, pl, st)
         : form == kPagesFp8   ? go_wide<kPagesFp8, 128>(a, pl, st) : go_wide<kPagesInt8, 128>(a, pl, st);
}

}  // namespace gkv
