// Attention of sequences with few new rows (at most 32 stacked query rows a key-value head: one token of up to 32 query
// heads, eight drafted tokens of four): bound by the read of the keys and values.
//
// The tiles of all (sequence, head) pairs are cut into equal stretches, one a workgroup, whatever the lengths (attend.hpp).
// A tile's keys are dealt to the four waves; a wave brings its 32 NB keys and values through LDS of its own, with coalesced
// 16-byte loads of the next tile in flight while this one is multiplied, and keeps its own running maximum, sum and O^T:
// no barrier until the stretch of a pair ends and the waves' parts are joined.  The stretch's next pair is looked up a pair ahead, and its first
// keys, values and queries are on their way while the parts are joined (64 tokens over 400 to 5000 keys 98.7 -> 91.3 us with a scale a row, 92.8 -> 86.2
// in blocks).  A pair that one workgroup holds whole is finished there; the parts of others go to scratch memory and are joined by a second launch.
//
// Measured (bf16 rows, d = 128, eight key heads of four, the kernel alone): one token over 131072 keys 97 us, 5.5 TB/s (reading alone is faster than the 4.6 to 4.8 of
// a copy); 64 tokens over 400 to 5000 keys each in fp8 pages 86 us, 4.5 TB/s, in blocks 80 to 83 us, 4.7 to 4.9; every pair that lies in two stretches costs
// some 5 us, which is why 64 tokens over 2816 keys each, a pair a stretch, take 71 us in blocks and 63 of them 84; one token over 2048 keys 8.7 us, a chain of look-ups,
// loads, two products and the join of the waves with a tile a workgroup.  States of d = 64, sixteen heads, 64 tokens over 200 to 1500 of them: 53 us, 4.2 TB/s.
// Slower: three workgroups a compute unit, 768 or 1024 of them in all (in blocks too: 64 tokens over 4096 keys 101 -> 127), 64 keys a wave.
#pragma once
#include "attend_tile.hpp"
#include "kernels.hpp"

namespace gkv {

namespace {

// A wave's place in the LDS: KEYS rows of keys, then of values, and the scales of both.
template <typename T, int FORM, int D, int NB> struct WavePlace {
    using L = Tile<T, FORM, D, 32 * NB, 64>;
    static constexpr int kPitch = L::kKeyPitch, kValues = L::kHalves ? L::kValPitch : kPitch, kRows = 32 * NB * kValues;   // kValues >= kPitch
    static constexpr int kBytes = kRows + (FORM == kPagesPlain || in_blocks(FORM) ? 0 : 2 * 32 * NB * 4);
};

#define GKV_KERNEL attend_few_kernel   // pages of rows, plain or with a scale each
#define GKV_CROSS false
#include "attend_few.inc"
#undef GKV_KERNEL
#undef GKV_CROSS
#define GKV_KERNEL blocks_few_kernel   // pages in blocks
#define GKV_CROSS false
#include "attend_few.inc"
#undef GKV_KERNEL
#undef GKV_CROSS
#define GKV_KERNEL cross_few_kernel   // rows that see all of a sequence
#define GKV_CROSS true
#include "attend_few.inc"
#undef GKV_KERNEL
#undef GKV_CROSS

template <typename T, int FORM, int D, int NB, bool CROSS> constexpr auto few_kernel()
{
    if constexpr (CROSS) return &cross_few_kernel<T, FORM, D, NB>;
    else if constexpr (in_blocks(FORM)) return &blocks_few_kernel<T, FORM, D, NB>;
    else return &attend_few_kernel<T, FORM, D, NB>;
}

// 32-key blocks of a wave's share of a tile: as many as put 8 KiB of keys in flight.  (fp32 rows of 64, us, two blocks, which leave one workgroup a compute
// unit for their registers, / one: a token over 65536 keys 89 / 73, 64 tokens over 1000 to 5000 231 / 176.)
constexpr int few_blocks(int D, bool wide_rows) { return D <= 64 && !wide_rows ? 2 : 1; }   // wide_rows: cached in 32 bits
template <typename T, int FORM, int D> constexpr int blocks_of() { return few_blocks(D, FORM == kPagesPlain && sizeof(T) == 4); }

template <typename T, int FORM, int D, bool CROSS>
hipError_t go_few(const AttendArgs &a, const FewPlan &pl, hipStream_t st)
{
    constexpr int NB = blocks_of<T, FORM, D>();
    using P = WavePlace<TileType<T, FORM>, FORM, D, NB>;
    const int tiles = 4 * P::kBytes + (in_thirds<T, FORM>() ? 3 : 1) * 32 * P::kPitch;
    const int joined = (256 + 4 * pl.join.slot_rows * (D + 4) + pl.join.slot_rows) * 4;
    const int lds = tiles > joined ? tiles : joined;
    auto kernel = few_kernel<T, FORM, D, NB, CROSS>();
    if (lds > 64 * 1024 && !allow_big_lds(reinterpret_cast<const void *>(kernel))) return hipErrorInvalidValue;
    kernel<<<pl.join.n_wg, 256, lds, st>>>(a, pl);
    return hipGetLastError();
}

template <typename T, int FORM, bool CROSS> hipError_t go_few_d(const AttendArgs &a, const FewPlan &pl, hipStream_t st)
{
    if (a.b.d <= 64) return go_few<T, FORM, 64, CROSS>(a, pl, st);
    if constexpr (sizeof(T) == 2)
        if (a.b.d > 128) return go_few<T, FORM, 256, CROSS>(a, pl, st);
    return go_few<T, FORM, 128, CROSS>(a, pl, st);
}
template <int FORM, bool CROSS> hipError_t few_of(const AttendArgs &a, const FewPlan &pl, int dtype, hipStream_t st)
{
    return dtype == 0 ? go_few_d<float, FORM, CROSS>(a, pl, st) : go_few_d<uint16_t, FORM, CROSS>(a, pl, st);
}

}  // namespace

}  // namespace gkv
