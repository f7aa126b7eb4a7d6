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
// over 2000 and over 5000 keys 206 us, 97 TFLOP/s of the 153 that a library product of 8192 cubed reaches.  In blocks of int8 the drafts take 41 us: a tile costs a fifth fewer vector
// instructions, but the two waves of a SIMD wait for one another's chains (products, softmax, products, decode, barrier); two tiles on their way, the decode
// between the products, units of one tile: 46.6, 47.0, 47.7 us a call against 47.3.
#pragma once
#include "attend_tile.hpp"
#include "kernels.hpp"

namespace gkv {

namespace {

// Bytes of a tile's scales in the LDS: two a key, or two for each of up to four groups of 16 keys.
constexpr int scale_bytes(int form, int keys) { return form == kPagesPlain ? 0 : in_blocks(form) ? 32 : 2 * keys * 4; }

// Bytes of the third part of a wave's queries in the LDS (attend_many.inc).
template <int D> constexpr int kThirdBytes = 32 * (2 * D + 16);

#define GKV_KERNEL attend_many_kernel   // pages of rows, plain or with a scale each
#define GKV_CROSS false
#include "attend_many.inc"
#undef GKV_KERNEL
#undef GKV_CROSS
#define GKV_KERNEL blocks_many_kernel   // pages in blocks
#define GKV_CROSS false
#include "attend_many.inc"
#undef GKV_KERNEL
#undef GKV_CROSS
#define GKV_KERNEL cross_many_kernel   // rows that see all of a sequence
#define GKV_CROSS true
#include "attend_many.inc"
#undef GKV_KERNEL
#undef GKV_CROSS

template <typename T, int FORM, int D, int NB, int RG, bool CROSS> constexpr auto many_kernel()
{
    if constexpr (CROSS) return &cross_many_kernel<T, FORM, D, NB, RG>;
    else if constexpr (in_blocks(FORM)) return &blocks_many_kernel<T, FORM, D, NB, RG>;
    else return &attend_many_kernel<T, FORM, D, NB, RG>;
}

// Keys of a tile: 64, where the LDS holds two such tiles for two workgroups, otherwise 32.
template <typename T, int D> constexpr int many_tile_keys() { return D * (int)sizeof(T) <= 256 ? 64 : 32; }

template <typename T, int FORM, int D, int RG, bool CROSS>
hipError_t go_many_rows(const AttendArgs &a, const ManyPlan &pl, hipStream_t st)
{
    constexpr int KEYS = many_tile_keys<T, D>(), NB = KEYS * RG / 128;
    using L = Tile<TileType<T, FORM>, FORM, D, KEYS, 256>;
    const int tiles = 2 * (KEYS * (L::kKeyPitch + L::kValPitch) + scale_bytes(FORM, KEYS)) + (in_thirds<T, FORM>() && D >= 128 ? 4 * kThirdBytes<D> : 0);
    const int joined = RG == 4 ? 0 : (64 * RG + 32 * RG * (D + 4)) * 4;
    const int lds = tiles > joined ? tiles : joined;
    auto kernel = many_kernel<T, FORM, D, NB, RG, CROSS>();
    if (lds > 64 * 1024 && !allow_big_lds(reinterpret_cast<const void *>(kernel))) return hipErrorInvalidValue;
    kernel<<<pl.join.n_wg, 256, lds, st>>>(a, pl);
    return hipGetLastError();
}

template <typename T, int FORM, int D, bool CROSS>
hipError_t go_many(const AttendArgs &a, const ManyPlan &pl, hipStream_t st)
{
    if constexpr (many_tile_keys<T, D>() == 64)
        if (pl.block_rows == 64) return go_many_rows<T, FORM, D, 2, CROSS>(a, pl, st);
    return go_many_rows<T, FORM, D, 4, CROSS>(a, pl, st);
}

template <typename T, int FORM, bool CROSS> hipError_t go_many_d(const AttendArgs &a, const ManyPlan &pl, hipStream_t st)
{
    if (a.b.d <= 64) return go_many<T, FORM, 64, CROSS>(a, pl, st);
    if constexpr (sizeof(T) == 2)
        if (a.b.d > 128) return go_many<T, FORM, 256, CROSS>(a, pl, st);
    return go_many<T, FORM, 128, CROSS>(a, pl, st);
}
template <int FORM, bool CROSS> hipError_t many_of(const AttendArgs &a, const ManyPlan &pl, int dtype, hipStream_t st)
{
    return dtype == 0 ? go_many_d<float, FORM, CROSS>(a, pl, st) : go_many_d<uint16_t, FORM, CROSS>(a, pl, st);
}

}  // namespace

}  // namespace gkv
