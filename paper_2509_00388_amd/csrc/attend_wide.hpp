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
// instead of padded) 1130.  In blocks of fp8 2000 rows over 24000 keys take 750 to 760 us (plain pages 755 to 765, fp8 with a scale a row 925 to 945); six sequences of 445
// rows of two heads a group over 1000 to 9000 states 169, of which the parts of blocks that two workgroups share are 12 in the join and about as much
// in the kernel (8 of 512 rows over 8192, a block a workgroup: 976 TFLOP/s).  Slower there: waves without rows that leave a tile out, with longer units for
// blocks that are half full (182), units of one tile (185); a higher priority for the products' waves (822 for 745).
#pragma once
#include "attend_many.hpp"

#include <type_traits>

namespace gkv {

namespace {

constexpr int kWideRows = 256, kTiles = 3;   // tiles in the LDS

template <int FORM, int D> struct WideTile {
    using L = Tile<uint16_t, FORM, D, 64, 512>;
    static constexpr int kKeys = 64 * L::kKeyPitch, kVals = 64 * L::kValPitch;
    static constexpr int kBytes = kKeys + kVals + scale_bytes(FORM, 64);   // keys, values, their scales
};

#define GKV_KERNEL attend_wide_kernel   // pages of rows, plain or with a scale each
#define GKV_CROSS false
#include "attend_wide.inc"
#undef GKV_KERNEL
#undef GKV_CROSS
#define GKV_KERNEL blocks_wide_kernel   // pages in blocks
#define GKV_CROSS false
#include "attend_wide.inc"
#undef GKV_KERNEL
#undef GKV_CROSS
#define GKV_KERNEL cross_wide_kernel   // rows that see all of a sequence
#define GKV_CROSS true
#include "attend_wide.inc"
#undef GKV_KERNEL
#undef GKV_CROSS

template <int FORM, int D, bool CROSS> constexpr auto wide_kernel()
{
    if constexpr (CROSS) return &cross_wide_kernel<FORM, D>;
    else if constexpr (in_blocks(FORM)) return &blocks_wide_kernel<FORM, D>;
    else return &attend_wide_kernel<FORM, D>;
}

template <int FORM, int D, bool CROSS> hipError_t go_wide(const AttendArgs &a, const ManyPlan &pl, hipStream_t st)
{
    constexpr int lds = kTiles * WideTile<FORM, D>::kBytes;
    auto kernel = wide_kernel<FORM, D, CROSS>();
    if (lds > 64 * 1024 && !allow_big_lds(reinterpret_cast<const void *>(kernel), lds)) return hipErrorInvalidValue;
    kernel<<<pl.join.n_wg, 512, lds, st>>>(a, pl);
    return hipGetLastError();
}
template <int FORM, bool CROSS> hipError_t wide_of(const AttendArgs &a, const ManyPlan &pl, hipStream_t st)
{
    return a.b.d <= 64 ? go_wide<FORM, 64, CROSS>(a, pl, st) : go_wide<FORM, 128, CROSS>(a, pl, st);
}

}  // namespace

}  // namespace gkv
