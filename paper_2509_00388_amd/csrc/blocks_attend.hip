// Causal attention over pages of 8-bit codes with a scale for each block of tokens and head: the kernels of attend_few.hpp, attend_many.hpp
// and attend_wide.hpp.
#include "attend_few.hpp"
#include "attend_wide.hpp"

namespace gkv {

hipError_t launch_blocks_few(const AttendArgs &a, const FewPlan &pl, int dtype, int form, hipStream_t st)
{
    return form == kBlocksFp8 ? few_of<kBlocksFp8, false>(a, pl, dtype, st) : few_of<kBlocksInt8, false>(a, pl, dtype, st);
}

hipError_t launch_blocks_many(const AttendArgs &a, const ManyPlan &pl, int dtype, int form, hipStream_t st)
{
    return form == kBlocksFp8 ? many_of<kBlocksFp8, false>(a, pl, dtype, st) : many_of<kBlocksInt8, false>(a, pl, dtype, st);
}

hipError_t launch_blocks_wide(const AttendArgs &a, const ManyPlan &pl, int form, hipStream_t st)
{
    return form == kBlocksFp8 ? wide_of<kBlocksFp8, false>(a, pl, st) : wide_of<kBlocksInt8, false>(a, pl, st);
}

}  // namespace gkv
