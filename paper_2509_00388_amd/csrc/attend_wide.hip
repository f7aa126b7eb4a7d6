// Attention over pages of rows with more than 128 stacked rows: the kernels of attend_wide.hpp.
#include "attend_wide.hpp"

namespace gkv {

hipError_t launch_attend_wide(const AttendArgs &a, const ManyPlan &pl, int form, bool cross, hipStream_t st)
{
    if (cross) return launch_cross_wide(a, pl, form, st);
    if (in_blocks(form)) return launch_blocks_wide(a, pl, form, st);
    return form == kPagesPlain ? wide_of<kPagesPlain, false>(a, pl, st)
         : form == kPagesFp8   ? wide_of<kPagesFp8, false>(a, pl, st) : wide_of<kPagesInt8, false>(a, pl, st);
}

}  // namespace gkv
