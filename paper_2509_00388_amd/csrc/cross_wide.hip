// Attention of rows over all that another sequence holds: the kernels of attend_wide.hpp.
#include "attend_wide.hpp"

namespace gkv {

hipError_t launch_cross_wide(const AttendArgs &a, const ManyPlan &pl, int form, hipStream_t st)
{
    return with_form(form, [&](auto f) { return wide_of<decltype(f)::value, true>(a, pl, st); });
}

}  // namespace gkv
