// Attention of rows over all that another sequence holds: the kernels of attend_many.hpp.
#include "attend_many.hpp"

namespace gkv {

hipError_t launch_cross_many(const AttendArgs &a, const ManyPlan &pl, int dtype, int form, hipStream_t st)
{
    return with_form(form, [&](auto f) { return many_of<decltype(f)::value, true>(a, pl, dtype, st); });
}

}  // namespace gkv
