// Attention of rows over all that another sequence holds: the kernels of attend_few.hpp.
#include "attend_few.hpp"

namespace gkv {

hipError_t launch_cross_few(const AttendArgs &a, const FewPlan &pl, int dtype, int form, hipStream_t st)
{
    return with_form(form, [&](auto f) { return few_of<decltype(f)::value, true>(a, pl, dtype, st); });
}

}  // namespace gkv
