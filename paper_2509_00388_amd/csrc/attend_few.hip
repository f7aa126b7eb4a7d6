// Attention over pages of rows with few stacked rows: the kernels of attend_few.hpp, and how their work is planned.
#include "attend_few.hpp"

namespace gkv {

bool attend_mfma_applies(int dtype, int d) { return d <= (dtype == 0 ? 128 : 256); }   // (32-bit rows of 256 would fill the LDS)

FewPlan few_plan(const PagedBatch &b, int dtype, int form, int G)
{
    const int D = attend_width(b.d);
    FewPlan p{};
    p.tile_keys = 4 * 32 * few_blocks(D, form == kPagesPlain && dtype == 0);
    const long rows = (long)b.max_rows * G;
    p.join.slot_rows = rows < kFewRows ? (int)rows : kFewRows;
    p.join.slot_floats = (p.join.slot_rows * (D + 2) + 3) & ~3;
    p.join.rows_per_wg = 1;
    const long cap = (((long)b.table_pages << b.page_shift) + p.tile_keys - 1) / p.tile_keys * b.H * b.n_seqs;
    p.join.n_wg = cap < kMostFewWorkgroups ? (int)cap : kMostFewWorkgroups;
    return p;
}

hipError_t launch_attend_few(const AttendArgs &a, const FewPlan &pl, int dtype, int form, bool cross, hipStream_t st)
{
    if (cross) return launch_cross_few(a, pl, dtype, form, st);
    if (in_blocks(form)) return launch_blocks_few(a, pl, dtype, form, st);
    return form == kPagesPlain ? few_of<kPagesPlain, false>(a, pl, dtype, st)
         : form == kPagesFp8   ? few_of<kPagesFp8, false>(a, pl, dtype, st) : few_of<kPagesInt8, false>(a, pl, dtype, st);
}

}  // namespace gkv
