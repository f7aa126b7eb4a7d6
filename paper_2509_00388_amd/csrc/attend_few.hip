// Attention over pages of rows with few stacked rows: the kernels of attend_few.hpp, and how their work is planned.
#include "attend_few.hpp"

namespace gkv {

bool attend_mfma_applies(int dtype, int d) { return d <= (dtype == 0 ? 128 : 256); }   // (32-bit rows of 256 would fill the LDS)

// Whether workgroups take whole pairs and none is split: what the others would take off a workgroup is less than what it costs to leave parts
// and to launch the kernel that joins them, if the longest sequence that may be has few tiles, or the pairs are as many as fill the
// card but not so many that a long one among short ones holds it up.  (us, split / whole, lengths from an eighth to all of the tiles, fp8 blocks of d = 128 and eight
// key heads, or plain states of d = 64 and sixteen: 1 sequence of 3 tiles 10.7 / 9.1, of 4 10.6 / 11.7; 16 of 3 13.3 / 10.6, of 8 19.7 / 17.7, of 12
// 19.7 / 21.3; 64 of 8 34 / 23.8, of 12 42.4 / 32.5; 128 of 8 54 / 44, of 18 93.6 / 93.2; states of 64 sequences of 4 46.7 / 41, of 8 74.3 / 74.2, of 12 102 / 104, of 256
// of 4 140 / 136, of 6 191 / 196, of 8 241 / 263.  Beyond 8 tiles it goes either way: 64 sequences of 12 tiles gain in fp8 and lose over states.)  Causal attention over pages of rows always splits, so that its sums keep their order.
bool few_whole(long tiles, long pairs) { return tiles <= 3 || (tiles <= 8 && pairs >= 128 && pairs <= 1024); }

FewPlan few_plan(const PagedBatch &b, int dtype, int form, int G, bool cross)
{
    const int D = attend_width(b.d);
    FewPlan p{};
    const int tile_keys = 4 * 32 * few_blocks(D, form == kPagesPlain && dtype == 0);
    const long rows = (long)b.max_rows * G;
    p.join.slot_rows = rows < kFewRows ? (int)rows : kFewRows;
    p.join.slot_floats = (p.join.slot_rows * (D + 2) + 3) & ~3;
    p.join.rows_per_wg = 1;
    const long tiles = (((long)b.table_pages << b.page_shift) + tile_keys - 1) / tile_keys;   // of the longest sequence that may be
    p.whole = (cross || in_blocks(form)) && few_whole(tiles, (long)b.H * b.n_seqs);
    const long cap = (p.whole ? 1 : tiles) * b.H * b.n_seqs;
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
