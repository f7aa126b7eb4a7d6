// Attention over pages of rows with many stacked rows: the kernels of attend_many.hpp, and how their work is planned.
#include "attend_many.hpp"

namespace gkv {

ManyPlan many_plan(const PagedBatch &b, int dtype, int form, int G, bool leave_few, bool cross)
{
    const int D = attend_width(b.d);
    ManyPlan p{};
    p.leave_few = leave_few;
    p.tile_keys = D * (dtype == 0 ? 4 : 2) <= 256 ? 64 : 32;
    // (us, blocks of 256 rows and of 128, one sequence of so many rows of eight key heads of four over 8000 tokens: 160 36.2 / 40.2, 256 39.5 /
    // 42.9, 800 57.2 / 66.1, 2000 102 / 111; 8 sequences of 256 over 4000 72.5 / 103.  Blocks of 64 rows and of 128: 16 sequences of 64 over
    // 8000 tokens 122 / 127.)
    const long most_rows = (long)b.max_rows * G;
    p.wide = dtype != 0 && D <= 128 && most_rows > 128;
    p.block_rows = p.wide ? 256 : p.tile_keys == 64 && most_rows <= 64 ? 64 : 128;
    p.join.slot_rows = p.block_rows;
    p.join.slot_floats = p.block_rows * (D + 2);
    p.join.rows_per_wg = 8;
    const long blocks = (long)b.n_rows * G / p.block_rows + b.n_seqs;   // at least those of all sequences
    // Units of 256 keys with blocks of 64 rows, of 128 with larger ones, of 64 in fp32, whose tiles take longest; more where their
    // number could pass 31 bits.  Shorter units share the work out better, longer ones leave fewer parts to be joined.  (us, units of
    // 256 / 128 keys, eight key heads of four but for the last: 4 sequences of 12 rows over 2000 tokens 23 / 28, 500 rows over 8000 107 / 103, 500 over 500
    // 32 / 29; fp32, 256 / 64 keys: 701 rows over 3000 and over 5000 tokens 962 / 888, 256 rows over 2000 117 / 122, d = 64 and eight
    // heads, 300 over 900 34 / 30.)
    const long cap = (long)b.table_pages << b.page_shift;
    long units = 0;
    const int keys = p.block_rows == 64 ? 256 : dtype == 0 ? 64 : 128;
    for (p.step = keys / p.tile_keys;; p.step *= 2) {
        units = (blocks / 2 + b.n_seqs) * (2 * (cap / ((long)p.tile_keys * p.step) + 1) + 2) * b.H;
        if (units <= INT32_MAX || p.tile_keys * p.step >= 1 << 29) break;
    }
    p.block_shift = __builtin_ctz((unsigned)p.block_rows);
    p.unit_shift = __builtin_ctz((unsigned)(p.tile_keys * p.step));
    p.single = cap <= (long)p.tile_keys * p.step;
    const int most = p.wide ? 256 : 512;   // one or two workgroups a compute unit
    p.join.n_wg = units > INT32_MAX ? 0 : units < most ? (int)units : most;
    // Few blocks in many parts keep the joining launch waiting: where their keys are not many, which the device finds out, half the workgroups do.  (us, 512 /
    // 256, one sequence of 16 rows over 20000 keys, four heads of seven 51.1 / 38.5, eight of four 45.8 / 40.8, with 32-bit rows over other states 58.5 / 44.9, 56.1 / 53.7; one of
    // 30 over 10000 43.2 / 34.0, two of 12 over 8000 43.2 / 29.0; but two of 16 over 40000 64.3 / 70.7, with 32-bit rows 124 / 151, and with more blocks 20 of 16 over 300 to
    // 900 29.0 / 31.4.  Causal attention over pages of rows keeps the order of its sums.)
    if ((cross || in_blocks(form)) && blocks * b.H <= 32) p.half_to = 163840u >> p.unit_shift;
    return p;
}

hipError_t launch_attend_many(const AttendArgs &a, const ManyPlan &pl, int dtype, int form, bool cross, hipStream_t st)
{
    if (cross) return launch_cross_many(a, pl, dtype, form, st);
    if (in_blocks(form)) return launch_blocks_many(a, pl, dtype, form, st);
    return form == kPagesPlain ? many_of<kPagesPlain, false>(a, pl, dtype, st)
         : form == kPagesFp8   ? many_of<kPagesFp8, false>(a, pl, dtype, st) : many_of<kPagesInt8, false>(a, pl, dtype, st);
}

}  // namespace gkv
