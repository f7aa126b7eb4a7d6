// Arguments of the attention kernels (attend.hip, attend_few.hip, attend_many.hip).
#pragma once
#include "paged.hpp"

namespace gkv {

// Stacked query rows: the G query heads of a key-value head, token by token (row r is token r / G, head r % G of them).
struct AttendArgs {
    PagedBatch b;
    const void *Q, *Kpages, *Vpages;
    const float *Kscale, *Vscale;
    void *out;
    float *lse;   // [n_rows, H_q] or null
    int G;
    float c;      // softmax scale times log2(e)
    long q_row, q_head, o_row, o_head;   // strides in elements
};

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kFewRows = 32;   // stacked rows up to which a sequence goes to the kernel for few rows

// The logarithm of the sum from its base-2 parts (m: maximum, l: sum of 2^(x - m), 0 where nothing is seen).
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2; }
__device__ __forceinline__ float inverse_of(float l) { return l == 0.f ? 0.f : 1.f / l; }

// ---- how work is cut ----------------------------------------------------------------------------------
// The lengths are known to the device alone, so each workgroup adds up for itself what lies before its share.  `weight(s)` is
// the work of sequence s in whatever unit; workgroups of NW waves, `part`: 20 words of LDS.
template <int NW, typename W> __device__ uint32_t weigh(int n_seqs, uint32_t *part, W &&weight)
{
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    uint32_t total = 0;
    for (int first = 0; first < n_seqs; first += 64 * NW) {
        const int s = first + tid;
        const uint32_t all = wave_sum_u32(s < n_seqs ? weight(s) : 0u);
        __syncthreads();
        if (lane == 0) part[wv] = all;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) total += part[w];
    }
    return total;
}
// The sequence that holds unit `first(total)` (below the total), the units before it and the total; -1 if first() says so.
template <int NW, typename W, typename F>
__device__ int find_share(int n_seqs, uint32_t &total, uint32_t &before, uint32_t *part, W &&weight, F &&first)
{
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    uint32_t w = tid < n_seqs ? weight(tid) : 0;
    if (tid == 0) part[16] = (uint32_t)n_seqs;   // (found nowhere: only where row numbers that do not ascend overflow the sums)
    uint32_t at = block_scan_add<NW>(w, part, lane, wv, total);
    if (n_seqs > 64 * NW) total = weigh<NW>(n_seqs, part, weight);   // (more sequences than threads: in a pass of its own)
    const int64_t unit = first(total);
    if (unit < 0) return -1;
    for (int s0 = 0; ; s0 += 64 * NW) {
        if (s0 > 0) {
            uint32_t here;
            const uint32_t base = part[18];
            w = s0 + tid < n_seqs ? weight(s0 + tid) : 0;
            __syncthreads();
            at = base + block_scan_add<NW>(w, part, lane, wv, here);
        }
        if (unit >= at && unit < (int64_t)at + w) { part[16] = (uint32_t)(s0 + tid); part[17] = at; }
        if (tid == 64 * NW - 1) part[18] = at + w;
        __syncthreads();
        if (unit < (int64_t)part[18] || s0 + 64 * NW >= n_seqs) break;
    }
    before = part[17];
    return __builtin_amdgcn_readfirstlane((int)part[16]);
}

// Equal stretches of `total` units for n workgroups: the first unit of the w-th, and the one that takes a unit.
__device__ __forceinline__ uint32_t stretch_first(uint32_t total, int w, int n) { return (uint32_t)((uint64_t)total * w / n); }
__device__ __forceinline__ int stretch_owner(uint32_t total, uint32_t unit, int n)
{
    return min((int)((((uint64_t)unit + 1) * n - 1) / total), n - 1);
}

// What a workgroup leaves of a block of rows that others hold parts of too: every workgroup has two slots, for the part its
// stretch begins with and the part it ends with, and a record of a block whose first part it holds.  The other parts of
// that block are the first slots of the workgroups behind it.
struct JoinRecord {
    int32_t parts;       // 0: none
    int32_t slot;        // of the first part
    int32_t row0, h;     // the sequence's first row, the key-value head
    int32_t stacked, rows;   // stacked rows stacked .. stacked + rows - 1 of the sequence
    int32_t unused[2];
};
struct JoinPlan {
    int n_wg, slot_rows, slot_floats;   // a slot: [slot_rows, D] sums, [slot_rows] maxima and sums of weights
    int rows_per_wg;
    JoinRecord *records;   // [n_wg]
    float *slots;          // [2 n_wg, slot_floats]
};

// Few rows: the tiles of all (sequence, key-value head) pairs, one after the other, are cut into equal stretches, one a
// workgroup (no more stretches than tiles).
constexpr int kMostFewWorkgroups = 512;   // two a compute unit
struct FewPlan {
    JoinPlan join;
    int tile_keys;
};
__device__ __forceinline__ bool has_few(const SeqRows &q, int G) { return q.n > 0 && q.n * (long)G <= kFewRows; }
__device__ __forceinline__ uint32_t few_tiles(const SeqRows &q, const AttendArgs &a, const FewPlan &p)   // of a head
{
    return has_few(q, a.G) ? max(1, (q.len + p.tile_keys - 1) / p.tile_keys) : 0;
}

// Many rows: blocks of R stacked rows of a head, and of the key tiles that each sees so many units of `step` tiles.  The units of
// all (sequence, head, block) are cut into equal stretches as above.  A causal chunk's blocks see more and more keys; so that the work
// before a block follows from the lengths without a sum over blocks, they lie in pairs, the last with the first and so on, whose
// units are nearly the same number: a pair gets room for W = units(first) + units(last) + 2 of them, what is left of it is
// empty.  (Units u of a block that sees e keys are max(1, ceil(e / K)); e grows evenly up to rounding down by less than 1, a
// convex function of evenly spaced numbers is largest in sum at the ends, and rounding up adds less than 1 to either of two.)
struct ManyPlan {
    JoinPlan join;
    int block_rows, tile_keys, step;
    int leave_few;    // sequences of few rows are the other kernel's
    int wide;         // blocks of 256 rows (attend_wide.hip)
};
struct ManySeq {
    int rows, blocks;        // stacked
    uint32_t pair, middle;   // units of a pair of blocks, of the block that is left in the middle
    uint32_t per_head;
};
// Units of block k of a sequence; `whole`: as if it were full of rows.  (Stacked rows and positions are below 2^31 together.)
__device__ __forceinline__ uint32_t many_units(const SeqRows &q, int rows, int k, bool whole, const AttendArgs &a, const ManyPlan &p)
{
    const uint32_t end = (uint32_t)(k + 1) * p.block_rows;
    const int sees = q.len - q.n + (int)(((whole ? end : min(end, (uint32_t)rows)) - 1) / (uint32_t)a.G) + 1;
    const uint32_t keys = (uint32_t)p.tile_keys * p.step;
    return sees <= (int)keys ? 1u : ((uint32_t)sees + keys - 1) / keys;
}
__device__ __forceinline__ ManySeq many_seq(const SeqRows &q, const AttendArgs &a, const ManyPlan &p)
{
    ManySeq m{};
    if (q.n <= 0 || (p.leave_few && has_few(q, a.G))) return m;
    m.rows = q.n * a.G;
    m.blocks = (m.rows + p.block_rows - 1) / p.block_rows;
    if (m.blocks > 1) m.pair = many_units(q, m.rows, 0, true, a, p) + many_units(q, m.rows, m.blocks - 1, true, a, p) + 2;
    if (m.blocks & 1) m.middle = many_units(q, m.rows, m.blocks / 2, false, a, p);
    m.per_head = m.blocks / 2 * m.pair + m.middle;
    return m;
}
// The next part of a stretch pos .. last - 1: units u0 .. u1 - 1 of a block's `units`.  False at the stretch's end.
struct ManyPart {
    SeqRows sq;
    int rows, h, block;   // rows: stacked rows of the sequence
    uint32_t u0, u1, units;
};
__device__ __forceinline__ bool next_part(const AttendArgs &a, const ManyPlan &pl, uint32_t &pos, uint32_t last, int &s,
                                          uint32_t &before, ManyPart &p)
{
    while (pos < last && s < a.b.n_seqs) {
        p.sq = seq_rows(a.b, s);
        const ManySeq ms = many_seq(p.sq, a, pl);
        if (ms.per_head == 0 || pos >= before + ms.per_head * a.b.H) {   // the next sequence
            before += ms.per_head * a.b.H;
            ++s;
            continue;
        }
        p.rows = ms.rows;
        p.h = (int)((pos - before) / ms.per_head);
        uint32_t at = (pos - before) % ms.per_head;
        const int pair = ms.pair ? (int)min(at / ms.pair, (uint32_t)ms.blocks / 2) : 0;
        at -= (uint32_t)pair * ms.pair;
        p.u0 = at;
        p.block = ms.blocks - 1 - pair;
        p.units = many_units(p.sq, p.rows, p.block, false, a, pl);
        if (p.u0 >= p.units) {
            p.u0 -= p.units;
            p.block = pair;
            p.units = many_units(p.sq, p.rows, pair, false, a, pl);
            if (p.u0 >= p.units) {   // the pair's empty rest
                pos += ms.pair - at;
                continue;
            }
        }
        p.u1 = min(p.units, p.u0 + (last - pos));
        return true;
    }
    return false;
}

// ---- launchers ------------------------------------------------------------------------------------------
bool attend_mfma_applies(int dtype, int d);   // whether the matrix-core kernels take this head dimension
FewPlan few_plan(const PagedBatch &b, int dtype, int form, int G);
ManyPlan many_plan(const PagedBatch &b, int dtype, int G, bool leave_few);   // no workgroups: more units than 31 bits count
hipError_t launch_attend_generic(const AttendArgs &a, int dtype, int form, hipStream_t st);
hipError_t launch_attend_few(const AttendArgs &a, const FewPlan &pl, int dtype, int form, hipStream_t st);
hipError_t launch_attend_many(const AttendArgs &a, const ManyPlan &pl, int dtype, int form, hipStream_t st);
hipError_t launch_attend_wide(const AttendArgs &a, const ManyPlan &pl, int form, hipStream_t st);
hipError_t launch_attend_join(const AttendArgs &a, const JoinPlan &few, const JoinPlan &many, int dtype, hipStream_t st);   // n_wg 0: none
inline size_t join_record_bytes(const JoinPlan &p) { return (size_t)p.n_wg * sizeof(JoinRecord); }
inline size_t join_slot_bytes(const JoinPlan &p) { return (size_t)2 * p.n_wg * p.slot_floats * 4; }

// Head dimension that the matrix-core kernels fill d up to.
inline int attend_width(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

}  // namespace gkv
