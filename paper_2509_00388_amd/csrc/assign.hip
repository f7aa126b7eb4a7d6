// Pages of a pool dealt to the sequences of a batch, and the numbers that the other calls go by (graphkv_cache_assign).
//
// A sequence with had tokens keeps some, gets new ones and then needs ceil(want / page) - ceil(had / page) pages: more, which
// come from the top of a stack of free ones, or fewer, and then the rest go back to it.  Where in the stack, and from which row on
// its rows lie, follows from sums over the sequences before it; who is refused follows from the same sums, since once the rows or
// pages asked for pass what there is, they do so for all later sequences that ask for any.
//
//   asked  = sums of new rows                -> rows that do not fit are refused
//   taken, given = sums of pages             -> pages beyond free + given are refused
//   start  = sums of the rows that are left  -> row numbers
//
// Up to 4096 sequences a workgroup does all this, up to four sequences a thread, with three scans; beyond, workgroups of 1024 each go as far as they get
// without the others' sums, leave theirs, and begin anew in the next launch: four of them, whatever the number.  Page numbers
// and rows are dealt to the threads one by one, whoever's they are, and find their sequence in the sums, which lie in the LDS.  Few rows
// are told their places in the same launch, many in one of their own.  Nothing but latency: a batch's numbers are a few kilobytes.  A token each of 64
// sequences 4.0 us, 1000 sequences of which 111 end and are followed by prompts, 4400 pages that move and 126000 rows, 9.4 + 4.0, a prompt of 120000 rows
// 4.2 + 2.9; a call takes the host 9.
#include "kernels.hpp"
#include "paged.hpp"

namespace gkv {

namespace {

constexpr int kChunk = 1024;   // threads of a workgroup, and its sequences where there are several

__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Sums of two numbers of the threads before this one, of NW waves; sums that pass 32 bits stay at the largest number.
struct Two {
    uint32_t a, b;
};
__device__ __forceinline__ Two add_both(Two x, Two y) { return {add_sat(x.a, y.a), add_sat(x.b, y.b)}; }
template <int NW> __device__ __forceinline__ Two scan_sat(Two v, Two *part, Two &total)   // part: NW of them
{
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Two incl{wave_scan_op(v.a, 0u, add_sat), wave_scan_op(v.b, 0u, add_sat)};
    __syncthreads();   // (the scan before is done with `part`)
    if (lane == kWave - 1) part[wv] = incl;
    __syncthreads();
    const Two mine = lane < NW ? part[lane] : Two{0, 0};
    const Two sums{wave_scan_op(mine.a, 0u, add_sat), wave_scan_op(mine.b, 0u, add_sat)};
    auto of_lane = [](uint32_t x, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); };
    total = {of_lane(sums.a, 63), of_lane(sums.b, 63)};
    const Two before{(uint32_t)__shfl_up((int)incl.a, 1, kWave), (uint32_t)__shfl_up((int)incl.b, 1, kWave)};
    return add_both(lane > 0 ? before : Two{0, 0}, wv > 0 ? Two{of_lane(sums.a, wv - 1), of_lane(sums.b, wv - 1)} : Two{0, 0});
}

// The first of n ascending sums that is above i (n if none is).
__device__ __forceinline__ int first_above(const uint32_t *sums, int n, uint32_t i)
{
    int lo = 0;
    for (int len = n; len > 0;) {
        const int half = len >> 1;
        if (sums[lo + half] <= i) { lo += half + 1; len -= half + 1; }
        else len = half;
    }
    return lo;
}

__device__ __forceinline__ uint32_t pages_of(uint32_t tokens, int shift) { return (tokens + (1u << shift) - 1) >> shift; }

// Place of a position in the pool (of head 0, in tokens), -1 if it has none.
__device__ __forceinline__ int slot_of(const AssignArgs &a, int s, int pos)
{
    const int page = a.table[(long)s * a.table_pages + (pos >> a.page_shift)];
    return (unsigned)page < (unsigned)a.n_pages ? (page << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : -1;
}

// Sums of the chunks before mine, of them all, of two arrays that the launch before left.
template <int NW> __device__ __forceinline__ Two chunks_before(const uint32_t *x, const uint32_t *y, int chunks, int mine, Two *part, Two &all)
{
    const int t = threadIdx.x;
    const Two v = t < chunks ? Two{x[t], y[t]} : Two{0, 0};
    Two before;
    scan_sat<NW>(t < mine ? v : Two{0, 0}, part, before);
    scan_sat<NW>(v, part, all);
    return before;
}

// PHASE 0: all at once, a single chunk.  1 to 4: as far as the sums of the launches before allow (AssignSums).  A thread has ITEMS sequences that are
// next to one another.
template <int NT, int ITEMS, int PHASE>
__global__ __launch_bounds__(NT) void assign_kernel(AssignArgs a, AssignSums sums)
{
    constexpr int NW = NT / kWave, N = NT * ITEMS;
    extern __shared__ __align__(16) uint32_t lists[];   // of the chunk's sequences: sums of pages, of rows, first entries, lengths
    __shared__ Two part[NW];
    uint32_t *by_page = lists, *by_row = lists + N;
    int *first_entry = reinterpret_cast<int *>(lists + 2 * N), *length = first_entry + N;
    const int t = threadIdx.x, chunk = blockIdx.x, base = chunk * N, mine = t * ITEMS, chunks = gridDim.x;
    const int here = min(N, a.n_seqs - base);   // sequences of the chunk
    const uint32_t cap = (uint32_t)a.table_pages << a.page_shift;

    uint32_t had[ITEMS], want[ITEMS], fresh[ITEMS], n_free = 0;
    bool ok[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) had[i] = want[i] = fresh[i] = 0;
    if (here > 0) {
        int len[ITEMS], keep[ITEMS], more[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int s = base + min(mine + i, here - 1);
            len[i] = a.len_before[s];
            keep[i] = a.keep ? a.keep[s] : INT32_MAX;
            more[i] = a.new_rows[s];
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (mine + i >= here) continue;
            had[i] = min((uint32_t)max(len[i], 0), cap);
            fresh[i] = (uint32_t)max(more[i], 0);
            want[i] = min((uint32_t)max(keep[i], 0), had[i]) + fresh[i];   // (below 2^30 + 2^31)
        }
    }
    // (the numbers of free pages before and after may be one: phases beyond the first read what that one saw)
    if (PHASE <= 1) n_free = (uint32_t)min(max(a.free_before[0], 0), a.n_pages);
    else n_free = sums.n_free[0];
    uint32_t sum = 0;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        ok[i] = fresh[i] <= (uint32_t)a.max_rows && want[i] <= cap;
        if (!ok[i]) fresh[i] = 0;
        sum = add_sat(sum, fresh[i]);
    }

    Two all, before{0, 0};
    if (PHASE >= 2) before = chunks_before<NW>(sums.asked, sums.asked, chunks, chunk, part, all);
    uint32_t asked = add_sat(before.a, scan_sat<NW>({sum, 0}, part, all).a);
    if (PHASE == 1) {
        if (t == 0) sums.asked[chunk] = all.a;
        if (t == 0 && chunk == 0) sums.n_free[0] = n_free;
        return;
    }
    uint32_t pages[ITEMS], take[ITEMS], give[ITEMS];
    Two moved{0, 0};
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        asked = add_sat(asked, fresh[i]);
        ok[i] = ok[i] && (fresh[i] == 0 || asked <= (uint32_t)a.n_rows);
        pages[i] = pages_of(had[i], a.page_shift);
        const uint32_t after = pages_of(want[i], a.page_shift);
        take[i] = ok[i] && after > pages[i] ? after - pages[i] : 0;
        give[i] = ok[i] && after < pages[i] ? pages[i] - after : 0;
        moved = add_both(moved, {take[i], give[i]});
    }
    moved = scan_sat<NW>(moved, part, all);
    const uint32_t given_here = all.b;
    if (PHASE == 2) {
        if (t == 0) { sums.taken[chunk] = all.a; sums.given[chunk] = all.b; }
        return;
    }
    before = {0, 0};
    if (PHASE >= 3) before = chunks_before<NW>(sums.taken, sums.given, chunks, chunk, part, all);
    const uint32_t taken_before = before.a, given_before = before.b, given_all = all.b;
    const uint32_t total = min(add_sat(n_free, given_all), (uint32_t)a.n_pages);   // (more only where a page has two owners)
    Two served{0, 0};
    uint32_t taken[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        moved = add_both(moved, {take[i], give[i]});
        taken[i] = moved.a;
        ok[i] = ok[i] && (take[i] == 0 || add_sat(taken_before, moved.a) <= total);
        if (PHASE == 0 || PHASE == 3) {
            by_page[mine + i] = moved.b;
            first_entry[mine + i] = (int)pages[i] - (int)moved.b;   // (what it gives back ends with its last page)
        }
        fresh[i] = ok[i] ? fresh[i] : 0;
        served = add_both(served, {fresh[i], ok[i] ? take[i] : 0});
    }
    if (PHASE == 0 || PHASE == 3) {
        // Pages that come back: number i of all to entry total - 1 - i, so that what was taken last lies on top again where a
        // call undoes another.
        if (given_here > 0) {
            __syncthreads();
            const uint32_t room = total - n_free > given_before ? total - n_free - given_before : 0;
            for (uint32_t i = t; i < min(given_here, room); i += NT) {
                const int owner = first_above(by_page, here, i);
                if (owner < here)
                    a.free_pages[total - 1 - (given_before + i)] = a.table[(long)(base + owner) * a.table_pages + (first_entry[owner] + (int)i)];
            }
        }
    }
    uint32_t row = scan_sat<NW>(served, part, all).a;   // (those that are served come first: their sums of pages are `taken`)
    const uint32_t rows_all = all.a, out_all = all.b;
    if (PHASE == 3) {
        if (t == 0) { sums.rows[chunk] = rows_all; sums.out[chunk] = out_all; }
        return;
    }
    before = {0, 0};
    if (PHASE == 4) before = chunks_before<NW>(sums.rows, sums.out, chunks, chunk, part, all);
    const uint32_t start_before = before.a, rows_total = all.a, out_total = all.b;
    __syncthreads();   // (pages that came back may be dealt out again)
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int len = (int)(ok[i] ? want[i] : had[i]);
        if (mine + i < here) {
            a.seq_len[base + mine + i] = len;
            a.row_start[base + mine + i] = (int32_t)(start_before + row);
        }
        row = add_sat(row, fresh[i]);
        by_page[mine + i] = taken[i];
        by_row[mine + i] = row;
        first_entry[mine + i] = (int)pages[i] - (int)(taken[i] - take[i]);
        length[mine + i] = len;
    }
    if (t == 0 && chunk == 0) {
        a.free_after[0] = (int32_t)(total - out_total);
        a.row_start[a.n_seqs] = (int32_t)rows_total;
    }
    __syncthreads();
    for (uint32_t i = t; i < out_all; i += NT) {
        const int owner = first_above(by_page, here, i);
        if (owner < here)
            a.table[(long)(base + owner) * a.table_pages + (first_entry[owner] + (int)i)] = a.free_pages[total - 1 - (taken_before + i)];
    }
    if (PHASE == 0 && a.rows_here) {
        __syncthreads();
        for (int r = t; r < a.n_rows; r += NT) {
            int pos = -1, slot = -1;
            if (r < (int)rows_all) {
                const int owner = first_above(by_row, here, (uint32_t)r);
                pos = length[owner] - (int)by_row[owner] + r;
                slot = slot_of(a, owner, pos);
            }
            if (a.positions) a.positions[r] = pos;
            if (a.slots) a.slots[r] = slot;
        }
    }
}

// The sequence of row r (below the last row number) by a vote of 64 row numbers at a time, for the whole wave.
__device__ __forceinline__ int seq_of(const AssignArgs &a, int r, int lane)
{
    int lo = 0, n = a.n_seqs;   // it is one of the n sequences from lo on
    while (n > 1) {
        const int piece = (n + kWave - 1) / kWave, ask = lo + min((lane + 1) * piece, n);   // the last of each piece
        const int ended = (int)__popcll(__ballot(a.row_start[ask] <= r && ask < lo + n));
        lo += ended * piece;
        n = min(piece, n - ended * piece);
    }
    return lo;
}

// Position and place of each row, a row a thread.  A wave finds the sequences of its first and last row, which with many rows a sequence are the same or
// next to one another, and each lane its own between them.
__global__ __launch_bounds__(256) void assign_rows_kernel(AssignArgs a)
{
    const int r = blockIdx.x * 256 + threadIdx.x, lane = threadIdx.x & 63, first = __builtin_amdgcn_readfirstlane(r);
    const int rows = a.row_start[a.n_seqs];
    int pos = -1, slot = -1;
    if (first < rows) {
        int lo = seq_of(a, first, lane);
        const int last = seq_of(a, min(first + kWave, rows) - 1, lane);
        for (int len = last - lo; len > 0;) {   // the first that ends behind the row
            const int half = len >> 1;
            if (a.row_start[lo + half + 1] <= r) { lo += half + 1; len -= half + 1; }
            else len = half;
        }
        if (r < rows) {
            pos = a.seq_len[lo] - a.row_start[lo + 1] + r;
            slot = slot_of(a, lo, pos);
        }
    }
    if (r >= a.n_rows) return;
    if (a.positions) a.positions[r] = pos;
    if (a.slots) a.slots[r] = slot;
}

int chunks_of(int n_seqs, int chunk) { return n_seqs > chunk ? (n_seqs + chunk - 1) / chunk : 1; }

}  // namespace

size_t assign_scratch_bytes(int n_seqs) { return n_seqs <= kChunk ? 0 : (size_t)(5 * chunks_of(n_seqs, kChunk) + 1) * 4; }

hipError_t launch_assign(const AssignArgs &args, void *scratch, hipStream_t st)
{
    AssignArgs a = args;
    const bool maps = (a.positions || a.slots) && a.n_rows > 0;
    auto go = [&](auto kernel, int threads, int items, const AssignSums &sums) {
        const int lds = threads * items * 16;
        if (lds >= 64 * 1024 && !allow_big_lds(reinterpret_cast<const void *>(kernel))) return false;
        kernel<<<chunks_of(a.n_seqs, threads * items), threads, lds, st>>>(a, sums);
        return true;
    };
    // (one launch of 1024 threads with 2 or 4 sequences each / four: 1100 sequences of a row 7.5 / 21.4 us, 2000 8.3 / 21.5, 3000 12.5 / 21.8, 4000 13.6 / 22.6; with 8,
    // 6000 24.7 / 22.6.  1433 that end and are followed by prompts of up to 174 rows 35.8 / 37.9, but 4000 of which half do, of up to 60, 61 / 33: many pages
    // are several workgroups' work.)
    const int items = a.n_seqs <= kChunk ? 1 : a.n_seqs <= 2 * kChunk ? 2 : a.n_seqs <= 4 * kChunk && a.n_rows >> a.page_shift <= 4096 ? 4 : 0;
    if (items > 0) {
        // (256 threads are done sooner with their barriers, 1024 with thousands of pages, which few sequences ask for where they have many rows: 64 sequences with
        // a row each 4.2 / 5.0 us, one of 4000 rows, of 16000 and of 60000 in pages of 16 5.4 / 5.5, 6.0 / 6.2, 8.2 / 7.0)
        const bool small = a.n_seqs <= 256 && a.n_rows >> a.page_shift <= 1024;
        // (rows told here or by a launch of their own: 64 sequences of 4, 16 and 32 rows 4.2 / 5.4, 6.0 / 6.1, 8.3 / 6.4 us, 1000 of 1, 2 and 4 rows 5.9 / 8.0,
        // 6.8 / 8.1, 8.7 / 7.9)
        a.rows_here = maps && a.n_rows <= (small ? 1024 : 2048);
        if (!(small        ? go(assign_kernel<256, 1, 0>, 256, 1, AssignSums{})
              : items == 1 ? go(assign_kernel<kChunk, 1, 0>, kChunk, 1, AssignSums{})
              : items == 2 ? go(assign_kernel<kChunk, 2, 0>, kChunk, 2, AssignSums{}) : go(assign_kernel<kChunk, 4, 0>, kChunk, 4, AssignSums{})))
            return hipErrorInvalidValue;
    } else {
        const int chunks = chunks_of(a.n_seqs, kChunk);
        uint32_t *w = reinterpret_cast<uint32_t *>(scratch);
        const AssignSums sums{w, w + chunks, w + 2 * chunks, w + 3 * chunks, w + 4 * chunks, w + 5 * chunks};
        go(assign_kernel<kChunk, 1, 1>, kChunk, 1, sums);
        go(assign_kernel<kChunk, 1, 2>, kChunk, 1, sums);
        go(assign_kernel<kChunk, 1, 3>, kChunk, 1, sums);
        go(assign_kernel<kChunk, 1, 4>, kChunk, 1, sums);
    }
    if (maps && !a.rows_here) assign_rows_kernel<<<(a.n_rows + 255) / 256, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace gkv
