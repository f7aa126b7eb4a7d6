// What the kernels of the paged cache share: how a batch of sequences lies in the pages of a pool, and the numbers of a
// pool's rows.  Everything that a kernel takes from device memory (lengths, row numbers, page numbers) is brought into its
// range before it is used, so that no content of these arrays makes a kernel read or write outside the tensors.
#pragma once
#include "common.hpp"

namespace gkv {

enum PageForm : int { kPagesPlain = 0, kPagesFp8 = 1, kPagesInt8 = 2 };

struct PagedBatch {
    const int32_t *table;       // [n_seqs, table_pages]
    const int32_t *seq_len;     // [n_seqs]
    const int32_t *row_start;   // [n_seqs + 1]
    int n_seqs, table_pages, n_pages, n_rows, max_rows;
    int H, d, page_shift;       // page_shift: log2 of the tokens a page holds
};

// Rows row0 .. row0 + n - 1 of the row tensors are the last n of the sequence's len tokens.
struct SeqRows {
    int row0, n, len;
};
__device__ __forceinline__ SeqRows seq_rows(const PagedBatch &b, int s)
{
    const int r0 = min(max(b.row_start[s], 0), b.n_rows), r1 = min(max(b.row_start[s + 1], r0), b.n_rows);
    return {r0, min(r1 - r0, b.max_rows), min(max(b.seq_len[s], 0), b.table_pages << b.page_shift)};
}

// The sequence that owns a row (the same in all lanes of the wave), n_seqs if none does.  Row numbers ascend, so it is the
// number of sequences that end at or before the row: a vote of 64 at a time.
__device__ __forceinline__ int seq_of_row(const PagedBatch &b, int row, int lane)
{
    int s = 0;
    for (int first = 0; first < b.n_seqs; first += kWave) {
        const int i = first + lane;
        const int ended = (int)__popcll(__ballot(i < b.n_seqs && b.row_start[min(i, b.n_seqs - 1) + 1] <= row));
        s += ended;
        if (ended < kWave) break;
    }
    return s;
}

// Number of the pool's row that holds head 0 of position pos (0 <= pos < tokens of the table) of a sequence, -1 where the
// page number is none of the pool's; head h's is h pages' worth of tokens further.
__device__ __forceinline__ int page_of(const PagedBatch &b, int s, int pos)
{
    const int page = b.table[(long)s * b.table_pages + (pos >> b.page_shift)];
    return (unsigned)page < (unsigned)b.n_pages ? page : -1;
}
// The table's entry as it is, for kernels that ask for it long before they use it: the comparison that page_of() makes would wait
// for it, and for every load asked for before it.
__device__ __forceinline__ int raw_page(const PagedBatch &b, int s, int pos)
{
    return b.table[(long)s * b.table_pages + (pos >> b.page_shift)];
}
__device__ __forceinline__ bool is_page(const PagedBatch &b, int page) { return (unsigned)page < (unsigned)b.n_pages; }
__device__ __forceinline__ int pool_row(const PagedBatch &b, int page, int h, int pos)
{
    return ((page * b.H + h) << b.page_shift) + (pos & ((1 << b.page_shift) - 1));
}

// ---- 8-bit codes ------------------------------------------------------------------------------------
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Four codes of a word as floats (exact).
template <int FORM> __device__ __forceinline__ void decode4(uint32_t w, float *o)
{
    if constexpr (FORM == kPagesFp8) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), c = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        o[0] = a[0]; o[1] = a[1]; o[2] = c[0]; o[3] = c[1];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (float)((int32_t)(w << (24 - 8 * e)) >> 24);
    }
}

// The values of a 16-byte piece of a cached row of rows of type T.
template <typename T, int FORM> struct Cached {
    static constexpr int kBytes = FORM == kPagesPlain ? (int)sizeof(T) : 1;   // of a value
    static constexpr int kPerVec = 16 / kBytes;
    __device__ static __forceinline__ void unpack(const uint4 &v, float *o)
    {
        if constexpr (FORM == kPagesPlain) {
            Elem<T>::unpack(v, o);
        } else {
            decode4<FORM>(v.x, o); decode4<FORM>(v.y, o + 4); decode4<FORM>(v.z, o + 8); decode4<FORM>(v.w, o + 12);
        }
    }
};

// Two floats to bf16, nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    union { b2 v; uint32_t u; } x;
    x.v = b2{(__bf16)lo, (__bf16)hi};
    return x.u;
}

}  // namespace gkv
