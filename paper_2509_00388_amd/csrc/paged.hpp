// What the kernels of the paged cache share: how a batch of sequences lies in the pages of a pool, and the numbers of a
// pool's rows.  Everything that a kernel takes from device memory (lengths, row numbers, page numbers) is brought into its
// range before it is used, so that no content of these arrays makes a kernel read or write outside the tensors.
#pragma once
#include "common.hpp"

#include <type_traits>

namespace gkv {

// How a pool holds its rows.  In the last two a scale belongs to a block of tokens of a head and not to a row of it; the codes are the same.
enum PageForm : int { kPagesPlain = 0, kPagesFp8 = 1, kPagesInt8 = 2, kBlocksFp8 = 5, kBlocksInt8 = 6 };
constexpr int code_of(int form) { return form & 3; }
constexpr bool in_blocks(int form) { return (form & 4) != 0; }

struct PagedBatch {
    const int32_t *table;       // [n_seqs, table_pages]
    const int32_t *seq_len;     // [n_seqs]
    const int32_t *row_start;   // [n_seqs + 1]
    int n_seqs, table_pages, n_pages, n_rows, max_rows;
    int H, d, page_shift;       // page_shift: log2 of the tokens a page holds
    int scale_shift;            // in blocks: log2 of the tokens a scale belongs to
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

// The first of the n sequences from lo on of which ends(s) is false (the same in all lanes of the wave), where ends(s) ascends from true to false; at most
// 64 are left for the caller's lanes to look at: lo and n are narrowed down by votes, each of which leaves a 64th.
template <typename F> __device__ __forceinline__ void narrow_down(int &lo, int &n, int lane, F ends)
{
    while (n > kWave) {
        const int piece = (n + kWave - 1) / kWave, last = lo + min((lane + 1) * piece, n) - 1;   // the last of the lane's piece
        const int ended = (int)__popcll(__ballot(ends(last)));
        lo += min(ended * piece, n);
        n = min(piece, max(n - ended * piece, 0));
    }
}
// The sequence that owns a row (the same in all lanes of the wave), n_seqs if none does.  Row numbers ascend, so it is the
// number of sequences that end at or before the row.
__device__ __forceinline__ int seq_of_row(const PagedBatch &b, int row, int lane)
{
    int lo = 0, n = b.n_seqs;
    auto ends = [&](int s) { return b.row_start[s + 1] <= row; };
    narrow_down(lo, n, lane, ends);
    return lo + (int)__popcll(__ballot(lane < n && ends(lo + lane)));
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

// Number of the scale of a row of the pool.
template <int FORM> __device__ __forceinline__ int scale_of_row(const PagedBatch &b, int row)
{
    return in_blocks(FORM) ? row >> b.scale_shift : row;
}

// ---- 8-bit codes ------------------------------------------------------------------------------------
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Four codes of a word as floats (exact).
template <int FORM> __device__ __forceinline__ void decode4(uint32_t w, float *o)
{
    if constexpr (code_of(FORM) == kPagesFp8) {
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

// Rows whose largest magnitude is below this are stored as zeros: the quotients by their scale would leave the range of
// normal 32-bit numbers.
constexpr float kLeastMax = 0x1p-100f;

// The scale that brings the largest magnitude a to the largest code.  fp8: the least power of two 2^k with a <= 448 * 2^k
// (a code's precision does not depend on its size, so a power of two costs none, and the division by it is exact);
// int8: a / 127.  0 for rows that are stored as zeros.
template <int FORM> __device__ __forceinline__ float scale_of(float a)
{
    if (!(a >= kLeastMax)) return 0.f;
    if (code_of(FORM) == kPagesInt8) return a / 127.f;
    const uint32_t u = __float_as_uint(a);   // a = (1 + mantissa) * 2^(exponent - 127), 448 = 1.75 * 2^8
    return __uint_as_float(((u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0)) << 23);
}

// Nearest integer to x / s, ties to the even one, by the real quotient: the product with the reciprocal is at most one
// step off, and x - q s is a number of 24 bits, so that comparing it with s / 2 is exact.
__device__ __forceinline__ int int8_code(float x, float s, float inv)
{
    float q = rintf(x * inv);
    const float r = fmaf(-q, s, x), half = 0.5f * s;
    if (fabsf(r) > half || (fabsf(r) == half && ((int)q & 1))) q += copysignf(1.f, r);
    return (int)fminf(fmaxf(q, -127.f), 127.f);
}

template <int FORM> __device__ __forceinline__ uint32_t encode4(const float *x, float s, float inv)
{
    if (code_of(FORM) == kPagesFp8) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
    }
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= (uint32_t)(int8_code(x[e], s, inv) & 0xff) << (8 * e);
    return w;
}

// f(std::integral_constant<int, FORM>) for a pool's form.
template <typename F> auto with_form(int form, F &&f)
{
    switch (form) {
        case kPagesFp8: return f(std::integral_constant<int, kPagesFp8>{});
        case kPagesInt8: return f(std::integral_constant<int, kPagesInt8>{});
        case kBlocksFp8: return f(std::integral_constant<int, kBlocksFp8>{});
        case kBlocksInt8: return f(std::integral_constant<int, kBlocksInt8>{});
        default: return f(std::integral_constant<int, kPagesPlain>{});
    }
}

// ---- pages dealt to sequences (assign.hip) -----------------------------------------------------------
struct AssignArgs {
    const int32_t *keep, *new_rows, *len_before, *free_before;   // [n_seqs] (keep may be null), [1]
    int32_t *seq_len, *table, *free_pages, *free_after;          // [n_seqs], [n_seqs, table_pages], [n_pages], [1]
    int32_t *row_start, *positions, *slots;                      // [n_seqs + 1], [n_rows] or null
    int n_seqs, table_pages, n_pages, n_rows, max_rows, page_shift;
    int rows_here;              // the kernel of the sums writes positions and slots too
};
struct AssignSums {             // of each chunk of sequences; n_free: [1]
    uint32_t *asked, *taken, *given, *rows, *out, *n_free;
};
size_t assign_scratch_bytes(int n_seqs);
hipError_t launch_assign(const AssignArgs &a, void *scratch, hipStream_t st);

// Two floats to bf16, nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    union { b2 v; uint32_t u; } x;
    x.v = b2{(__bf16)lo, (__bf16)hi};
    return x.u;
}

}  // namespace gkv
