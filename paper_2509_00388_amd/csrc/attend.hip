// Attention of new tokens over a paged cache, scalar kernel for any type and head dimension (GRAPHKV_IMPL_GENERIC, and
// head dimensions that the matrix-core kernels do not take).
//
//   x_j = scale q . k_j,  m = max x_j,  l = sum 2^(x_j - m),  out = sum 2^(x_j - m) v_j / l   (base 2, over visible keys)
//
// in one pass over the keys with a running maximum: when it grows, the sums so far are multiplied by 2^(old - new).
// A workgroup per (row, query head) takes 256 keys at a time, a key a thread for the products with the query and a
// dimension a thread for the sums.  Keys that a row does not see are never touched.
#include "attend_tile.hpp"
#include "kernels.hpp"

namespace gkv {

namespace {

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ void put(float *p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t *p, float x) { *p = (uint16_t)pack_bf16(x, 0.f); }

template <typename T, int FORM>
__global__ __launch_bounds__(256) void attend_generic_kernel(AttendArgs a)
{
    using C = Cached<T, FORM>;
    __shared__ float q[512], p[256], red[16];
    __shared__ int at[256];
    const int row = blockIdx.x, hq = blockIdx.y, h = hq / a.G, tid = threadIdx.x, d = a.b.d;
    const int s = seq_of_row(a.b, row, tid & 63);
    if (s >= a.b.n_seqs) return;
    const SeqRows sq = seq_rows(a.b, s);
    if (row < sq.row0 || row >= sq.row0 + sq.n) return;
    const int seen = max(0, sq.len - sq.n + (row - sq.row0) + 1);   // keys 0 .. seen - 1
    const T *qr = reinterpret_cast<const T *>(a.Q) + row * a.q_row + hq * a.q_head;
    for (int i = tid; i < d; i += 256) q[i] = to_float(qr[i]);
    float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
    __syncthreads();
    for (int first = 0; first < seen; first += 256) {
        const int pos = first + tid, page = pos < seen ? page_of(a.b, s, pos) : -1;
        const int r = page < 0 ? -1 : pool_row(a.b, page, h, pos);
        float x = -INFINITY;
        if (r >= 0) {
            const uint4 *k = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(a.Kpages) + (long)r * d * C::kBytes);
            float dot = 0.f;
            for (int i = 0; i < d; i += C::kPerVec) {
                float v[C::kPerVec];
                C::unpack(k[i / C::kPerVec], v);
#pragma unroll
                for (int e = 0; e < C::kPerVec; ++e) dot = fmaf(q[i + e], v[e], dot);
            }
            x = dot * a.c * (FORM == kPagesPlain ? 1.f : a.Kscale[r]);
        }
        const float top = fmaxf(m, block_max(x, red));
        const float shift = top == -INFINITY ? 0.f : top;   // (nothing seen yet: all terms are 2^-inf)
        const float w = exp2f(x - shift), fade = exp2f(m - shift);
        at[tid] = r;
        p[tid] = FORM == kPagesPlain || r < 0 ? w : w * a.Vscale[r];
        l = l * fade + block_sum(w, red);
        m = top;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = tid + 256 * u;
            if (i >= d) continue;
            float sum = acc[u] * fade;
            for (int j = 0; j < min(256, seen - first); ++j)
                if (at[j] >= 0) sum = fmaf(p[j], cached_value<T, FORM>(a.Vpages, (long)at[j] * d + i), sum);
            acc[u] = sum;
        }
        __syncthreads();
    }
    T *out = reinterpret_cast<T *>(a.out) + row * a.o_row + hq * a.o_head;
#pragma unroll
    for (int u = 0; u < 2; ++u)
        if (tid + 256 * u < d) put(out + tid + 256 * u, acc[u] * inverse_of(l));
    if (a.lse && tid == 0) a.lse[(long)row * a.b.H * a.G + hq] = lse_of(m, l);
}

}  // namespace

hipError_t launch_attend_generic(const AttendArgs &a, int dtype, int form, hipStream_t st)
{
    const dim3 grid(a.b.n_rows, a.b.H * a.G);
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(a); return hipGetLastError(); };
    if (dtype == 0)
        return form == kPagesPlain ? go(attend_generic_kernel<float, kPagesPlain>)
             : form == kPagesFp8   ? go(attend_generic_kernel<float, kPagesFp8>) : go(attend_generic_kernel<float, kPagesInt8>);
    return form == kPagesPlain ? go(attend_generic_kernel<uint16_t, kPagesPlain>)
         : form == kPagesFp8   ? go(attend_generic_kernel<uint16_t, kPagesFp8>) : go(attend_generic_kernel<uint16_t, kPagesInt8>);
}

}  // namespace gkv
