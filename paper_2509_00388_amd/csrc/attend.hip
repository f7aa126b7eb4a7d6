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

// The parts of blocks of rows that several workgroups hold, put together: workgroup (y, w) takes rows y * rows_per_wg and on of the
// block whose first part workgroup w of the kernel for few rows, or behind those of the one for many, held (in this order, so that the few w that hold one spread over all XCDs).  A row is 256 / GROUPS lanes wide, four sums a lane; where the parts are many, several
// groups of lanes share a row's.
template <typename T, int D>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, JoinPlan few, JoinPlan many)
{
    constexpr int LANES = D / 4, GROUPS = 256 / LANES;
    __shared__ float4 sums[GROUPS][LANES];
    __shared__ float totals[GROUPS];
    const bool second = (int)blockIdx.y >= few.n_wg;
    const JoinPlan pl = second ? many : few;
    const int me = blockIdx.y - (second ? few.n_wg : 0);
    const JoinRecord rec = pl.records[me];
    const int first = blockIdx.x * pl.rows_per_wg, last = min(first + pl.rows_per_wg, rec.rows);
    if (rec.parts == 0 || first >= last) return;
    int share = 1;   // groups a row
    while (share < GROUPS && (share < rec.parts / 16 || 2 * share * (last - first) <= GROUPS)) share *= 2;
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES, mine = group % share, at_once = GROUPS / share;
    const float *slot0 = pl.slots + (size_t)rec.slot * pl.slot_floats;
    const float *slots = pl.slots + (size_t)2 * me * pl.slot_floats;   // part k > 0: 2 k slots further
    for (int r0 = first; r0 < last; r0 += at_once) {
        const int r = min(r0 + group / share, last - 1);
        const int stat = pl.slot_rows * D + 2 * r, at = r * D + 4 * lane;
        float m = -INFINITY, l = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int k = mine; k < rec.parts; k += share) {
            const float *p = k == 0 ? slot0 : slots + (size_t)2 * k * pl.slot_floats;
            const float4 y = *reinterpret_cast<const float4 *>(p + at);
            const float2 ml = *reinterpret_cast<const float2 *>(p + stat);
            const float top = fmaxf(m, ml.x), shift = top == -INFINITY ? 0.f : top;
            const float f = __builtin_amdgcn_exp2f(m - shift), g = __builtin_amdgcn_exp2f(ml.x - shift);
            m = top;
            l = l * f + ml.y * g;
            v.x = v.x * f + y.x * g; v.y = v.y * f + y.y * g; v.z = v.z * f + y.z * g; v.w = v.w * f + y.w * g;
        }
        if (share > 1) {
            // (groups of a row: bring them to the row's maximum, then one of them adds them up)
            __syncthreads();
            if (lane == 0) totals[group] = m;
            __syncthreads();
            const int g0 = group - mine;
            float top = -INFINITY;
            for (int g = 0; g < share; ++g) top = fmaxf(top, totals[g0 + g]);
            const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
            m = top;
            sums[group][lane] = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
            __syncthreads();
            if (lane == 0) totals[group] = l * f;
            __syncthreads();
            l = 0.f;
            v = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int g = 0; g < share; ++g) {
                const float4 y = sums[g0 + g][lane];
                l += totals[g0 + g];
                v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w;
            }
        }
        if (mine != 0 || r0 + group / share >= last) continue;
        const int stacked = rec.stacked + r, token = rec.row0 + stacked / a.G, head = rec.h * a.G + stacked % a.G;
        if (a.lse && lane == 0) a.lse[(long)token * a.b.H * a.G + head] = lse_of(m, l);
        if (4 * lane >= a.b.d) continue;
        const float f = inverse_of(l);
        T *to = reinterpret_cast<T *>(a.out) + token * a.o_row + head * a.o_head + 4 * lane;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(to) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
        else *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(v.x * f, v.y * f), pack_bf16(v.z * f, v.w * f));
    }
}

}  // namespace

hipError_t launch_attend_join(const AttendArgs &a, const JoinPlan &few, const JoinPlan &many, int dtype, hipStream_t st)
{
    auto chunks = [](const JoinPlan &p) { return p.n_wg ? (p.slot_rows + p.rows_per_wg - 1) / p.rows_per_wg : 0; };
    const dim3 grid(max(chunks(few), chunks(many)), few.n_wg + many.n_wg);
    const int D = attend_width(a.b.d);
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(a, few, many); return hipGetLastError(); };
    if (dtype == 0) return D == 64 ? go(attend_join_kernel<float, 64>) : go(attend_join_kernel<float, 128>);
    return D == 64 ? go(attend_join_kernel<uint16_t, 64>) : D == 128 ? go(attend_join_kernel<uint16_t, 128>) : go(attend_join_kernel<uint16_t, 256>);
}

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
