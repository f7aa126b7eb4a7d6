// Rows written to the pages of a cache and read back (graphkv_cache_write, graphkv_cache_read).
//
// A wave takes a row with all its heads, so that the row's sequence and page are looked up once, or, where rows are few, some of its heads
// (turns_grid()); a head's values lie in as
// many lanes as it has 16-byte pieces (a power of two, at most 64, a second turn for the rest).  Both kernels are bound by
// memory: every byte is moved once, with 16-byte accesses on the wider side.  Measured (bf16 rows, eight heads of 128, pages of 64,
// fp8): 32768 rows written in 44 us and read back in 46, 204 MB, at 4.6 and 4.4 TB/s, where a copy of 4 GiB reaches 4.6;
// 96 rows, a token of each of so many sequences, 5 us in a trace, of which the chain of four loads before the first store is most.
#include "kernels.hpp"
#include "paged.hpp"

namespace gkv {

namespace {

// One tensor's values of a (row, head), TURNS pieces a lane, encoded and stored.
template <typename T, int FORM, int TURNS>
__device__ __forceinline__ void store_row(const uint4 (&v)[TURNS], int pieces, int at, int group, long row, void *pages,
                                          float *scales)
{
    constexpr int PER = Elem<T>::kPerVec;
    if constexpr (FORM == kPagesPlain) {
        uint4 *to = reinterpret_cast<uint4 *>(pages) + row * pieces;
#pragma unroll
        for (int t = 0; t < TURNS; ++t)
            if (at + t * group < pieces) to[at + t * group] = v[t];
    } else {
        float x[TURNS][PER], a = 0.f;
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            Elem<T>::unpack(v[t], x[t]);
#pragma unroll
            for (int e = 0; e < PER; ++e) a = fmaxf(a, fabsf(x[t][e]));
        }
        for (int o = group >> 1; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor(a, o, kWave));
        const float s = scale_of<FORM>(a), inv = s > 0.f ? 1.f / s : 0.f;
        if (at == 0) scales[row] = s;
        char *to = reinterpret_cast<char *>(pages) + row * (pieces * PER);
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            if (at + t * group >= pieces) continue;
            uint32_t w[PER / 4];
#pragma unroll
            for (int e = 0; e < PER; e += 4) w[e / 4] = s > 0.f ? encode4<FORM>(x[t] + e, s, inv) : 0u;
            if constexpr (PER == 8) *reinterpret_cast<uint2 *>(to + (at + t * group) * PER) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t *>(to + (at + t * group) * PER) = w[0];
        }
    }
}

template <typename T, int FORM, int TURNS>
__global__ __launch_bounds__(256) void cache_write_kernel(PagedBatch b, const T *__restrict__ K, const T *__restrict__ V,
                                                          long row_stride, long head_stride, void *Kpages, void *Vpages,
                                                          float *Kscale, float *Vscale, int group)
{
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= b.n_rows) return;
    const int at = lane & (group - 1), heads = kWave / group, pieces = b.d / Elem<T>::kPerVec;
    const int s = seq_of_row(b, row, lane);
    if (s >= b.n_seqs) return;
    const SeqRows q = seq_rows(b, s);
    const int pos = q.len - q.n + (row - q.row0);
    if (row < q.row0 || row >= q.row0 + q.n || pos < 0) return;
    const int page = page_of(b, s, pos);
    if (page < 0) return;
    for (int h = lane / group + heads * blockIdx.y; h < b.H; h += heads * gridDim.y) {
        const T *k = K + row * row_stride + h * head_stride, *v = V + row * row_stride + h * head_stride;
        uint4 kv[TURNS], vv[TURNS];
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const bool in = at + t * group < pieces;
            kv[t] = in ? reinterpret_cast<const uint4 *>(k)[at + t * group] : make_uint4(0, 0, 0, 0);
            vv[t] = in ? reinterpret_cast<const uint4 *>(v)[at + t * group] : make_uint4(0, 0, 0, 0);
        }
        const long to = pool_row(b, page, h, pos);
        store_row<T, FORM>(kv, pieces, at, group, to, Kpages, Kscale);
        store_row<T, FORM>(vv, pieces, at, group, to, Vpages, Vscale);
    }
}

template <typename T> __device__ __forceinline__ void put_values(T *to, const float *x, int n);
template <> __device__ __forceinline__ void put_values<float>(float *to, const float *x, int n)
{
    for (int e = 0; e < n; e += 4) *reinterpret_cast<float4 *>(to + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
}
template <> __device__ __forceinline__ void put_values<uint16_t>(uint16_t *to, const float *x, int n)
{
    for (int e = 0; e < n; e += 8)
        *reinterpret_cast<uint4 *>(to + e) = make_uint4(pack_bf16(x[e], x[e + 1]), pack_bf16(x[e + 2], x[e + 3]),
                                                        pack_bf16(x[e + 4], x[e + 5]), pack_bf16(x[e + 6], x[e + 7]));
}

// code * s in 32 bits, to odd: cut off towards zero, with the last bit set if anything was lost.  (The product of an integer code has up to
// 31 bits; rounded to the nearest 32-bit number, it can land on the middle of two bf16 numbers that it only lies next to, and be rounded
// the wrong way from there.)
__device__ __forceinline__ float product_to_odd(float code, float s)
{
    const float p = code * s, lost = fmaf(code, s, -p);   // (exact)
    const uint32_t u = __float_as_uint(p);
    return fabsf(lost) > 0.f ? __uint_as_float((u - ((lost < 0.f) != (p < 0.f) ? 1u : 0u)) | 1u) : p;
}

// A 16-byte piece of a cached row to the row tensor: code times scale, rounded once to T.  (e4m3 codes times a power of two are exact in
// 32 bits.  int8 to bf16, 32768 rows of eight heads of 128, us: twice rounded 42.6, every value to odd 44.5, where a piece needs it 43.2.)
template <typename T, int FORM>
__device__ __forceinline__ void restore(const uint4 &v, float s, T *to)
{
    if constexpr (FORM == kPagesPlain) {
        *reinterpret_cast<uint4 *>(to) = v;
    } else {
        float x[16];
        Cached<T, FORM>::unpack(v, x);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] *= s;
        if constexpr (code_of(FORM) == kPagesInt8 && sizeof(T) == 2) {
            bool middle = false;
#pragma unroll
            for (int e = 0; e < 16; ++e) middle |= (__float_as_uint(x[e]) & 0xffffu) == 0x8000u;
            if (middle) {   // (one piece of 4000)
                Cached<T, FORM>::unpack(v, x);
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = product_to_odd(x[e], s);
            }
        }
        put_values<T>(to, x, 16);
    }
}

template <typename T, int FORM>
__device__ __forceinline__ void read_row(const PagedBatch &b, const void *__restrict__ Kpages, const void *__restrict__ Vpages,
                                         const float *__restrict__ Kscale, const float *__restrict__ Vscale, T *K, T *V, long row_stride,
                                         long head_stride, int group)
{
    using C = Cached<T, FORM>;
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= b.n_rows) return;
    const int at = lane & (group - 1), heads = kWave / group, pieces = b.d / C::kPerVec;
    const int s = seq_of_row(b, row, lane);
    if (s >= b.n_seqs) return;
    const SeqRows q = seq_rows(b, s);
    const int pos = q.len - q.n + (row - q.row0);
    if (row < q.row0 || row >= q.row0 + q.n) return;
    const int page = pos < 0 ? -1 : page_of(b, s, pos);
    for (int h = lane / group + heads * blockIdx.y; h < b.H; h += heads * gridDim.y) {
        const long from = pool_row(b, max(page, 0), h, max(pos, 0));
        for (int p = at; p < pieces; p += group) {
            uint4 kv = reinterpret_cast<const uint4 *>(Kpages)[from * pieces + p];
            uint4 vv = reinterpret_cast<const uint4 *>(Vpages)[from * pieces + p];
            float ks = 1.f, vs = 1.f;
            if (FORM != kPagesPlain) {
                ks = Kscale[scale_of_row<FORM>(b, (int)from)];
                vs = Vscale[scale_of_row<FORM>(b, (int)from)];
            }
            if (page < 0) {   // a row that has no place reads as zeros
                kv = vv = make_uint4(0, 0, 0, 0);
                ks = vs = 0.f;
            }
            const long to = row * row_stride + h * head_stride + (long)p * C::kPerVec;
            restore<T, FORM>(kv, ks, K + to);
            restore<T, FORM>(vv, vs, V + to);
        }
    }
}

template <typename T, int FORM>
__global__ __launch_bounds__(256) void cache_read_kernel(PagedBatch b, const void *__restrict__ Kpages,
                                                         const void *__restrict__ Vpages, const float *__restrict__ Kscale,
                                                         const float *__restrict__ Vscale, T *K, T *V, long row_stride,
                                                         long head_stride, int group)
{
    read_row<T, FORM>(b, Kpages, Vpages, Kscale, Vscale, K, V, row_stride, head_stride, group);
}
// (pages in blocks)
template <typename T, int FORM>
__global__ __launch_bounds__(256) void blocks_read_kernel(PagedBatch b, const void *__restrict__ Kpages,
                                                          const void *__restrict__ Vpages, const float *__restrict__ Kscale,
                                                          const float *__restrict__ Vscale, T *K, T *V, long row_stride,
                                                          long head_stride, int group)
{
    read_row<T, FORM>(b, Kpages, Vpages, Kscale, Vscale, K, V, row_stride, head_stride, group);
}

// Lanes that take a (row, head) of so many pieces.
int lanes_for(int pieces)
{
    int g = 1;
    while (g < pieces && g < kWave) g <<= 1;
    return g;
}

// Four rows a workgroup; the turns that a wave would take over a row's heads, one load after the other, are dealt to several waves
// as long as the card has room for them at once, 8192 in 256 compute units.  (us, one wave a row / dealt: 2011 fp32 rows of 16 heads of 64
// written as int8 11.6 / 9.5; a call for 256 bf16 rows of 32 heads of 128 20.7 / 13.2.)
dim3 turns_grid(const PagedBatch &b, int group)
{
    const int turns = (b.H * group + kWave - 1) / kWave, room = 8192 / b.n_rows;
    return dim3((b.n_rows + 3) / 4, room < 1 ? 1 : room < turns ? room : turns);
}

}  // namespace

template <typename T, int FORM>
static hipError_t write_rows(const PagedBatch &b, const void *K, const void *V, long row_stride, long head_stride,
                             void *Kpages, void *Vpages, float *Kscale, float *Vscale, hipStream_t st)
{
    const int pieces = b.d / Elem<T>::kPerVec, group = lanes_for(pieces);
    const dim3 grid = turns_grid(b, group);
    if (pieces <= kWave)
        cache_write_kernel<T, FORM, 1><<<grid, 256, 0, st>>>(b, (const T *)K, (const T *)V, row_stride, head_stride, Kpages,
                                                             Vpages, Kscale, Vscale, group);
    else
        cache_write_kernel<T, FORM, 2><<<grid, 256, 0, st>>>(b, (const T *)K, (const T *)V, row_stride, head_stride, Kpages,
                                                             Vpages, Kscale, Vscale, group);
    return hipGetLastError();
}

hipError_t launch_cache_write(const PagedBatch &b, int dtype, int form, const void *K, const void *V, long row_stride,
                              long head_stride, void *Kpages, void *Vpages, float *Kscale, float *Vscale, hipStream_t st)
{
    auto go = [&](auto f) { return f(b, K, V, row_stride, head_stride, Kpages, Vpages, Kscale, Vscale, st); };
    if (in_blocks(form)) return launch_blocks_write(b, dtype, form, K, V, row_stride, head_stride, Kpages, Vpages, Kscale, Vscale, st);
    if (dtype == 0)
        return form == kPagesPlain ? go(write_rows<float, kPagesPlain>)
             : form == kPagesFp8   ? go(write_rows<float, kPagesFp8>) : go(write_rows<float, kPagesInt8>);
    return form == kPagesPlain ? go(write_rows<uint16_t, kPagesPlain>)
         : form == kPagesFp8   ? go(write_rows<uint16_t, kPagesFp8>) : go(write_rows<uint16_t, kPagesInt8>);
}

template <typename T, int FORM>
static hipError_t read_rows(const PagedBatch &b, const void *Kpages, const void *Vpages, const float *Kscale,
                            const float *Vscale, void *K, void *V, long row_stride, long head_stride, hipStream_t st)
{
    const int group = lanes_for(b.d / Cached<T, FORM>::kPerVec);
    auto go = [&](auto kernel) {
        kernel<<<turns_grid(b, group), 256, 0, st>>>(b, Kpages, Vpages, Kscale, Vscale, (T *)K, (T *)V, row_stride, head_stride, group);
        return hipGetLastError();
    };
    if constexpr (in_blocks(FORM)) return go(blocks_read_kernel<T, FORM>);
    else return go(cache_read_kernel<T, FORM>);
}

hipError_t launch_cache_read(const PagedBatch &b, int dtype, int form, const void *Kpages, const void *Vpages,
                             const float *Kscale, const float *Vscale, void *K, void *V, long row_stride, long head_stride,
                             hipStream_t st)
{
    return with_form(form, [&](auto f) {
        constexpr int FORM = decltype(f)::value;
        auto go = [&](auto read) { return read(b, Kpages, Vpages, Kscale, Vscale, K, V, row_stride, head_stride, st); };
        return dtype == 0 ? go(read_rows<float, FORM>) : go(read_rows<uint16_t, FORM>);
    });
}

}  // namespace gkv
