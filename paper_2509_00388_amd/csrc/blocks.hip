// Rows written to pages of 8-bit codes with a scale for each block of tokens of a head (graphkv_cache_write).
//
// The scale of a block is that of its largest magnitude, so rows of a block are encoded together.  Rows that a call adds to
// a block which holds earlier tokens keep its scale if it is enough for them; otherwise the scale grows to theirs, and the codes that are there are
// rounded again, round(code * old / new): a power of two apart for e4m3, in 64 bits for integers.
//
// A wave or a workgroup takes a block of a head: the largest magnitude of its new rows, then their codes; rows stay in registers between the two where
// they are few enough, else they are read again.  Which block it is follows from the row numbers: the room for blocks that the sequences before have
// ascends with them, so that votes find the sequence.  Bound by memory where rows are many: 20000 bf16 rows of eight heads of 128 to fp8 in blocks of 64 in 28 us, 4.4 TB/s; 2055 fp32 rows of
// sixteen heads of 64 to int8 in blocks of 16 in 11 us, a round of waves; a token each of 64 sequences in 4.2 us, a chain of look-ups and loads.  Blocks found from rows that
// begin one cost 64 sequences of 8 rows 10.7 us of a call where these cost 6.8; from counts of the sequences before, 2000 sequences of a row 44 instead of 17.
#include "kernels.hpp"
#include "paged.hpp"

namespace gkv {

namespace {

// The largest of a wave's numbers that are not below 0, in all lanes.
__device__ __forceinline__ float wave_largest(float x) { return __uint_as_float(wave_max_u32(__float_as_uint(x))); }

// Codes 0 .. 15 of a piece, to the scale `after`.
template <int FORM> __device__ __forceinline__ uint4 encode_again(const uint4 &v, float before, float after)
{
    const uint32_t in[4] = {v.x, v.y, v.z, v.w};
    uint32_t out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x[4];
        decode4<FORM>(in[i], x);
        if (code_of(FORM) == kPagesFp8) {
            out[i] = encode4<FORM>(x, after, before / after);   // (a power of two, or 0 where the codes become zeros)
        } else {
            out[i] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[i] |= (uint32_t)((int)rint((double)x[e] * (double)before / (double)after) & 0xff) << (8 * e);
        }
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}

// What a thread has of a block's new rows of one tensor: rows first + t * step, a piece of 16 bytes each.
template <typename T> __device__ __forceinline__ float largest_of(const uint4 &v, float a)
{
    float x[Elem<T>::kPerVec];
    Elem<T>::unpack(v, x);
#pragma unroll
    for (int e = 0; e < Elem<T>::kPerVec; ++e) a = fmaxf(a, fabsf(x[e]));
    return a;
}
template <typename T, int FORM> __device__ __forceinline__ void put_codes(char *to, const uint4 &v, float s, float inv)
{
    constexpr int PER = Elem<T>::kPerVec;
    float x[PER];
    uint32_t w[PER / 4];
    Elem<T>::unpack(v, x);
#pragma unroll
    for (int e = 0; e < PER; e += 4) w[e / 4] = s > 0.f ? encode4<FORM>(x + e, s, inv) : 0u;
    if constexpr (PER == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t *>(to) = w[0];
}

struct BlocksWrite {
    const void *K, *V;
    long row_stride, head_stride;
    void *Kpages, *Vpages;
    float *Kscale, *Vscale;
    int group, by_row;   // lanes of a row; room for blocks: one a row, or rows / tokens + 2 a sequence
};

// A block of a head is WAVES waves' work: of one, so that four heads share a workgroup, or of all four.  HELD: pieces of each tensor that a thread
// keeps between the two passes over the block's rows.
template <typename T, int FORM, int WAVES, int HELD>
__global__ __launch_bounds__(256) void blocks_write_kernel(PagedBatch b, BlocksWrite w)
{
    constexpr int PER = Elem<T>::kPerVec, THREADS = 64 * WAVES;
    __shared__ float tops[2][4];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = WAVES == 1 ? blockIdx.y * 4 + wv : blockIdx.y, tid = WAVES == 1 ? lane : threadIdx.x;
    if (h >= b.H) return;
    const int at = tid & (w.group - 1), mine = tid / w.group, step = THREADS / w.group, pieces = b.d / PER;
    const int tokens = 1 << b.scale_shift;
    const T *K = reinterpret_cast<const T *>(w.K) + h * w.head_stride, *V = reinterpret_cast<const T *>(w.V) + h * w.head_stride;

    // Each sequence has room for as many blocks as its rows may lie in, and this is one of them.
    const int number = blockIdx.x;
    auto room_to = [&](int s) {   // of all sequences up to s
        const int rows = min(max(b.row_start[s + 1], 0), b.n_rows);
        return w.by_row ? rows : (rows >> b.scale_shift) + 2 * (s + 1);
    };
    int s = 0, among = b.n_seqs;
    narrow_down(s, among, lane, [&](int x) { return room_to(x) <= number; });
    if (among == 0) return;
    const int x = s + min(lane, among - 1);
    const SeqRows q = seq_rows(b, x);
    const int l = (int)__popcll(__ballot(lane < among && room_to(x) <= number));
    if (l >= among) return;
    auto of_lane = [l](int v) { return __builtin_amdgcn_readlane(v, l); };
    s += l;
    const int q_row0 = of_lane(q.row0), n = of_lane(q.n), len = of_lane(q.len), which = number - (w.by_row ? q_row0 : (q_row0 >> b.scale_shift) + 2 * s);
    // (more rows than the sequence is long: the first have no place)
    const int lo = max(len - n, 0), row0 = q_row0 + n - len;   // the first new position, the row of position 0, were it there
    if (n <= 0 || len <= 0 || which < 0 || which > ((len - 1) >> b.scale_shift) - (lo >> b.scale_shift)) return;
    const int begin = ((lo >> b.scale_shift) + which) << b.scale_shift;   // the block's first position
    const int pos = max(begin, lo), inside = pos - begin, rest = min(begin + tokens, len) - pos, first = row0 + pos;
    const int page = raw_page(b, s, pos);
    auto row_of = [&](const T *x, int r) { return reinterpret_cast<const uint4 *>(x + (first + r) * w.row_stride); };
    const bool held = rest <= HELD * step && pieces <= w.group;
    const int turns = (rest + step - 1) / step;
    uint4 kv[HELD], vv[HELD];
    if (held) {
#pragma unroll
        for (int t = 0; t < HELD; ++t) {   // (a turn or lane without a piece takes another's: neither largest nor code changes by that)
            const int r = min(mine + min(t, turns - 1) * step, rest - 1), p = min(at, pieces - 1);
            kv[t] = row_of(K, r)[p];
            vv[t] = row_of(V, r)[p];
        }
    }
    if (!is_page(b, page)) return;

    const int base = pool_row(b, page, h, begin), block = base >> b.scale_shift;
    const float kb = inside > 0 ? w.Kscale[block] : 0.f, vb = inside > 0 ? w.Vscale[block] : 0.f;
    char *kto = reinterpret_cast<char *>(w.Kpages) + (long)base * b.d, *vto = reinterpret_cast<char *>(w.Vpages) + (long)base * b.d;
    float ks, vs, kinv, vinv;
    // The block's scales, from its new rows' largest magnitudes; codes that are there to the new ones.
    auto settle = [&](float ka, float va) {
        ka = wave_largest(ka);
        va = wave_largest(va);
        if constexpr (WAVES > 1) {
            if (lane == 0) { tops[0][wv] = ka; tops[1][wv] = va; }
            __syncthreads();
            ka = fmaxf(fmaxf(tops[0][0], tops[0][1]), fmaxf(tops[0][2], tops[0][3]));
            va = fmaxf(fmaxf(tops[1][0], tops[1][1]), fmaxf(tops[1][2], tops[1][3]));
        }
        ks = fmaxf(kb, scale_of<FORM>(ka));
        vs = fmaxf(vb, scale_of<FORM>(va));
        kinv = ks > 0.f ? 1.f / ks : 0.f;
        vinv = vs > 0.f ? 1.f / vs : 0.f;
        if (tid == 0) { w.Kscale[block] = ks; w.Vscale[block] = vs; }
        const int old = kb < ks || vb < vs ? inside * (b.d / 16) : 0;   // (the codes before the first new row are a run of them)
#pragma unroll 1
        for (int p = tid; p < old; p += THREADS) {
            if (kb < ks) { uint4 *x = reinterpret_cast<uint4 *>(kto) + p; *x = encode_again<FORM>(*x, kb, ks); }
            if (vb < vs) { uint4 *x = reinterpret_cast<uint4 *>(vto) + p; *x = encode_again<FORM>(*x, vb, vs); }
        }
        kto += (long)inside * b.d;
        vto += (long)inside * b.d;
    };
    if (held) {
        float ka = 0.f, va = 0.f;
#pragma unroll
        for (int t = 0; t < HELD; ++t) {
            ka = largest_of<T>(kv[t], ka);
            va = largest_of<T>(vv[t], va);
        }
        settle(ka, va);
#pragma unroll
        for (int t = 0; t < HELD; ++t)   // (what was unpacked for the largest is not kept: it would take the registers of half the waves)
            asm volatile("" : "+v"(kv[t].x), "+v"(kv[t].y), "+v"(kv[t].z), "+v"(kv[t].w), "+v"(vv[t].x), "+v"(vv[t].y), "+v"(vv[t].z), "+v"(vv[t].w));
#pragma unroll
        for (int t = 0; t < HELD; ++t)
            if (t < turns) {
                const int to = min(mine + t * step, rest - 1) * b.d + min(at, pieces - 1) * PER;
                put_codes<T, FORM>(kto + to, kv[t], ks, kinv);
                put_codes<T, FORM>(vto + to, vv[t], vs, vinv);
            }
    } else {
        float ka = 0.f, va = 0.f;
        for (int r = mine; r < rest; r += step)
#pragma unroll 1
            for (int p = at; p < pieces; p += w.group) {
                ka = largest_of<T>(row_of(K, r)[p], ka);
                va = largest_of<T>(row_of(V, r)[p], va);
            }
        settle(ka, va);
        for (int r = mine; r < rest; r += step)
#pragma unroll 1
            for (int p = at; p < pieces; p += w.group) {
                put_codes<T, FORM>(kto + (long)r * b.d + p * PER, row_of(K, r)[p], ks, kinv);
                put_codes<T, FORM>(vto + (long)r * b.d + p * PER, row_of(V, r)[p], vs, vinv);
            }
    }
}

}  // namespace

hipError_t launch_blocks_write(const PagedBatch &b, int dtype, int form, const void *K, const void *V, long row_stride,
                               long head_stride, void *Kpages, void *Vpages, float *Kscale, float *Vscale, hipStream_t st)
{
    const int pieces = b.d / (dtype == 0 ? 4 : 8);
    int group = 1;
    while (group < pieces && group < kWave) group <<= 1;
    const int tokens = 1 << b.scale_shift, most = b.max_rows < tokens ? b.max_rows : tokens;   // new rows of a block
    const int at_once = kWave / group;   // rows that a wave takes at once
    const bool one_wave = most <= 8 * at_once;   // (400 rows of 128 bf16: blocks of 32 in 9.9 us by a wave, 13.3 by four; of 64, twice as many turns, 22.2 and 12.6)
    // n rows of a sequence lie in (n - 2) / tokens + 2 blocks at most, and in n.
    const long blocks = b.n_rows / tokens + 2l * b.n_seqs;
    const int by_row = blocks >= b.n_rows;
    const BlocksWrite w{K, V, row_stride, head_stride, Kpages, Vpages, Kscale, Vscale, group, by_row};
    const dim3 grid(by_row ? b.n_rows : (int)blocks, one_wave ? (b.H + 3) / 4 : b.H);
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(b, w); return hipGetLastError(); };
    auto with_size = [&](auto type, auto f) {
        using T = decltype(type);
        constexpr int FORM = decltype(f)::value;
        // (pieces held, one / eight, us of a call: 64 sequences of a row 5.8 / 6.4, 2000 17.2 / 26.2)
        return most <= at_once ? go(blocks_write_kernel<T, FORM, 1, 1>)
             : one_wave        ? go(blocks_write_kernel<T, FORM, 1, 8>) : go(blocks_write_kernel<T, FORM, 4, 4>);
    };
    auto with_type = [&](auto f) {
        if (dtype == 0) return with_size(float{}, f);
        return with_size(uint16_t{}, f);
    };
    return form == kBlocksFp8 ? with_type(std::integral_constant<int, kBlocksFp8>{}) : with_type(std::integral_constant<int, kBlocksInt8>{});
}

}  // namespace gkv
