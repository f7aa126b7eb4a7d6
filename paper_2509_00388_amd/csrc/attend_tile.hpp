// Pieces of the attention kernels on the matrix cores: operands of v_mfma_f32_32x32x16_bf16 (rows in bf16) and
// v_mfma_f32_32x32x2_f32 (rows in 32 bits), keys and values on their way through the LDS, the softmax of a tile.
//
// The logits are computed with keys as rows and queries as columns, S^T = K Q^T: a lane then owns one query, and
// of a block of 32 keys it holds 16 (acc_row()), its other half-wave the rest.  The product with the values takes them as
// they lie: O^T = V^T P^T contracts over keys, and the order of a contraction is free as long as both operands keep to it,
// so P^T needs no exchange between lanes.  V^T in bf16 comes out of the LDS by gfx950's transposing read.
#pragma once
#include "attend.hpp"

namespace gkv {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Rows of 32 bits over codes in blocks, which bf16 holds as they are: queries and weights are cut into three bf16 parts of eight bits each, which
// are all that they have, and the products are three of the bf16 instruction, sixteen times as fast as that of 32 bits, over tiles of half the size.  (us, the 32-bit instruction / three
// parts, eight key heads of four, d = 128, fp8 in blocks: 200 tokens over 500 to 1500 keys 366 / 123, a token over 30000 66.5 / 29.6, 32 x 8 drafts over 300 to 2000 103 / 50, 1000 rows
// over 2000 300 / 107, two sequences of 700 over 8000 1678 / 473.  Rows with a scale each keep to the 32-bit instruction and its order of sums.)
template <typename T, int FORM> constexpr bool in_thirds() { return sizeof(T) == 4 && in_blocks(FORM); }
template <typename T, int FORM> using TileType = std::conditional_t<in_thirds<T, FORM>(), uint16_t, T>;   // of a tile's values in the LDS

// The parts of x: cut off, exactly; infinities and NaN have one.
__device__ __forceinline__ void cut_in_thirds(float x, float (&part)[3])
{
    part[0] = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    const float rest = x - part[0];
    part[1] = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
    part[2] = rest - part[1];
}

// Row of the 32x32 result in accumulator register i of a lane in half-wave hh (its column is lane % 32).
__device__ __forceinline__ constexpr int acc_row(int i, int hh) { return 8 * (i >> 2) + 4 * hh + (i & 3); }

__device__ __forceinline__ void add_block(const uint4 &a, const uint4 &b, f32x16 &acc, float)   // 32 bytes a row: 8 values
{
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), acc, 0, 0, 0);
}
__device__ __forceinline__ void add_block(const uint4 &a, const uint4 &b, f32x16 &acc, uint16_t)   // 32 bytes: 16 values
{
    union { uint4 u; bf16x8 v; } x{a}, y{b};
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.v, y.v, acc, 0, 0, 0);
}

__device__ __forceinline__ float other_half_max(float x)   // with the lane 32 places away
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_half_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Geometry of a tile of KEYS cached rows of width D (d filled up with zeros to 64, 128 or 256), moved by NT threads.
// The LDS holds values of type T; a row of keys is padded by 16 bytes, a row of values so that the transposing reads of
// four keys and 32 dimensions spread over the banks.
template <typename T, int FORM, int D, int KEYS, int NT> struct Tile {
    static constexpr int kCached = FORM == kPagesPlain ? (int)sizeof(T) : 1;   // bytes of a cached value
    static constexpr int kPieces = D * kCached / 16;                             // 16-byte pieces of a cached row
    static constexpr int kPer = (KEYS * kPieces + NT - 1) / NT;                  // pieces of a thread
    static constexpr bool kSpare = KEYS * kPieces < NT;                          // threads without one
    static constexpr int kRowStep = NT / kPieces;                                // rows between two of its pieces
    // Sixteen codes are 32 bytes in the LDS: two writes of 16.  In one place they would lie 32 bytes from those of the next lane, and half of the
    // banks would take them all; so the first halves of a segment's eight pieces lie together, the second halves 128 bytes behind.  (us, so / in one
    // place, pages in blocks: 2000 rows of four query heads a key head over 24000 keys, fp8 775 / 842, int8 758 / 818; six sequences of 445 rows over 1000 to 9000 states 175 / 190;
    // 64 tokens over 400 to 5000 keys the same.  Not with a scale a row, where the largest fp8 variant has no registers for it: 949 / 931.)
    static constexpr bool kHalves = in_blocks(FORM) && sizeof(T) == 2 && D >= 128;
    static constexpr int kKeyPitch = D * (int)sizeof(T) + 16, kValPitch = D * (int)sizeof(T) + (sizeof(T) == 2 && !kHalves ? 64 : 32);
    static constexpr int kDecoded = 16 / kCached * (int)sizeof(T);               // bytes of a piece in the LDS
    static constexpr int kHalf = kHalves ? 128 : 16;                             // between the two of a piece
    // Where a piece lies in a row.
    __device__ static __forceinline__ constexpr int piece_at(int piece) { return kHalves ? (piece >> 3) * 256 + (piece & 7) * 16 : piece * kDecoded; }
    // The 32 bytes of a row of keys that a matrix step takes: 16 of them here, 16 kHalf further.
    __device__ static __forceinline__ constexpr int step_at(int step) { return kHalves ? (step >> 3) * 256 + (step & 7) * 16 : 32 * step; }
    // Where a lane's values for the transposing reads of a block of 32 dimensions lie in a row.
    __device__ static __forceinline__ int value_at(int lane)
    {
        const int i = lane & 3, group = (lane >> 4) & 1;
        return kHalves ? group * 16 + (i >> 1) * 128 + (i & 1) * 8 : group * 32 + i * 8;
    }
    __device__ static __forceinline__ constexpr int block_at(int block) { return kHalves ? (block >> 2) * 256 + (block & 3) * 32 : 64 * block; }
    static constexpr int kSteps = D * (int)sizeof(T) / 32;                       // matrix steps of a row of keys
    static constexpr int kWaveRows = 64 / kPieces < 1 ? 1 : 64 / kPieces;        // rows of a wave's turn, next to one another
    static_assert((kSpare || KEYS * kPieces % NT == 0) && NT % kPieces == 0, "whole rows a turn");

    // Whether a piece holds an infinity or a NaN.
    __device__ static __forceinline__ bool odd(const uint4 &v)
    {
        auto any = [&](auto f) { return f(v.x) || f(v.y) || f(v.z) || f(v.w); };
        if constexpr (code_of(FORM) == kPagesFp8) return any([](uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0; });
        if constexpr (code_of(FORM) == kPagesInt8) return false;
        if constexpr (sizeof(T) == 4) return any([](uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; });
        return any([](uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u || (w & 0x7f80u) == 0x7f80u; });
    }
    // Rows of the tile, of those that this wave moves, that hold one (the pieces of a row lie in lanes of one wave).
    __device__ static __forceinline__ uint64_t odd_rows(const uint4 (&r)[kPer], int first_row)   // first_row: of lane 0
    {
        uint64_t rows = 0;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const uint64_t votes = __ballot(odd(r[u]));
            if (votes == 0) continue;
#pragma unroll
            for (int k = 0; k < 64 / kPieces; ++k)
                if ((votes >> (k * kPieces)) & (~0ull >> (64 - kPieces))) rows |= 1ull << (first_row + k + u * kRowStep);
        }
        return rows;
    }

    // The pieces of a thread: lane j has in `at` the number of the pool's row of the tile's row j.  `together`: the rows of a wave's turn
    // lie in one page (which holds kWaveRows tokens), so that their place is the same for all lanes and costs scalar instructions only; through
    // the LDS, which other waves keep busy, the numbers of a tile's rows take several hundred clocks.  offset: the lane's
    // place within the turn, in bytes.
    __device__ static __forceinline__ void ask(const void *pages, int at, bool together, int wave_row, int my_row, int row_bytes, uint32_t offset,
                                               uint4 (&r)[kPer])
    {
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            if (together) {
                const uint64_t first = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(at, wave_row + u * kRowStep) * (uint32_t)row_bytes;
                r[u] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(pages) + first + offset);
            } else {
                const uint64_t row = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (my_row + u * kRowStep), at);
                r[u] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(pages) + row * (uint32_t)row_bytes + offset % (uint32_t)row_bytes);
            }
        }
    }
    // A piece without what is not to be seen.
    __device__ static __forceinline__ uint4 only(const uint4 &v, bool seen)
    {
        const uint32_t m = seen ? ~0u : 0u;
        return make_uint4(v.x & m, v.y & m, v.z & m, v.w & m);
    }
    // One piece to its place in the LDS, decoded.
    __device__ static __forceinline__ void put(unsigned char *to, const uint4 &v)
    {
        uint4 *w = reinterpret_cast<uint4 *>(to);
        if constexpr (FORM == kPagesPlain) {
            w[0] = v;
        } else {
            if constexpr (code_of(FORM) == kPagesFp8 && sizeof(T) == 2) {   // (two codes an instruction, the scale 1)
                typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                const uint32_t c[4] = {v.x, v.y, v.z, v.w};
                union { bf16x2 b[8]; uint4 u[2]; } y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y.b[2 * e] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[e], 1.f, false);
                    y.b[2 * e + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[e], 1.f, true);
                }
                w[0] = y.u[0];
                w[kHalf / 16] = y.u[1];
                return;
            }
            float x[16];
            Cached<T, FORM>::unpack(v, x);
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    w[e / 4] = make_uint4(__float_as_uint(x[e]), __float_as_uint(x[e + 1]), __float_as_uint(x[e + 2]), __float_as_uint(x[e + 3]));
            } else {   // (codes are exact in bf16)
#pragma unroll
                for (int e = 0; e < 16; e += 8)
                    w[e / 8 * (kHalf / 16)] = make_uint4(pack_bf16(x[e], x[e + 1]), pack_bf16(x[e + 2], x[e + 3]),
                                          pack_bf16(x[e + 4], x[e + 5]), pack_bf16(x[e + 6], x[e + 7]));
            }
        }
    }
};

// Query rows as operands: rows row_of() of a lane, zeros past d and where there is no row.
template <typename T, int STEPS>
__device__ __forceinline__ void load_query(const T *row, int d, int hh, uint4 (&q)[STEPS])
{
    constexpr int PER = 16 / (int)sizeof(T);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int at = (2 * s + hh) * PER;
        q[s] = row && at < d ? *reinterpret_cast<const uint4 *>(row + at) : make_uint4(0, 0, 0, 0);
    }
}

// Four values of a query row in three parts of four bf16 numbers.
__device__ __forceinline__ void query_in_thirds(const uint4 &v, uint2 (&to)[3])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float part[4][3];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float x = __uint_as_float(w[e]);
        cut_in_thirds(x, part[e]);
        if (!(fabsf(x) <= 3.40282347e38f)) { part[e][0] = x; part[e][1] = part[e][2] = 0.f; }   // (an infinity or a NaN)
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) to[k] = make_uint2(pack_bf16(part[0][k], part[1][k]), pack_bf16(part[2][k], part[3][k]));
}
// Query rows of 32 bits as operands in three parts.
template <int STEPS>
__device__ __forceinline__ void load_query_in_thirds(const float *row, int d, int hh, uint4 (&q)[3][STEPS])
{
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        uint2 part[2][3];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int at = (2 * s + hh) * 8 + 4 * e;
            query_in_thirds(row && at < d ? *reinterpret_cast<const uint4 *>(row + at) : make_uint4(0, 0, 0, 0), part[e]);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) q[k][s] = make_uint4(part[0][k].x, part[0][k].y, part[1][k].x, part[1][k].y);
    }
}

// A lane's weights of a block of 32 keys in bf16, as operands of two matrix steps.  The rounding, at most 2^-8 of a weight, is the price of
// the bf16 matrix instruction: an output is off by about as much as by its own rounding to bf16.  Keeping what it leaves in a second
// operand (add_values_twice()) makes it 2^-15 and doubles the product: us, one operand / two:
//   attend_few   plain pages: a token over 131072 keys 105.9 / 106.1, 64 tokens 148.4 / 149.5, d = 64 84.9 / 85.6, d = 256 296.4 / 298.6
//                fp8, int8 pages, 64 tokens: 97.3 / 99.5, 98.6 / 102; d = 64 63.9 / 66.6, 63.2 / 67
//   attend_many  int8 drafts 49.4 / 51.8, seven chunks of 25 rows over 4000 keys 55.8 / 58.4
//   attend_wide  2048 rows over 32768 keys 1080 / 1473
// So few rows over plain pages, which are bound by memory, take two; values in 8 bits are far less exact than their weights.
struct Weights {
    bf16x8 w[2];
};
__device__ __forceinline__ Weights pack_weights(const float (&p)[16])
{
    Weights r;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        union { uint4 u; bf16x8 v; } w;
        w.u = make_uint4(pack_bf16(p[8 * s], p[8 * s + 1]), pack_bf16(p[8 * s + 2], p[8 * s + 3]),
                         pack_bf16(p[8 * s + 4], p[8 * s + 5]), pack_bf16(p[8 * s + 6], p[8 * s + 7]));
        r.w[s] = w.v;
    }
    return r;
}

// O^T += V^T P^T over a block of 32 keys: vt is the block's first row of values in the LDS, as L lays it out with PITCH bytes a row.
template <typename L, int D, int PITCH>
__device__ __forceinline__ void add_values(const unsigned char *vt, const Weights &p, int lane, f32x16 (&o)[D / 32])
{
    const int i = lane & 15, hh = lane >> 5;
    const unsigned char *at = vt + (4 * hh + (i >> 2)) * PITCH + L::value_at(lane);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
            // two groups of four keys, as acc_row() deals them out
            typedef __attribute__((address_space(3))) bf16x4 lds4;
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(at + 16 * s * PITCH + L::block_at(b)));
            const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(at + (16 * s + 8) * PITCH + L::block_at(b)));
            o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), p.w[s], o[b], 0, 0, 0);
        }
}
template <typename L, int D, int PITCH>
__device__ __forceinline__ void add_values(const unsigned char *vt, const float (&p)[16], int lane, f32x16 (&o)[D / 32], uint16_t)
{
    add_values<L, D, PITCH>(vt, pack_weights(p), lane, o);
}
// The same with weights in two bf16 operands: the first cut off, the second what that leaves, at most 2^-7 of the weight and rounded by 2^-8 of
// itself.  Where an infinite value meets them, both have to be above 0 (inf - inf, 0 x inf): the second is 2^-22 of the weight too large.
template <typename L, int D, int PITCH>
__device__ __forceinline__ void add_values_twice(const unsigned char *vt, const float (&p)[16], int lane, f32x16 (&o)[D / 32])
{
    float high[16], rest[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        high[i] = __uint_as_float(__float_as_uint(p[i]) & 0xffff0000u);
        rest[i] = fmaf(p[i], 1.f + 0x1p-22f, -high[i]);
    }
    add_values<L, D, PITCH>(vt, pack_weights(high), lane, o);
    add_values<L, D, PITCH>(vt, pack_weights(rest), lane, o);
}
// The same with 32-bit weights in three, nothing of which is lost.
template <typename L, int D, int PITCH>
__device__ __forceinline__ void add_values_in_thirds(const unsigned char *vt, const float (&p)[16], int lane, f32x16 (&o)[D / 32])
{
    const int i = lane & 15, hh = lane >> 5;
    const unsigned char *at = vt + (4 * hh + (i >> 2)) * PITCH + L::value_at(lane);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        float part[8][3];
#pragma unroll
        for (int e = 0; e < 8; ++e) cut_in_thirds(p[8 * s + e], part[e]);
        union { uint4 u; bf16x8 v; } w[3];
#pragma unroll
        for (int k = 0; k < 3; ++k)
            w[k].u = make_uint4(pack_bf16(part[0][k], part[1][k]), pack_bf16(part[2][k], part[3][k]), pack_bf16(part[4][k], part[5][k]), pack_bf16(part[6][k], part[7][k]));
        bf16x8 v[D / 32];
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
            typedef __attribute__((address_space(3))) bf16x4 lds4;
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(at + 16 * s * PITCH + L::block_at(b)));
            const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(at + (16 * s + 8) * PITCH + L::block_at(b)));
            v[b] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
#pragma unroll
        for (int k = 2; k >= 0; --k)
#pragma unroll
            for (int b = 0; b < D / 32; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[b], w[k].v, o[b], 0, 0, 0);
    }
}
template <typename L, int D, int PITCH>
__device__ __forceinline__ void add_values(const unsigned char *vt, const float (&p)[16], int lane, f32x16 (&o)[D / 32], float)
{
    const unsigned char *at = vt + 4 * (lane >> 5) * PITCH + (lane & 31) * 4;
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
            const float v = *reinterpret_cast<const float *>(at + acc_row(i, 0) * PITCH + 128 * b);
            o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[i], o[b], 0, 0, 0);
        }
}

// The keys of a tile that a lane's query sees, those of its half-wave at the places acc_row(i, 0): keys that exist (`vis`) and
// do not come after the tile's key `limit`.
__device__ __forceinline__ uint64_t seen_keys(uint64_t vis, int limit, int hh)
{
    const uint64_t before = limit < 0 ? 0 : limit >= 63 ? ~0ull : (2ull << limit) - 1;
    return (vis & before) >> (4 * hh);
}

// The running maximum may stay behind the true one by so much before o is brought to it: weights up to 2^8 instead of 1 change
// nothing in sums of 32 bits and nothing in the relative rounding of the weights, while of a wave's 32 queries one has a larger maximum in
// most tiles (random logits: two of three at the 32nd, one of four at the hundredth), each time for all of o's registers.  (us, without / with:
// attend_many, 300 rows of 4000 keys, d = 256 143 / 125, fp32 two sequences of 701 rows 900 / 856, 16 x 8 int8 drafts 51.2 / 49.4;
// attend_wide, 2048 rows of 32768 keys 1062 / 1032; attend_few, 64 sequences in fp8 98.2 / 97.1.)
constexpr float kMaxLag = 8.f;

// The reference m brought to the tile's maximum `top` (of all keys so far) where it has to be, sums with it; returns what to take from logits.
template <int DB>
__device__ __forceinline__ float follow_maximum(float top, float &m, float &l, f32x16 (&o)[DB])
{
    // (The vote only says whether any row has something to do: each row's reference follows its own maxima, so that how its weights are rounded
    // does not depend on what other rows see.)
    if (__any(top > m + kMaxLag)) {
        const bool grown = top > m + kMaxLag;
        const float fade = grown ? __builtin_amdgcn_exp2f(m - top) : 1.f;
        l *= fade;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][i] *= fade;
        m = grown ? top : m;
    }
    return m == -INFINITY ? 0.f : m;   // (nothing seen yet: all weights are 2^-inf)
}

// One tile of logits (NB blocks of 32 keys) to weights 2^(x - m), with the running reference m (the maximum, or up to kMaxLag below it) and
// sum l of the lane's query; o is brought to the new one.  ks: the keys' scales times c (8-bit), NB x 32 of them; c: otherwise.
// `all`: every row sees every key; otherwise `seen` has the keys that the lane's query sees (seen_keys()).
template <int FORM, int NB, int DB>
__device__ __forceinline__ void softmax_tile(f32x16 (&x)[NB], const float *ks, float c, bool all, uint64_t seen, int hh,
                                             float &m, float &l, f32x16 (&o)[DB], float (&p)[NB][16])
{
    if constexpr (FORM != kPagesPlain) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 f = *reinterpret_cast<const float4 *>(ks + 32 * b + 8 * j + 4 * hh);
                x[b][4 * j] *= f.x; x[b][4 * j + 1] *= f.y; x[b][4 * j + 2] *= f.z; x[b][4 * j + 3] *= f.w;
            }
        c = 1.f;
    }
    if (!all) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[b][i] = (seen >> (32 * b + acc_row(i, 0))) & 1 ? x[b][i] : -INFINITY;
    }
    float top = x[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, x[b][i]);
    const float shift = follow_maximum<DB>(fmaxf(m, other_half_max(top) * c), m, l, o);   // (c > 0)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[b][i] = __builtin_amdgcn_exp2f(fmaf(x[b][i], c, -shift));
            l += p[b][i];
        }
}

// The same where 16 keys from a multiple of 16 on share a scale (pages in blocks): kc[g]: the scale of group g's keys times c, vs[g]: that of its values, the first above 0.
// The weights come out times the values' scales, multiplied behind the sum.  (With the scale's logarithm in the exponent and the sum taken back by the scale's inverse, 2000 rows over
// 24000 keys in fp8 took 819 us where they take 835, but a weight whose product with its value's scale is below 2^-126 was missing from the sum; with a vote that tells such tiles
// apart, 888.)
template <int NB, int DB>
__device__ __forceinline__ void softmax_blocks(f32x16 (&x)[NB], float (&kc)[2 * NB], float (&vs)[2 * NB], bool all, uint64_t seen, int hh,
                                               float &m, float &l, f32x16 (&o)[DB], float (&p)[NB][16])
{
    if (!all) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[b][i] = (seen >> (32 * b + acc_row(i, 0))) & 1 ? x[b][i] : -INFINITY;
        // (the scales of a group that the lane sees nothing of may be anything)
#pragma unroll
        for (int g = 0; g < 2 * NB; ++g) {
            const bool any = ((seen >> (32 * (g / 2) + 16 * (g & 1))) & 0x0f0f) != 0;
            kc[g] = any ? kc[g] : 1.f;
            vs[g] = any ? vs[g] : 1.f;
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int g = 0; g < 2 * NB; ++g) {
        float most = x[g / 2][8 * (g & 1)];
#pragma unroll
        for (int i = 1; i < 8; ++i) most = fmaxf(most, x[g / 2][8 * (g & 1) + i]);
        top = fmaxf(top, most * kc[g]);
    }
    const float shift = follow_maximum<DB>(fmaxf(m, other_half_max(top)), m, l, o);
#pragma unroll
    for (int g = 0; g < 2 * NB; ++g) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float &w = p[g / 2][8 * (g & 1) + i];
            w = __builtin_amdgcn_exp2f(fmaf(x[g / 2][8 * (g & 1) + i], kc[g], -shift));
            sum += w;
            w *= vs[g];
        }
        l += sum;
    }
}
// The same with the groups' numbers from the LDS: kc at ks[0], vs at ks[4] on.
template <int NB, int DB>
__device__ __forceinline__ void softmax_groups(f32x16 (&x)[NB], const float *ks, bool all, uint64_t seen, int hh, float &m, float &l,
                                               f32x16 (&o)[DB], float (&p)[NB][16])
{
    float kc[2 * NB], vs[2 * NB];
#pragma unroll
    for (int g = 0; g < 2 * NB; ++g) {
        kc[g] = ks[g];
        vs[g] = ks[4 + g];
    }
    softmax_blocks<NB, DB>(x, kc, vs, all, seen, hh, m, l, o, p);
}
// A keys' scale times c as those need it, above 0: it multiplies the logits of hidden keys too, -infinity.  What is 0, in a block of zeros or next to it, becomes the least number:
// logits are off by 2^-21 then at most.
__device__ __forceinline__ float key_scale(float scale, float c)
{
    const float k = scale * c;
    return k == 0.f ? 0x1p-149f : k;
}

// The weights times the values' scales vs; keys that the lane does not see keep weight 0, whatever their scale.
template <int NB>
__device__ __forceinline__ void scale_weights(const float *vs, bool all, uint64_t seen, int hh, float (&p)[NB][16])
{
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float4 f = *reinterpret_cast<const float4 *>(vs + 32 * b + 8 * j + 4 * hh);
            p[b][4 * j] *= f.x; p[b][4 * j + 1] *= f.y; p[b][4 * j + 2] *= f.z; p[b][4 * j + 3] *= f.w;
        }
    if (!all) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) p[b][i] = (seen >> (32 * b + acc_row(i, 0))) & 1 ? p[b][i] : 0.f;
    }
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return bf16_to_f32(x); }

// A value of a cached row.
template <typename T, int FORM> __device__ __forceinline__ float cached_value(const void *rows, long at)
{
    if constexpr (code_of(FORM) == kPagesFp8) {
        float o[4];
        decode4<kPagesFp8>(reinterpret_cast<const uint8_t *>(rows)[at], o);
        return o[0];
    } else if constexpr (code_of(FORM) == kPagesInt8) {
        return (float)reinterpret_cast<const int8_t *>(rows)[at];
    } else if constexpr (sizeof(T) == 2) {
        return bf16_to_f32(reinterpret_cast<const uint16_t *>(rows)[at]);
    } else {
        return reinterpret_cast<const float *>(rows)[at];
    }
}

// Values with infinities or NaN at positions that only some of a block's queries see: in a tile's matrix product they would
// reach the others too (0 x inf), so they go through it as zeros, their rows are remembered, and what they add to O^T is
// added here, behind the tiles, to the queries that see them.  `odd`: rows of the tile that begins at position `first`;
// q: the lane's query row; m: its maximum.
template <typename T, int FORM, int DB>
__device__ __forceinline__ void add_odd_rows(const AttendArgs &a, int s, int h, uint64_t odd, int first, const T *q, int sees, float m,
                                               int hh, f32x16 (&o)[DB])
{
    constexpr int PER = 16 / (int)sizeof(T);
    for (; odd; odd &= odd - 1) {
        const int pos = first + __ffsll((unsigned long long)odd) - 1;
        const int page = page_of(a.b, s, pos);
        if (!q || pos > sees || page < 0) continue;
        const long row = pool_row(a.b, page, h, pos);
        float x = 0.f;   // (each half-wave every other piece of the row)
#pragma unroll 1
        for (int c = hh * PER; c < a.b.d; c += 2 * PER) {
            float y[PER];
            Elem<T>::unpack(*reinterpret_cast<const uint4 *>(q + c), y);
#pragma unroll
            for (int e = 0; e < PER; ++e) x = fmaf(y[e], cached_value<T, FORM>(a.Kpages, row * a.b.d + c + e), x);
        }
        x = other_half_sum(x) * a.c;
        float w;
        if constexpr (FORM == kPagesPlain) w = __builtin_amdgcn_exp2f(x - m);
        else w = __builtin_amdgcn_exp2f(x * a.Kscale[scale_of_row<FORM>(a.b, (int)row)] - m) * a.Vscale[scale_of_row<FORM>(a.b, (int)row)];
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int c = 32 * b + acc_row(i, hh);
                if (c < a.b.d) o[b][i] = fmaf(w, cached_value<T, FORM>(a.Vpages, row * a.b.d + c), o[b][i]);
            }
    }
}

}  // namespace gkv
