// Attention of sequences with many new rows (chunks of a prompt): bound by the matrix cores and the exponentials.
//
// A workgroup of four waves takes 128 stacked query rows of a head, 32 a wave in operand registers, and streams the keys and
// values that they see through the LDS in tiles: the next tile's loads are in flight, in registers, while this one is
// multiplied, and go to the other half of the LDS behind it; one barrier a tile.  Logits stay in registers: each wave turns
// its 32 x KEYS of them into weights and multiplies them with the values (attend_tile.hpp).  Where the blocks are too few to
// fill the chip the key tiles of a block are dealt to several workgroups and their parts joined by a second launch.
#include "attend_tile.hpp"
#include "kernels.hpp"

namespace gkv {

namespace {

template <typename T, int FORM, int D, int NB>
__global__ __launch_bounds__(256, (sizeof(T) == 4 || D > 128) ? 1 : 2) void attend_many_kernel(AttendArgs a, ManyPlan pl)
{
    constexpr int KEYS = 32 * NB, DB = D / 32;
    using L = Tile<T, FORM, D, KEYS, 256>;
    constexpr int KEYTILE = KEYS * L::kKeyPitch, HALF = KEYTILE + KEYS * L::kValPitch + (FORM == kPagesPlain ? 0 : 2 * KEYS * 4);
    constexpr uint64_t kAllKeys = KEYS == 64 ? ~0ull : (1ull << KEYS) - 1;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint32_t part[16];
    __shared__ unsigned long long odd_of[3];   // rows of the tile before, of this one and of the next that hold infinities or NaN
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hh = lane >> 5;
    const PagedBatch &b = a.b;

    // Workgroups that follow one another take the heads in turn, so that with eight of them a head's keys and values pass
    // through one XCD's L2; then the blocks of a run of keys, those that see the most keys first.
    const int h = blockIdx.x % b.H, rest = blockIdx.x / b.H, split = rest / pl.blocks;
    // (row numbers that do not ascend can count rows twice: blocks beyond those that the grid and the slots have room for are left out)
    const uint32_t unit = rest % pl.blocks;
    uint32_t total, before, block = 0;
    const int s = find_share(b.n_seqs, total, before, part, [&](int i) { return many_blocks(seq_rows(b, i), a, pl); },
                             [&](uint32_t all) {
                                 all = min(all, (uint32_t)pl.blocks);
                                 if (unit >= all) return (int64_t)-1;
                                 block = all - 1 - unit;
                                 return (int64_t)block;
                             });
    if (s < 0) return;
    const SeqRows sq = seq_rows(b, s);
    const int row0 = (int)(block - before) * kBlockRows, rows = sq.n * a.G;   // stacked rows of the sequence
    const int row = row0 + 32 * wv + l32;
    const int token = row / a.G, head = h * a.G + row % a.G;
    const int sees = sq.len - sq.n + token;                                      // last position the lane's row sees
    const int last_token = min(row0 + kBlockRows, rows) - 1;
    const int extent = max(0, sq.len - sq.n + last_token / a.G + 1);             // positions the block sees
    const int first_sees = sq.len - sq.n + row0 / a.G;                           // last position that all its rows see
    const int tiles = (extent + KEYS - 1) / KEYS;
    const int t0 = (int)((long)tiles * split / pl.splits), t1 = (int)((long)tiles * (split + 1) / pl.splits);

    const T *qrow = row < rows ? reinterpret_cast<const T *>(a.Q) + (sq.row0 + token) * a.q_row + head * a.q_head : nullptr;
    uint4 q[L::kSteps];
    load_query<T>(qrow, b.d, hh, q);

    float m = -INFINITY, l = 0.f;
    f32x16 o[DB];
#pragma unroll
    for (int x = 0; x < DB; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[x][i] = 0.f;

    const int pieces = b.d * L::kCached / 16, my_piece = tid % L::kPieces, my_row = tid / L::kPieces;
    const int wave_row = __builtin_amdgcn_readfirstlane(my_row);
    const int load_piece = min(my_piece, pieces - 1);
    const bool pad = my_piece >= pieces;
    const int my_key = lane & (KEYS - 1);   // lane j of each wave looks key j of a tile up
    auto entry = [&](int t) {
        const int pos = t * KEYS + my_key;
        return t < t1 && pos < extent ? page_of(b, s, pos) : -1;
    };
    auto place = [&](int page, int t) { return page < 0 ? 0 : pool_row(b, page, h, t * KEYS + my_key); };
    uint4 kr[L::kPer], vr[L::kPer];
    float ksr = 0.f, vsr = 0.f;
    auto load = [&](int at) {
#pragma unroll
        for (int u = 0; u < L::kPer; ++u) {
            const long r = __shfl(at, my_row + u * L::kRowStep, kWave);
            kr[u] = reinterpret_cast<const uint4 *>(a.Kpages)[r * pieces + load_piece];
            vr[u] = reinterpret_cast<const uint4 *>(a.Vpages)[r * pieces + load_piece];
        }
        if (FORM != kPagesPlain) { ksr = a.Kscale[at]; vsr = a.Vscale[at]; }
    };
    auto store = [&](int t, int page, uint64_t vis) {
        unsigned char *kt = smem + (t & 1) * HALF, *vt = kt + KEYTILE;
        uint64_t hide = ~vis, odd = 0;
        if (t * KEYS + KEYS - 1 > first_sees) {   // some rows do not see all of it
            odd = L::odd_rows(vr, wave_row) & vis;
            if (odd && lane == 0) atomicOr(&odd_of[t % 3], (unsigned long long)odd);
        }
#pragma unroll
        for (int u = 0; u < L::kPer; ++u) {
            const int r = my_row + u * L::kRowStep, c = my_piece * (16 / L::kCached) * (int)sizeof(T);
            // (places that hold no key of the sequence may hold anything: zeros instead)
            L::put(kt + r * L::kKeyPitch + c, L::only(kr[u], !(pad || ((hide >> r) & 1))));
            L::put(vt + r * L::kValPitch + c, L::only(vr[u], !(pad || (((hide | odd) >> r) & 1))));
        }
        if (FORM != kPagesPlain && wv == 0 && lane < KEYS) {
            float *ks = reinterpret_cast<float *>(vt + KEYS * L::kValPitch);
            ks[lane] = page >= 0 ? ksr * a.c : 0.f;
            ks[KEYS + lane] = page >= 0 ? vsr : 0.f;
        }
    };
    if (tid < 3) odd_of[tid] = 0;
    int page = entry(t0), at = place(page, t0), page1 = entry(t0 + 1);
    uint64_t vis = __ballot(page >= 0) & kAllKeys;
    load(at);
    __syncthreads();
    store(t0, page, vis);
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int at1 = place(page1, t + 1), page2 = entry(t + 2);
        const uint64_t vis1 = __ballot(page1 >= 0) & kAllKeys;
        load(at1);
        const unsigned char *kt = smem + (t & 1) * HALF, *vt = kt + KEYTILE;
        const float *ks = reinterpret_cast<const float *>(vt + KEYS * L::kValPitch);
        const uint64_t odd = odd_of[t % 3];
        if (tid == 0) odd_of[(t + 2) % 3] = 0;   // (its readers are behind the last barrier, its next writers behind the next)
        const bool all = vis == kAllKeys && t * KEYS + KEYS - 1 <= first_sees;
        f32x16 x[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[n][i] = 0.f;
#pragma unroll
            for (int st = 0; st < L::kSteps; ++st)
                add_block(*reinterpret_cast<const uint4 *>(kt + (32 * n + l32) * L::kKeyPitch + 32 * st + 16 * hh), q[st], x[n], T{});
        }
        float p[NB][16];
        const uint64_t seen = seen_keys(vis, sees - t * KEYS, hh);
        softmax_tile<FORM, NB, DB>(x, ks, a.c, all, seen, hh, m, l, o, p);
        if constexpr (FORM != kPagesPlain) scale_weights<NB>(ks + KEYS, all, seen, hh, p);
#pragma unroll
        for (int n = 0; n < NB; ++n) add_values<D, L::kValPitch>(vt + 32 * n * L::kValPitch, p[n], lane, o, T{});
        if (odd) add_odd_rows<T, FORM, NB, DB>(a.Vpages, odd, at, b.d, p, sees - t * KEYS, lane, o);
        store(t + 1, page1, vis1);
        __syncthreads();
        vis = vis1;
        at = at1;
        page1 = page2;
    }

    l = other_half_sum(l);
    if (row >= rows) return;
    if (pl.splits > 1) {
        float *slot = pl.slots + ((size_t)(split * pl.blocks + block) * b.H + h) * pl.slot_floats;
        const int r = 32 * wv + l32;
        if (hh == 0) { slot[kBlockRows * D + 2 * r] = m; slot[kBlockRows * D + 2 * r + 1] = l; }
#pragma unroll
        for (int x = 0; x < DB; ++x)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<float4 *>(slot + r * D + 32 * x + 8 * j + 4 * hh) =
                    make_float4(o[x][4 * j], o[x][4 * j + 1], o[x][4 * j + 2], o[x][4 * j + 3]);
        return;
    }
    if (a.lse && hh == 0) a.lse[(long)(sq.row0 + token) * b.H * a.G + head] = lse_of(m, l);
    const float f = inverse_of(l);
    T *to = reinterpret_cast<T *>(a.out) + (sq.row0 + token) * a.o_row + head * a.o_head;
#pragma unroll
    for (int x = 0; x < DB; ++x)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = 32 * x + 8 * j + 4 * hh;
            if (c >= b.d) continue;
            if constexpr (sizeof(T) == 4)
                *reinterpret_cast<float4 *>(to + c) = make_float4(o[x][4 * j] * f, o[x][4 * j + 1] * f, o[x][4 * j + 2] * f, o[x][4 * j + 3] * f);
            else
                *reinterpret_cast<uint2 *>(to + c) = make_uint2(pack_bf16(o[x][4 * j] * f, o[x][4 * j + 1] * f),
                                                                pack_bf16(o[x][4 * j + 2] * f, o[x][4 * j + 3] * f));
        }
}

// The parts of a block's runs of keys: a workgroup a (row, key-value head).
template <typename T, int D>
__global__ __launch_bounds__(256) void attend_join_many_kernel(AttendArgs a, ManyPlan pl)
{
    __shared__ uint32_t part[16];
    const PagedBatch &b = a.b;
    const int row = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
    const int s = seq_of_row(b, row, tid & 63);
    if (s >= b.n_seqs) return;
    const SeqRows sq = seq_rows(b, s);
    if (row < sq.row0 || row >= sq.row0 + sq.n || many_blocks(sq, a, pl) == 0) return;
    uint32_t before;
    weigh(b.n_seqs, s, before, part, [&](int i) { return many_blocks(seq_rows(b, i), a, pl); });
    if (before + ((row - sq.row0 + 1) * a.G - 1) / kBlockRows >= (uint32_t)pl.blocks) return;
    for (int e = tid; e < a.G * (D / 4); e += 256) {
        const int g = e / (D / 4), c4 = 4 * (e % (D / 4)), stacked = (row - sq.row0) * a.G + g, r = stacked % kBlockRows;
        const float *slot = pl.slots + ((size_t)(before + stacked / kBlockRows) * b.H + h) * pl.slot_floats;
        const size_t step = (size_t)pl.blocks * b.H * pl.slot_floats;
        float top = -INFINITY, sum = 0.f;
        for (int k = 0; k < pl.splits; ++k) top = fmaxf(top, slot[k * step + kBlockRows * D + 2 * r]);
        const float shift = top == -INFINITY ? 0.f : top;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < pl.splits; ++k) {
            const float *p = slot + k * step;
            const float f = __builtin_amdgcn_exp2f(p[kBlockRows * D + 2 * r] - shift);
            const float4 y = *reinterpret_cast<const float4 *>(p + r * D + c4);
            sum = fmaf(p[kBlockRows * D + 2 * r + 1], f, sum);
            v.x = fmaf(y.x, f, v.x); v.y = fmaf(y.y, f, v.y); v.z = fmaf(y.z, f, v.z); v.w = fmaf(y.w, f, v.w);
        }
        if (a.lse && c4 == 0) a.lse[(long)row * b.H * a.G + h * a.G + g] = lse_of(top, sum);
        if (c4 >= b.d) continue;
        const float f = inverse_of(sum);
        T *to = reinterpret_cast<T *>(a.out) + row * a.o_row + (h * a.G + g) * a.o_head + c4;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(to) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
        else *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(v.x * f, v.y * f), pack_bf16(v.z * f, v.w * f));
    }
}

// 32-key blocks of a tile: two, where the LDS holds two such tiles for two workgroups.
template <typename T, int D> constexpr int many_key_blocks() { return D * (int)sizeof(T) <= 256 ? 2 : 1; }

template <typename T, int FORM, int D>
hipError_t go_many(const AttendArgs &a, const ManyPlan &pl, hipStream_t st)
{
    constexpr int NB = many_key_blocks<T, D>(), KEYS = 32 * NB;
    using L = Tile<T, FORM, D, KEYS, 256>;
    const int lds = 2 * (KEYS * (L::kKeyPitch + L::kValPitch) + (FORM == kPagesPlain ? 0 : 8 * KEYS));
    auto kernel = attend_many_kernel<T, FORM, D, NB>;
    if (lds > 64 * 1024 && !allow_big_lds(reinterpret_cast<const void *>(kernel))) return hipErrorInvalidValue;
    kernel<<<dim3((unsigned)((size_t)pl.blocks * pl.splits * a.b.H)), 256, lds, st>>>(a, pl);
    return hipGetLastError();
}

template <typename T, int FORM> hipError_t go_many_d(const AttendArgs &a, const ManyPlan &pl, hipStream_t st)
{
    if (a.b.d <= 64) return go_many<T, FORM, 64>(a, pl, st);
    if constexpr (sizeof(T) == 2)
        if (a.b.d > 128) return go_many<T, FORM, 256>(a, pl, st);
    return go_many<T, FORM, 128>(a, pl, st);
}

}  // namespace

ManyPlan many_plan(const PagedBatch &b, int G, bool leave_few)
{
    const int D = attend_width(b.d);
    ManyPlan p{};
    p.leave_few = leave_few;
    p.blocks = (int)((long)b.n_rows * G / kBlockRows) + b.n_seqs;
    // Two workgroups a compute unit, but runs of at least 512 keys.
    const long cap = (((long)b.table_pages << b.page_shift) + 511) / 512, want = 512 / ((long)p.blocks * b.H);
    p.splits = (int)(want < 1 ? 1 : want < cap ? want : cap);
    p.slot_floats = kBlockRows * (D + 2);
    return p;
}

hipError_t launch_attend_many(const AttendArgs &a, const ManyPlan &pl, int dtype, int form, hipStream_t st)
{
    if (dtype == 0)
        return form == kPagesPlain ? go_many_d<float, kPagesPlain>(a, pl, st)
             : form == kPagesFp8   ? go_many_d<float, kPagesFp8>(a, pl, st) : go_many_d<float, kPagesInt8>(a, pl, st);
    return form == kPagesPlain ? go_many_d<uint16_t, kPagesPlain>(a, pl, st)
         : form == kPagesFp8   ? go_many_d<uint16_t, kPagesFp8>(a, pl, st) : go_many_d<uint16_t, kPagesInt8>(a, pl, st);
}

hipError_t launch_attend_join_many(const AttendArgs &a, const ManyPlan &pl, int dtype, hipStream_t st)
{
    const dim3 grid(a.b.n_rows, a.b.H);
    const int D = attend_width(a.b.d);
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(a, pl); return hipGetLastError(); };
    if (dtype == 0)
        return D == 64 ? go(attend_join_many_kernel<float, 64>) : go(attend_join_many_kernel<float, 128>);
    return D == 64 ? go(attend_join_many_kernel<uint16_t, 64>) : D == 128 ? go(attend_join_many_kernel<uint16_t, 128>) : go(attend_join_many_kernel<uint16_t, 256>);
}

}  // namespace gkv
