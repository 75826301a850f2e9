// Attention over the blocks that each query row keeps (gfx950):
//
//   out[row][h] = sum_t softmax_t(scale * q[row][h].K[t]) * V[t],  t <= position of the row, t in a block of selected[row][h / group]
//
// A list names blocks of the row's own sequence by their place in it, in any order; entries below 0 or past the row's own block are
// passed over.  A unit of work is (row, KV head, chunk of up to 16 of its heads).  How long a list is the host knows, so the launch is cut
// into equal parts without looking at the lengths:
//   few units: the list of each is cut over several workgroups; the last one to finish a part joins all of them
//     (each stores its part by device-scope accesses, waits for the stores and counts itself; nobody waits for anybody);
//   more: a workgroup per unit, whose wavefronts take the tiles of the list in turn and meet in LDS;
//   many: a wavefront per unit, nothing to join.
#include "cache_rows.h"
#include "kvc_internal.h"
#include "pa_partials.h"

namespace kvc {

namespace {

using namespace mfma;

constexpr int kWindow = 512;  // list entries whose places are held in LDS at a time (vector ALUs)

// ---- bf16 on the matrix cores, up to 16 heads of a KV head (blocks of 4 tokens and more)

// Weights as a sum of two bf16 values, see compute_tile of head_dim 64.
__device__ inline void split_weights(float p0, float p1, uint32_t *hi, uint32_t *lo) {
    const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
    *hi = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
    *lo = pack_bf16(__builtin_fmaf(p0, 1.f + FLT_EPSILON, -__uint_as_float(u0 & 0xffff0000u)),
                    __builtin_fmaf(p1, 1.f + FLT_EPSILON, -__uint_as_float(u1 & 0xffff0000u)));
}

// limit[h]: how many of this lane's tokens 16 h + 4 quad .. + 3 of the tile count; full: all of every lane's.
__device__ inline void attend_tile(HeadStateN<8> &st, Shape<128>::Tile &t, const bf16x8 (&qb)[4], float scale_log2e, const int (&limit)[1], bool full) {
    floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[j]), qb[j], s, 0, 0, 0);
    float sv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sv[i] = s[i] * scale_log2e;
    if (!full) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i >= limit[0]) {
                sv[i] = -INFINITY;
                t.v[i] = uint4{0u, 0u, 0u, 0u};
            }
    }
    const float mx = lanes::max_over_rows(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])));
    const float m_new = fmaxf(st.m, mx), alpha = __builtin_amdgcn_exp2f(st.m - m_new);
    st.m = m_new;
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(sv[i] - m_new);
    st.l = fmaf(st.l, alpha, (p[0] + p[1]) + (p[2] + p[3]));
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) st.acc[e] *= alpha;
    }
    uint2 hi, lo;
    split_weights(p[0], p[1], &hi.x, &lo.x);
    split_weights(p[2], p[3], &hi.y, &lo.y);
    const shortx4 ph = __builtin_bit_cast(shortx4, hi), pl = __builtin_bit_cast(shortx4, lo);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        auto dword = [&](int i) { return w == 0 ? t.v[i].x : w == 1 ? t.v[i].y : w == 2 ? t.v[i].z : t.v[i].w; };
        const uint32_t v0 = dword(0), v1 = dword(1), v2 = dword(2), v3 = dword(3);
        const shortx4 even = __builtin_bit_cast(shortx4, uint2{__builtin_amdgcn_perm(v1, v0, 0x05040100u), __builtin_amdgcn_perm(v3, v2, 0x05040100u)});
        const shortx4 odd = __builtin_bit_cast(shortx4, uint2{__builtin_amdgcn_perm(v1, v0, 0x07060302u), __builtin_amdgcn_perm(v3, v2, 0x07060302u)});
        st.acc[2 * w] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(even, ph, st.acc[2 * w], 0, 0, 0);
        st.acc[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(odd, ph, st.acc[2 * w + 1], 0, 0, 0);
        st.acc[2 * w] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(even, pl, st.acc[2 * w], 0, 0, 0);
        st.acc[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(odd, pl, st.acc[2 * w + 1], 0, 0, 0);
    }
}

__device__ inline void attend_tile(HeadStateN<4> &st, Shape<64>::Tile &t, const bf16x8 (&qb)[2], float scale_log2e, const int (&limit)[2], bool full) {
    float sv[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 2; ++j) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[2 * h + j]), qb[j], s, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) sv[4 * h + i] = s[i] * scale_log2e;
    }
    if (!full) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((i & 3) >= limit[i >> 2]) {
                sv[i] = -INFINITY;
                t.v[i] = uint2{0u, 0u};
            }
    }
    const float mx = lanes::max_over_rows(fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7]))));
    const float m_new = fmaxf(st.m, mx), alpha = __builtin_amdgcn_exp2f(st.m - m_new);
    st.m = m_new;
    float sum = 0.f;
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float p0 = __builtin_amdgcn_exp2f(sv[2 * i] - m_new), p1 = __builtin_amdgcn_exp2f(sv[2 * i + 1] - m_new);
        sum += p0 + p1;
        split_weights(p0, p1, hi + i, lo + i);
    }
    st.l = fmaf(st.l, alpha, sum);
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) st.acc[e] *= alpha;
    }
    const bf16x8 ph = __builtin_bit_cast(bf16x8, uint4{hi[0], hi[1], hi[2], hi[3]}), pl = __builtin_bit_cast(bf16x8, uint4{lo[0], lo[1], lo[2], lo[3]});
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        uint32_t d[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = w == 0 ? t.v[i].x : t.v[i].y;
        auto pairs = [&](uint32_t which) {
            return __builtin_bit_cast(bf16x8, uint4{__builtin_amdgcn_perm(d[1], d[0], which), __builtin_amdgcn_perm(d[3], d[2], which),
                                                    __builtin_amdgcn_perm(d[5], d[4], which), __builtin_amdgcn_perm(d[7], d[6], which)});
        };
        const bf16x8 even = pairs(0x05040100u), odd = pairs(0x07060302u);
        st.acc[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, ph, st.acc[2 * w], 0, 0, 0);
        st.acc[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, ph, st.acc[2 * w + 1], 0, 0, 0);
        st.acc[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, pl, st.acc[2 * w], 0, 0, 0);
        st.acc[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, pl, st.acc[2 * w + 1], 0, 0, 0);
    }
}

// Where unit u of a row's list lies (a unit is the part of a tile inside one block): its index in the pool, and how many of its tokens
// count.  A unit of which none does lies where the row's own block is: it may be loaded.
struct ListOf {
    const int32_t *selected, *table;
    int pos, own_block;  // position of the row, pool index of the block that holds it
    int num_kv_heads, kvh, block_size_log2, unit_log2, units_per_block_log2, budget, max_blocks_per_seq;
    // The entry and what the table says at it are asked for without waiting for the row's position.
    __device__ int2 unit(int u) const {
        const int entry = u >> units_per_block_log2, in_block = u & ((1 << units_per_block_log2) - 1);
        const int b = entry < budget ? selected[entry] : -1;
        const int named = table[min(max(b, 0), max_blocks_per_seq - 1)];
        const bool there = b >= 0 && b <= pos >> block_size_log2;
        const int block = there ? named : own_block;
        const int token = (b << block_size_log2) + (in_block << unit_log2);
        return int2{((block * num_kv_heads + kvh) << units_per_block_log2) + (there ? in_block : 0),
                    there ? min(max(pos + 1 - token, 0), 1 << unit_log2) : 0};
    }
};

// Tiles first, first + step, ... below `tiles` of a list's part that begins at tile0.  Whether any token counted.  A lane holds the place of
// one unit; 64 >> units_log2 tiles are known at a time.  UNIFORM: units of 16 tokens and more, whose places are the same for all lanes.
// AGAIN: rows near this one read the same blocks, so loads leave them in L2 (1000 rows of chunks, 32 / 8 heads of 64: XXX us, with
// the streaming loads of a decode step YYY).
template <int HD, bool UNIFORM, bool AGAIN>
__device__ inline bool attend_list(typename Shape<HD>::State &st, const bf16x8 (&qb)[Shape<HD>::kQ], const uint16_t *__restrict__ k_cache,
                                   const uint16_t *__restrict__ v_cache, const ListOf &list, float scale_log2e, int tile0, int tiles, int first, int step) {
    using TS = Shape<HD>;
    using Tile = typename TS::Tile;
    constexpr int kSubs = TS::kTokens / 16;
    struct Piece {
        Tile t;
        int limit[kSubs];
        bool full;
    };
    const int lane = threadIdx.x & 63, quad = lane >> 4, r = lane & 15;
    const int unit_log2 = list.unit_log2, units_log2 = TS::kTokensLog2 - unit_log2, unit_tokens = 1 << unit_log2;
    const int k_off = (r & (unit_tokens - 1)) * HD + 8 * quad, v_off = ((4 * quad) & (unit_tokens - 1)) * HD + HD / 16 * r;
    const size_t unit_elems = size_t(unit_tokens) * HD;
    bool any = false;
    for (int from = first; from < tiles; from += step << (6 - units_log2)) {
        const int mine = from + step * (lane >> units_log2);
        int2 e = {0, 0};
        if (mine < tiles) e = list.unit(((tile0 + mine) << units_log2) + (lane & ((1 << units_log2) - 1)));
        const uint64_t there = __ballot(e.y > 0);
        if (there == 0) continue;
        any = true;
        const int count = ((63 - __builtin_clzll(there)) >> units_log2) + 1;
        auto issue = [&](Piece &x, int i) __attribute__((always_inline)) {
            bool full = true;
#pragma unroll
            for (int h = 0; h < kSubs; ++h) {
                const uint16_t *kp, *vp;
                if constexpr (UNIFORM) {
                    // a unit is the tile, or (32-token tiles, blocks of 16) half of it
                    const bool half = kSubs == 2 && units_log2 == 1;
                    const int at = half ? 2 * i + h : i, in_unit = half ? 0 : 16 * h;
                    const size_t base = size_t(uint32_t(__builtin_amdgcn_readlane(e.x, at))) * unit_elems + in_unit * HD;
                    const int counts = __builtin_amdgcn_readlane(e.y, at) - in_unit;
                    kp = k_cache + base + k_off;
                    vp = v_cache + base + v_off;
                    full &= counts >= 16;
                    x.limit[h] = min(max(counts - 4 * quad, 0), 4);
                } else {
                    const int k_at = (i << units_log2) + ((16 * h + r) >> unit_log2), v_at = (i << units_log2) + ((16 * h + 4 * quad) >> unit_log2);
                    kp = k_cache + size_t(uint32_t(__shfl(e.x, k_at))) * unit_elems + k_off;
                    vp = v_cache + size_t(uint32_t(__shfl(e.x, v_at))) * unit_elems + v_off;
                    x.limit[h] = min(max(__shfl(e.y, v_at) - ((4 * quad) & (unit_tokens - 1)), 0), 4);
                    full &= __ballot(x.limit[h] < 4) == 0;
                }
                auto load16 = [](const uint16_t *p) { return AGAIN ? *reinterpret_cast<const uint4 *>(p) : load16_stream(p); };
                auto load8 = [](const uint16_t *p) { return AGAIN ? *reinterpret_cast<const uint2 *>(p) : load8_stream(p); };
                if constexpr (HD == 128) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) x.t.k[j] = load16(kp + 32 * j);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x.t.v[j] = load16(vp + j * HD);
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j) x.t.k[2 * h + j] = load16(kp + 32 * j);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x.t.v[4 * h + j] = load8(vp + j * HD);
                }
            }
            x.full = full;
        };
        auto compute = [&](Piece &x) __attribute__((always_inline)) { attend_tile(st, x.t, qb, scale_log2e, x.limit, x.full); };
        Piece A, B;
        issue(A, 0);
        int i = 0;
        for (; i + 2 < count; i += 2) {
            issue(B, i + 1);
            compute(A);
            issue(A, i + 2);
            compute(B);
        }
        if (i + 1 < count) {
            issue(B, i + 1);
            compute(A);
            compute(B);
        } else {
            compute(A);
        }
    }
    return any;
}

// The row, KV head and heads of a unit.
struct Unit {
    int row, kvh, head0, heads, n, pos;
    bool there;  // the row belongs to a sequence
    __device__ Unit(const SelectedArgs &a, const int32_t *q_start, const int32_t *context_lens, int row_, int kvh_, int chunk) {
        row = row_;
        kvh = kvh_;
        head0 = kvh * a.group + chunk * a.heads_per_chunk;
        heads = min(a.heads_per_chunk, (kvh + 1) * a.group - head0);
        there = find_row(row, q_start, context_lens, a.num_seqs, a.max_context_len, &n, &pos);
    }
};
__device__ inline ListOf list_of(const SelectedArgs &a, const Unit &u, const int32_t *selected, const int32_t *block_tables) {
    const int32_t *table = block_tables + int64_t(u.n) * a.max_blocks_per_seq;
    return ListOf{selected + (int64_t(u.row) * a.num_kv_heads + u.kvh) * a.budget, table, u.pos, table[u.pos >> a.block_size_log2],
                  a.num_kv_heads, u.kvh, a.block_size_log2, a.unit_log2, a.units_per_block_log2, a.budget, a.max_blocks_per_seq};
}

// A wavefront per unit; blockIdx.x = KV head + KV heads * group of kWaves rows, so that with 8 KV heads each XCD keeps one.
template <int HD, bool UNIFORM>
__global__ __launch_bounds__(kThreads, 3) void pa_selected_wave_kernel(
    const uint16_t *__restrict__ q, const uint16_t *__restrict__ k_cache, const uint16_t *__restrict__ v_cache, const int32_t *__restrict__ block_tables,
    const int32_t *__restrict__ context_lens, const int32_t *__restrict__ q_start, const int32_t *__restrict__ selected, uint16_t *__restrict__ out,
    SelectedArgs a) {
    using TS = Shape<HD>;
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, quad = lane >> 4, r = lane & 15;
    const int group = blockIdx.x / a.num_kv_heads, row = group * kWaves + wave;
    if (row >= a.total_q) return;
    const Unit u(a, q_start, context_lens, row, blockIdx.x - group * a.num_kv_heads, blockIdx.y);
    if (!u.there) return;
    uint16_t *dst = out + (int64_t(row) * a.num_q_heads + u.head0 + r) * HD + HD / 4 * quad;
    typename TS::State st;
    st.reset();
    bool any = false;
    if (u.pos >= 0) {
        bf16x8 qb[TS::kQ];
        load_q_operand(qb, q + (int64_t(row) * a.num_q_heads + u.head0 + (r < u.heads ? r : 0)) * HD, quad, r < u.heads);
        any = attend_list<HD, UNIFORM, true>(st, qb, k_cache, v_cache, list_of(a, u, selected, block_tables), a.scale_log2e, 0, a.tiles, 0, 1);
    }
    st.finish();
    if (r >= u.heads) return;
    const float inv = 1.0f / st.l;
#pragma unroll
    for (int v = 0; v < TS::kVecs; v += 2) {
        const float4 x = acc_vec(st, v), y = acc_vec(st, v + 1);
        const uint4 w = {pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv), pack_bf16(y.x * inv, y.y * inv), pack_bf16(y.z * inv, y.w * inv)};
        *reinterpret_cast<uint4 *>(dst + 4 * v) = any ? w : uint4{0u, 0u, 0u, 0u};
    }
}

// A workgroup per part of a unit's list; blockIdx.x = KV head + KV heads * row, blockIdx.y = chunk of heads, blockIdx.z = part.
template <int HD, bool UNIFORM, bool AGAIN, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void pa_selected_mfma_kernel(
    const uint16_t *__restrict__ q, const uint16_t *__restrict__ k_cache, const uint16_t *__restrict__ v_cache, const int32_t *__restrict__ block_tables,
    const int32_t *__restrict__ context_lens, const int32_t *__restrict__ q_start, const int32_t *__restrict__ selected, uint16_t *__restrict__ out,
    Workspace ws, SelectedArgs a) {
    using TS = Shape<HD>;
    constexpr int NV = TS::kVecs;
    __shared__ float4 s_acc[WAVES][16 * HD / 4];
    __shared__ float2 s_ml[kMaxSelectedParts][16];  // of the wavefronts, then of the parts
    __shared__ int s_last;
    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, quad = lane >> 4, r = lane & 15;
    const int row = blockIdx.x / a.num_kv_heads, parts = a.parts, part = blockIdx.z;
    const Unit u(a, q_start, context_lens, row, blockIdx.x - row * a.num_kv_heads, blockIdx.y);
    if (!u.there) return;
    uint16_t *dst = out + (int64_t(row) * a.num_q_heads + u.head0) * HD;
    if (u.pos < 0) {
        if (part == 0)
            for (int i = tid; i < u.heads * HD / 8; i += (64 * WAVES)) reinterpret_cast<uint4 *>(dst)[i] = uint4{0u, 0u, 0u, 0u};
        return;
    }
    bf16x8 qb[TS::kQ];
    load_q_operand(qb, q + (int64_t(row) * a.num_q_heads + u.head0 + (r < u.heads ? r : 0)) * HD, quad, r < u.heads);
    typename TS::State st;
    st.reset();
    const int tile0 = part * a.tiles_per_part;
    const bool any = attend_list<HD, UNIFORM, true>(st, qb, k_cache, v_cache, list_of(a, u, selected, block_tables), a.scale_log2e, tile0,
                                              min(a.tiles_per_part, a.tiles - tile0), wave, WAVES);
    st.finish();
    // a wavefront or part without a token says so with a maximum of -inf (with tokens it is -FLT_MAX at least)
#pragma unroll
    for (int v = 0; v < NV; ++v) s_acc[wave][(v * 4 + quad) * 16 + r] = acc_vec(st, v);
    if (quad == 0) s_ml[wave][r] = float2{any ? st.m : -INFINITY, st.l};
    __syncthreads();
    const int vecs = u.heads * HD / 4;
    const int64_t slot0 = (int64_t(blockIdx.x) * gridDim.y + blockIdx.y) * parts;
    const uint32_t slots = uint32_t(gridDim.x * gridDim.y) * parts, slot_vecs = 16 * HD / 4;
    const __amdgpu_buffer_rsrc_t acc_buf = raw_buffer(ws.acc, parts > 1 ? slots * slot_vecs * 16u : 0u), ml_buf = raw_buffer(ws.ml, parts > 1 ? slots * 16u * 8u : 0u);
    // vector f of the output: dims 4 d .. 4 d + 3 of a head
    auto place = [&](int f, int *head) __attribute__((always_inline)) {
        *head = f / (HD / 4);
        const int d = f % (HD / 4);
        return ((d % NV) * 4 + d / NV) * 16 + *head;  // a quad holds HD / 4 dims, NV vectors
    };
    auto add = [](float4 &x, float w, const float4 &y) __attribute__((always_inline)) {
        x.x = fmaf(w, y.x, x.x);
        x.y = fmaf(w, y.y, x.y);
        x.z = fmaf(w, y.z, x.z);
        x.w = fmaf(w, y.w, x.w);
    };
    auto write_out = [&](int f, const float4 &x, float M, float L) __attribute__((always_inline)) {
        const float inv = 1.0f / L;  // no token in the list: zeros
        const uint2 w = {pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv)};
        reinterpret_cast<uint2 *>(dst)[f] = M == -INFINITY ? uint2{0u, 0u} : w;
    };
    auto weight = [](float m, float M) __attribute__((always_inline)) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M); };
    for (int f = tid; f < vecs; f += (64 * WAVES)) {
        int head;
        const int at = place(f, &head);
        float M = -INFINITY, L = 0.f;
        float4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) M = fmaxf(M, s_ml[w][head].x);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float2 ml = s_ml[w][head];
            const float wgt = weight(ml.x, M);
            L = fmaf(wgt, ml.y, L);
            add(x, wgt, s_acc[w][at]);
        }
        if (parts == 1) {
            write_out(f, x, M, L);
        } else {
            store4_device_scope(acc_buf, (uint32_t(slot0 + part) * slot_vecs + at) * 16u, x.x, x.y, x.z, x.w);
            if (f % (HD / 4) == 0) store2_device_scope(ml_buf, (uint32_t(slot0 + part) * 16u + head) * 8u, M, L);
        }
    }
    if (parts == 1) return;
    // the count may become visible only after the part: every wavefront waits for its own stores, then all meet
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int32_t *const counter = ws.cnt + blockIdx.x * gridDim.y + blockIdx.y;
    if (tid == 0) s_last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
    __syncthreads();
    if (!s_last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");  // the fetches stay behind the count
    if (tid == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // thread (share, f) takes the parts share, share + shares, ... of vector f, the first of them beside the maxima and sums; the shares of
    // a vector meet in LDS
    const int shares = max(1, (64 * WAVES) / vecs), share = tid / vecs;
    constexpr int kBatch = 4;
    float4 y[kBatch];
    auto fetch = [&](int at, int p0) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            y[j] = load4_device_scope(acc_buf, (uint32_t(slot0 + min(p0 + j * shares, parts - 1)) * slot_vecs + at) * 16u);
    };
    int head0;
    if (share < shares) fetch(place(tid - share * vecs, &head0), share);
    for (int i = tid; i < parts * u.heads; i += (64 * WAVES)) {
        const int p = i / u.heads, head = i - p * u.heads;
        s_ml[p][head] = load2_device_scope(ml_buf, (uint32_t(slot0 + p) * 16u + head) * 8u);
    }
    __syncthreads();
    float4 *const s_share = &s_acc[0][0];
    for (int f0 = 0; f0 < vecs; f0 += (64 * WAVES)) {  // more than once only for more vectors than threads, one share each then
        const int f = shares > 1 ? tid - share * vecs : f0 + tid;
        const bool active = share < shares && f < vecs;
        int head = 0;
        float M = -INFINITY, L = 0.f;
        float4 x = {0.f, 0.f, 0.f, 0.f};
        if (active) {
            const int at = place(f, &head);
            for (int p = 0; p < parts; ++p) M = fmaxf(M, s_ml[p][head].x);
            for (int p0 = shares > 1 ? share : 0; p0 < parts; p0 += kBatch * shares) {
                if (p0 != share || f0 != 0) fetch(at, p0);
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    const int p = p0 + j * shares;
                    if (p >= parts) break;
                    add(x, weight(s_ml[p][head].x, M), y[j]);
                }
            }
            for (int p = 0; p < parts; ++p) L = fmaf(weight(s_ml[p][head].x, M), s_ml[p][head].y, L);
        }
        if (shares > 1) {
            if (active) s_share[tid] = x;
            __syncthreads();
            if (share == 0 && active)
                for (int i = 1; i < shares; ++i) add(x, 1.f, s_share[i * vecs + f]);
            if (share > 0) continue;
        }
        if (active) write_out(f, x, M, L);
    }
}

// ---- any type, block size and group on the vector ALUs: HEADS heads of a KV head per workgroup

template <class T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int N = 4;
    __device__ static void get(const uint4 &w, float (&x)[4]) {
        x[0] = __uint_as_float(w.x);
        x[1] = __uint_as_float(w.y);
        x[2] = __uint_as_float(w.z);
        x[3] = __uint_as_float(w.w);
    }
    __device__ static float out(float x) { return x; }
};
template <>
struct Vec<uint16_t> {
    static constexpr int N = 8;
    __device__ static void get(const uint4 &w, float (&x)[8]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
    __device__ static uint16_t out(float x) { return f32_to_bf16_rne(x); }
};

// x summed over aligned groups of LR lanes (8, 16 or 32) inside the vector ALU.
template <int LR>
__device__ inline float sum_over_lanes(float x) {
    x += lanes::permuted<lanes::kXor1>(x);
    x += lanes::permuted<lanes::kXor2>(x);
    x += lanes::permuted<lanes::kMirror8>(x);
    if constexpr (LR > 8) x += lanes::permuted<lanes::kMirror16>(x);
    if constexpr (LR > 16) {
        const lanes::Pair<float> b = lanes::pair_of<16>(x);
        x = b.first + b.second;
    }
    return x;
}
__device__ inline void store_device(float *p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline float load_device(const float *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Grid as above, the chunk of heads HEADS of them.
template <class T, int D, int HEADS>
__global__ __launch_bounds__(kThreads) void pa_selected_valu_kernel(const T *__restrict__ q, const T *__restrict__ k_cache, const T *__restrict__ v_cache,
                                                                    const int32_t *__restrict__ block_tables, const int32_t *__restrict__ context_lens,
                                                                    const int32_t *__restrict__ q_start, const int32_t *__restrict__ selected,
                                                                    T *__restrict__ out, Workspace ws, SelectedArgs a) {
    constexpr int N = Vec<T>::N, LR = D / N, TOKENS = 64 / LR, U = 4;
    __shared__ int2 s_entry[kWindow];  // pool index of a block, tokens of it that count
    __shared__ int s_last;
    __shared__ float s_m[kMaxSelectedParts][HEADS], s_l[kMaxSelectedParts][HEADS], s_acc[kWaves][HEADS][D];  // of the wavefronts; m, l of the parts
    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, c = lane % LR, tg = lane / LR;
    const int row = blockIdx.x / a.num_kv_heads, parts = a.parts, part = blockIdx.z;
    const Unit u(a, q_start, context_lens, row, blockIdx.x - row * a.num_kv_heads, blockIdx.y);
    if (!u.there) return;
    T *dst = out + (int64_t(row) * a.num_q_heads + u.head0) * D;
    if (u.pos < 0) {
        if (part == 0)
            for (int i = tid; i < HEADS * D; i += kThreads) dst[i] = T(0);
        return;
    }
    float x[HEADS][N], m[HEADS], l[HEADS], acc[HEADS][N];
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
        Vec<T>::get(*reinterpret_cast<const uint4 *>(q + (int64_t(row) * a.num_q_heads + u.head0 + h) * D + c * N), x[h]);
        m[h] = -FLT_MAX;
        l[h] = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[h][i] = 0.f;
    }
    const int32_t *list = selected + (int64_t(row) * a.num_kv_heads + u.kvh) * a.budget, *table = block_tables + int64_t(u.n) * a.max_blocks_per_seq;
    const int bs_log2 = a.block_size_log2, own = u.pos >> bs_log2, own_block = table[own];
    const int end = min(a.budget, (part + 1) * a.tiles_per_part);  // here a tile is a list entry
    bool any = false;
    for (int e0 = part * a.tiles_per_part; e0 < end; e0 += kWindow) {
        if (tid == 0) s_last = 0;
        __syncthreads();
        int last = 0;
        for (int i = tid; i < min(kWindow, end - e0); i += kThreads) {
            const int b = list[e0 + i];
            const bool there = b >= 0 && b <= own;
            s_entry[i] = int2{there ? table[b] : own_block, there ? min(u.pos + 1 - (b << bs_log2), 1 << bs_log2) : 0};
            if (there) last = i + 1;
        }
        if (last > 0) atomicMax(&s_last, last);
        __syncthreads();
        const int tokens = s_last << bs_log2;
        any |= tokens > 0;
        for (int t0 = wave * TOKENS * U; t0 < tokens; t0 += kWaves * TOKENS * U) {
            float kf[U][N], vf[U][N];
            bool counts[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int t = t0 + i * TOKENS + tg;
                const int2 e = s_entry[min(t, tokens - 1) >> bs_log2];
                const int slot = t & ((1 << bs_log2) - 1);
                counts[i] = t < tokens && slot < e.y;
                const int64_t at = (((int64_t(e.x) * a.num_kv_heads + u.kvh) << bs_log2) + (counts[i] ? slot : 0)) * D + c * N;
                Vec<T>::get(*reinterpret_cast<const uint4 *>(k_cache + at), kf[i]);
                Vec<T>::get(*reinterpret_cast<const uint4 *>(v_cache + at), vf[i]);
            }
#pragma unroll
            for (int i = 0; i < U; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) vf[i][j] = counts[i] ? vf[i][j] : 0.f;
#pragma unroll
            for (int h = 0; h < HEADS; ++h) {
                float s[U], top = m[h];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    float d = 0.f;
#pragma unroll
                    for (int j = 0; j < N; ++j) d = fmaf(x[h][j], kf[i][j], d);
                    s[i] = counts[i] ? sum_over_lanes<LR>(d) * a.scale : -INFINITY;
                    top = fmaxf(top, s[i]);
                }
                const float alpha = expf(m[h] - top);
                m[h] = top;
                l[h] *= alpha;
#pragma unroll
                for (int j = 0; j < N; ++j) acc[h][j] *= alpha;
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const float p = expf(s[i] - top);
                    l[h] += p;
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[h][j] = fmaf(p, vf[i][j], acc[h][j]);
                }
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {  // the lane groups of the wavefront
#pragma unroll
        for (int off = LR; off < 64; off <<= 1) {
            const float other = __shfl_xor(m[h], off), top = fmaxf(m[h], other), mine = expf(m[h] - top), theirs = expf(other - top);
            l[h] = l[h] * mine + __shfl_xor(l[h], off) * theirs;
#pragma unroll
            for (int i = 0; i < N; ++i) acc[h][i] = acc[h][i] * mine + __shfl_xor(acc[h][i], off) * theirs;
            m[h] = top;
        }
        if (tg == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) s_acc[wave][h][c * N + i] = acc[h][i];
            if (c == 0) {
                s_m[wave][h] = m[h];
                s_l[wave][h] = l[h];
            }
        }
    }
    __syncthreads();
    const int64_t unit = int64_t(blockIdx.x) * gridDim.y + blockIdx.y, slot0 = unit * parts;
    for (int f = tid; f < HEADS * D; f += kThreads) {
        const int h = f / D, d = f % D;
        float M = -FLT_MAX, L = 0.f, A = 0.f;
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][h]);
        for (int w = 0; w < kWaves; ++w) {
            const float wgt = expf(s_m[w][h] - M);
            L = fmaf(wgt, s_l[w][h], L);
            A = fmaf(wgt, s_acc[w][h][d], A);
        }
        if (parts == 1) {
            dst[f] = Vec<T>::out(any ? A / L : 0.f);
        } else {
            store_device(ws.acc + (slot0 + part) * (HEADS * D) + f, A);
            if (d == 0) {  // a part without a token says so
                store_device(ws.ml + ((slot0 + part) * HEADS + h) * 2, any ? M : -INFINITY);
                store_device(ws.ml + ((slot0 + part) * HEADS + h) * 2 + 1, L);
            }
        }
    }
    if (parts == 1) return;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");  // as above
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) s_last = __hip_atomic_fetch_add(ws.cnt + unit, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
    __syncthreads();
    if (!s_last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    if (tid == 0) __hip_atomic_store(ws.cnt + unit, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int i = tid; i < parts * HEADS; i += kThreads) {
        s_m[i / HEADS][i % HEADS] = load_device(ws.ml + (slot0 * HEADS + i) * 2);
        s_l[i / HEADS][i % HEADS] = load_device(ws.ml + (slot0 * HEADS + i) * 2 + 1);
    }
    __syncthreads();
    for (int f = tid; f < HEADS * D; f += kThreads) {
        const int h = f / D;
        float M = -INFINITY, L = 0.f, A = 0.f;
        for (int p = 0; p < parts; ++p) M = fmaxf(M, s_m[p][h]);
        constexpr int kBatch = 8;
        for (int p0 = 0; p0 < parts; p0 += kBatch) {
            float y[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) y[j] = load_device(ws.acc + (slot0 + min(p0 + j, parts - 1)) * (HEADS * D) + f);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                if (p0 + j >= parts) break;
                const float wgt = s_m[p0 + j][h] == -INFINITY ? 0.f : expf(s_m[p0 + j][h] - M);
                L = fmaf(wgt, s_l[p0 + j][h], L);
                A = fmaf(wgt, y[j], A);
            }
        }
        dst[f] = Vec<T>::out(M == -INFINITY ? 0.f : A / L);
    }
}

}  // namespace

hipError_t launch_attention_selected(const void *q, const void *k_cache, const void *v_cache, const int32_t *block_tables, const int32_t *context_lens,
                                     const int32_t *q_start, const int32_t *selected, void *out, Workspace ws, const SelectedArgs &a, int dtype,
                                     int head_dim, hipStream_t stream) {
    const unsigned chunks = unsigned((a.group + a.heads_per_chunk - 1) / a.heads_per_chunk);
    const dim3 grid(unsigned(a.total_q) * unsigned(a.num_kv_heads), chunks, unsigned(a.parts));
    if (a.on_mfma) {
        const auto *qp = static_cast<const uint16_t *>(q), *kp = static_cast<const uint16_t *>(k_cache), *vp = static_cast<const uint16_t *>(v_cache);
        auto *op = static_cast<uint16_t *>(out);
        const bool uniform = a.unit_log2 >= 4;
        if (a.wave_per_unit) {
            const dim3 waves(unsigned((a.total_q + kWaves - 1) / kWaves) * unsigned(a.num_kv_heads), chunks);
            auto launch = [&](auto kernel) { kernel<<<waves, dim3(kThreads), 0, stream>>>(qp, kp, vp, block_tables, context_lens, q_start, selected, op, a); };
            if (head_dim == 64) uniform ? launch(pa_selected_wave_kernel<64, true>) : launch(pa_selected_wave_kernel<64, false>);
            else uniform ? launch(pa_selected_wave_kernel<128, true>) : launch(pa_selected_wave_kernel<128, false>);
        } else {
            auto launch = [&](auto kernel) {
                kernel<<<grid, dim3(64 * a.waves), 0, stream>>>(qp, kp, vp, block_tables, context_lens, q_start, selected, op, ws, a);
            };
#define KVC_PARTS(HD, UNIFORM)                                                                                                     \
    do {                                                                                                                           \
        if (a.waves == 8) q_start ? launch(pa_selected_mfma_kernel<HD, UNIFORM, true, 8>) : launch(pa_selected_mfma_kernel<HD, UNIFORM, false, 8>); \
        else q_start ? launch(pa_selected_mfma_kernel<HD, UNIFORM, true, 4>) : launch(pa_selected_mfma_kernel<HD, UNIFORM, false, 4>); \
    } while (0)
            if (head_dim == 64) { if (uniform) KVC_PARTS(64, true); else KVC_PARTS(64, false); }
            else { if (uniform) KVC_PARTS(128, true); else KVC_PARTS(128, false); }
#undef KVC_PARTS
        }
        return hipGetLastError();
    }
    auto launch = [&](auto kernel, auto type) {
        using T = decltype(type);
        kernel<<<grid, dim3(kThreads), 0, stream>>>(static_cast<const T *>(q), static_cast<const T *>(k_cache), static_cast<const T *>(v_cache), block_tables,
                                                    context_lens, q_start, selected, static_cast<T *>(out), ws, a);
    };
#define KVC_SELECTED(T, D)                                                          \
    do {                                                                            \
        if (a.heads_per_chunk == 4) launch(pa_selected_valu_kernel<T, D, 4>, T());  \
        else if (a.heads_per_chunk == 2) launch(pa_selected_valu_kernel<T, D, 2>, T()); \
        else launch(pa_selected_valu_kernel<T, D, 1>, T());                         \
    } while (0)
    if (dtype == KVC_F32) {
        if (head_dim == 64) KVC_SELECTED(float, 64); else KVC_SELECTED(float, 128);
    } else {
        if (head_dim == 64) KVC_SELECTED(uint16_t, 64); else KVC_SELECTED(uint16_t, 128);
    }
#undef KVC_SELECTED
    return hipGetLastError();
}

}  // namespace kvc
