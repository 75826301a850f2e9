// Attention over the blocks that each query row keeps (gfx950):
//
//   out[row][h] = sum_t softmax_t(scale * q[row][h].K[t]) * V[t],  t <= position of the row, t in a block of selected[row][h / group]
//
// A list names blocks of the row's own sequence by their place in it, in any order; entries below 0 or past the row's own block are
// passed over.  One workgroup per (row, KV head, chunk of its heads); its wavefronts take the tiles of the list in turn and meet in LDS.
#include "cache_rows.h"
#include "kvc_internal.h"
#include "pa_partials.h"

namespace kvc {

namespace {

using namespace mfma;

constexpr int kWindow = 512;  // units whose places are held in LDS at a time

// ---- bf16 on the matrix cores, up to 16 heads of a KV head (blocks of 4 tokens and more)

// Weights as a sum of two bf16 values, see compute_tile of head_dim 64.
__device__ inline void split_weights(float p0, float p1, uint32_t *hi, uint32_t *lo) {
    const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
    *hi = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
    *lo = pack_bf16(__builtin_fmaf(p0, 1.f + FLT_EPSILON, -__uint_as_float(u0 & 0xffff0000u)),
                    __builtin_fmaf(p1, 1.f + FLT_EPSILON, -__uint_as_float(u1 & 0xffff0000u)));
}

// limit[h]: how many of this lane's tokens 16 h + 4 quad .. + 3 of the tile count.
__device__ inline void attend_tile(HeadStateN<8> &st, Shape<128>::Tile &t, const bf16x8 (&qb)[4], float scale_log2e, const int (&limit)[1]) {
    floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[j]), qb[j], s, 0, 0, 0);
    float sv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sv[i] = s[i] * scale_log2e;
    if (__builtin_amdgcn_ballot_w64(limit[0] < 4) != 0) {
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

__device__ inline void attend_tile(HeadStateN<4> &st, Shape<64>::Tile &t, const bf16x8 (&qb)[2], float scale_log2e, const int (&limit)[2]) {
    float sv[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 2; ++j) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[2 * h + j]), qb[j], s, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) sv[4 * h + i] = s[i] * scale_log2e;
    }
    if (__builtin_amdgcn_ballot_w64(limit[0] + limit[1] < 8) != 0) {
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
    int num_kv_heads, kvh, block_size_log2, unit_log2, units_per_block_log2, budget;
    __device__ int2 unit(int u) const {
        const int entry = u >> units_per_block_log2, in_block = u & ((1 << units_per_block_log2) - 1);
        const int b = entry < budget ? selected[entry] : -1;
        const bool there = b >= 0 && b <= pos >> block_size_log2;
        const int block = there ? table[b] : own_block;
        const int token = (b << block_size_log2) + (in_block << unit_log2);
        return int2{((block * num_kv_heads + kvh) << units_per_block_log2) + (there ? in_block : 0),
                    there ? min(max(pos + 1 - token, 0), 1 << unit_log2) : 0};
    }
};

template <int HD>
__global__ __launch_bounds__(kThreads, 2) void pa_selected_mfma_kernel(const uint16_t *__restrict__ q, const uint16_t *__restrict__ k_cache,
                                                                       const uint16_t *__restrict__ v_cache, const int32_t *__restrict__ block_tables,
                                                                       const int32_t *__restrict__ context_lens, const int32_t *__restrict__ q_start,
                                                                       const int32_t *__restrict__ selected, uint16_t *__restrict__ out, SelectedArgs a) {
    using TS = Shape<HD>;
    constexpr int kTokens = TS::kTokens, kSubs = kTokens / 16, NV = TS::kVecs;
    __shared__ int2 s_unit[kWindow];
    __shared__ int s_last;
    __shared__ float4 s_acc[kWaves][16 * HD / 4];
    __shared__ float2 s_ml[kWaves][16];
    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, quad = lane >> 4, r = lane & 15;
    const int kvh = blockIdx.x % a.num_kv_heads, row = blockIdx.x / a.num_kv_heads;
    const int head0 = kvh * a.group + blockIdx.y * a.heads_per_chunk, heads = min(a.heads_per_chunk, (kvh + 1) * a.group - head0);
    int n, pos;
    if (!find_row(row, q_start, context_lens, a.num_seqs, a.max_context_len, &n, &pos)) return;
    uint16_t *dst = out + (int64_t(row) * a.num_q_heads + head0) * HD;
    auto write_zeros = [&]() {
        for (int i = tid; i < heads * HD / 8; i += kThreads) reinterpret_cast<uint4 *>(dst)[i] = uint4{0u, 0u, 0u, 0u};
    };
    if (pos < 0) return write_zeros();
    bf16x8 qb[TS::kQ];
    load_q_operand(qb, q + (int64_t(row) * a.num_q_heads + head0 + (r < heads ? r : 0)) * HD, quad, r < heads);
    const int32_t *table = block_tables + int64_t(n) * a.max_blocks_per_seq;
    const ListOf list = {selected + (int64_t(row) * a.num_kv_heads + kvh) * a.budget, table, pos, table[pos >> a.block_size_log2],
                         a.num_kv_heads, kvh, a.block_size_log2, a.unit_log2, a.units_per_block_log2, a.budget};
    const int units_log2 = TS::kTokensLog2 - a.unit_log2, units = a.budget << a.units_per_block_log2;  // of a tile; of the list
    const int unit_tokens = 1 << a.unit_log2, k_off = (r & (unit_tokens - 1)) * HD + 8 * quad, v_off = ((4 * quad) & (unit_tokens - 1)) * HD + HD / 16 * r;
    const size_t unit_elems = size_t(unit_tokens) * HD;
    typename TS::State st;
    st.reset();
    bool any = false;
    for (int u0 = 0; u0 < units; u0 += kWindow) {
        if (tid == 0) s_last = 0;
        __syncthreads();
        int last = 0;
        for (int i = tid; i < kWindow; i += kThreads) {
            const int2 e = list.unit(u0 + i);
            s_unit[i] = e;
            if (e.y > 0) last = i + 1;
        }
        if (last > 0) atomicMax(&s_last, last);
        __syncthreads();
        const int tiles = (s_last + (1 << units_log2) - 1) >> units_log2;
        any |= tiles > 0;
        for (int it = wave; it < tiles; it += kWaves) {
            typename TS::Tile t;
            int limit[kSubs];
#pragma unroll
            for (int h = 0; h < kSubs; ++h) {
                const int2 *e = s_unit + (it << units_log2);
                const int kt = 16 * h + r, vt = 16 * h + 4 * quad;  // tokens of the tile
                const uint16_t *kp = k_cache + size_t(e[kt >> a.unit_log2].x) * unit_elems + k_off;
                const int2 ve = e[vt >> a.unit_log2];
                const uint16_t *vp = v_cache + size_t(ve.x) * unit_elems + v_off;
                limit[h] = min(max(ve.y - (vt & (unit_tokens - 1)), 0), 4);
                if constexpr (HD == 128) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) t.k[j] = load16_stream(kp + 32 * j);
#pragma unroll
                    for (int i = 0; i < 4; ++i) t.v[i] = load16_stream(vp + i * HD);
                } else {
                    const int in_unit = a.unit_log2 == 5 ? 16 * h * HD : 0;  // second half of a unit of 32 tokens
#pragma unroll
                    for (int j = 0; j < 2; ++j) t.k[2 * h + j] = load16_stream(kp + in_unit + 32 * j);
#pragma unroll
                    for (int i = 0; i < 4; ++i) t.v[4 * h + i] = load8_stream(vp + in_unit + i * HD);
                }
            }
            attend_tile(st, t, qb, a.scale_log2e, limit);
        }
        __syncthreads();
    }
    if (!any) return write_zeros();
    st.finish();
#pragma unroll
    for (int v = 0; v < NV; ++v) s_acc[wave][(v * 4 + quad) * 16 + r] = acc_vec(st, v);
    if (quad == 0) s_ml[wave][r] = float2{st.m, st.l};
    __syncthreads();
    for (int f = tid; f < heads * HD / 4; f += kThreads) {
        const int head = f / (HD / 4), d = f % (HD / 4);  // dims 4 d .. 4 d + 3
        const int vq = (d % NV) * 4 + d / NV;             // a quad holds HD / 4 dims, NV vectors
        float M = -INFINITY, L = 0.f;
        float4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_ml[w][head].x);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float2 ml = s_ml[w][head];
            const float wgt = __builtin_amdgcn_exp2f(ml.x - M);
            const float4 y = s_acc[w][vq * 16 + head];
            L = fmaf(wgt, ml.y, L);
            x.x = fmaf(wgt, y.x, x.x);
            x.y = fmaf(wgt, y.y, x.y);
            x.z = fmaf(wgt, y.z, x.z);
            x.w = fmaf(wgt, y.w, x.w);
        }
        const float inv = 1.0f / L;
        reinterpret_cast<uint2 *>(dst)[f] = uint2{pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv)};
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

template <class T, int D, int HEADS>
__global__ __launch_bounds__(kThreads) void pa_selected_valu_kernel(const T *__restrict__ q, const T *__restrict__ k_cache, const T *__restrict__ v_cache,
                                                                    const int32_t *__restrict__ block_tables, const int32_t *__restrict__ context_lens,
                                                                    const int32_t *__restrict__ q_start, const int32_t *__restrict__ selected,
                                                                    T *__restrict__ out, SelectedArgs a) {
    constexpr int N = Vec<T>::N, LR = D / N, TOKENS = 64 / LR, U = 4;
    __shared__ int2 s_entry[kWindow];  // pool index of a block, tokens of it that count
    __shared__ int s_last;
    __shared__ float s_m[kWaves][HEADS], s_l[kWaves][HEADS], s_acc[kWaves][HEADS][D];
    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, c = lane % LR, tg = lane / LR;
    const int kvh = blockIdx.x % a.num_kv_heads, row = blockIdx.x / a.num_kv_heads, head0 = kvh * a.group + blockIdx.y * HEADS;
    int n, pos;
    if (!find_row(row, q_start, context_lens, a.num_seqs, a.max_context_len, &n, &pos)) return;
    T *dst = out + (int64_t(row) * a.num_q_heads + head0) * D;
    if (pos < 0) {
        for (int i = tid; i < HEADS * D; i += kThreads) dst[i] = T(0);
        return;
    }
    float x[HEADS][N], m[HEADS], l[HEADS], acc[HEADS][N];
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
        Vec<T>::get(*reinterpret_cast<const uint4 *>(q + (int64_t(row) * a.num_q_heads + head0 + h) * D + c * N), x[h]);
        m[h] = -FLT_MAX;
        l[h] = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[h][i] = 0.f;
    }
    const int32_t *list = selected + (int64_t(row) * a.num_kv_heads + kvh) * a.budget, *table = block_tables + int64_t(n) * a.max_blocks_per_seq;
    const int bs_log2 = a.block_size_log2, own = pos >> bs_log2, own_block = table[own];
    bool any = false;
    for (int e0 = 0; e0 < a.budget; e0 += kWindow) {
        if (tid == 0) s_last = 0;
        __syncthreads();
        int last = 0;
        for (int i = tid; i < min(kWindow, a.budget - e0); i += kThreads) {
            const int b = list[e0 + i];
            const bool there = b >= 0 && b <= own;
            s_entry[i] = int2{there ? table[b] : own_block, there ? min(pos + 1 - (b << bs_log2), 1 << bs_log2) : 0};
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
            for (int u = 0; u < U; ++u) {
                const int t = t0 + u * TOKENS + tg;
                const int2 e = s_entry[min(t, tokens - 1) >> bs_log2];
                const int slot = t & ((1 << bs_log2) - 1);
                counts[u] = t < tokens && slot < e.y;
                const int64_t at = (((int64_t(e.x) * a.num_kv_heads + kvh) << bs_log2) + (counts[u] ? slot : 0)) * D + c * N;
                Vec<T>::get(*reinterpret_cast<const uint4 *>(k_cache + at), kf[u]);
                Vec<T>::get(*reinterpret_cast<const uint4 *>(v_cache + at), vf[u]);
#pragma unroll
                for (int i = 0; i < N; ++i) vf[u][i] = counts[u] ? vf[u][i] : 0.f;
            }
#pragma unroll
            for (int h = 0; h < HEADS; ++h) {
                float s[U], top = m[h];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float d = 0.f;
#pragma unroll
                    for (int i = 0; i < N; ++i) d = fmaf(x[h][i], kf[u][i], d);
#pragma unroll
                    for (int off = 1; off < LR; off <<= 1) d += __shfl_xor(d, off);
                    s[u] = counts[u] ? d * a.scale : -INFINITY;
                    top = fmaxf(top, s[u]);
                }
                const float alpha = expf(m[h] - top);
                m[h] = top;
                l[h] *= alpha;
#pragma unroll
                for (int i = 0; i < N; ++i) acc[h][i] *= alpha;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float p = expf(s[u] - top);
                    l[h] += p;
#pragma unroll
                    for (int i = 0; i < N; ++i) acc[h][i] = fmaf(p, vf[u][i], acc[h][i]);
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
    for (int f = tid; f < HEADS * D; f += kThreads) {
        const int h = f / D, d = f % D;
        float M = -FLT_MAX, L = 0.f, A = 0.f;
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][h]);
        for (int w = 0; w < kWaves; ++w) {
            const float wgt = expf(s_m[w][h] - M);
            L = fmaf(wgt, s_l[w][h], L);
            A = fmaf(wgt, s_acc[w][h][d], A);
        }
        dst[f] = Vec<T>::out(any ? A / L : 0.f);
    }
}

}  // namespace

hipError_t launch_attention_selected(const void *q, const void *k_cache, const void *v_cache, const int32_t *block_tables, const int32_t *context_lens,
                                     const int32_t *q_start, const int32_t *selected, void *out, SelectedArgs a, int total_q, int dtype,
                                     int head_dim, bool on_mfma, hipStream_t stream) {
    const unsigned pairs = unsigned(int64_t(total_q) * a.num_kv_heads);
    if (on_mfma) {
        const int tile_log2 = head_dim == 64 ? 5 : 4;
        a.unit_log2 = std::min(a.block_size_log2, tile_log2);
        a.units_per_block_log2 = a.block_size_log2 - a.unit_log2;
        const int chunks = (a.group + 15) / 16;
        a.heads_per_chunk = (a.group + chunks - 1) / chunks;
        auto launch = [&](auto kernel) {
            kernel<<<dim3(pairs, unsigned((a.group + a.heads_per_chunk - 1) / a.heads_per_chunk)), dim3(kThreads), 0, stream>>>(
                static_cast<const uint16_t *>(q), static_cast<const uint16_t *>(k_cache), static_cast<const uint16_t *>(v_cache), block_tables, context_lens,
                q_start, selected, static_cast<uint16_t *>(out), a);
        };
        if (head_dim == 64) launch(pa_selected_mfma_kernel<64>); else launch(pa_selected_mfma_kernel<128>);
        return hipGetLastError();
    }
    auto launch = [&](auto kernel, auto type, int heads) {
        using T = decltype(type);
        kernel<<<dim3(pairs, unsigned(a.group / heads)), dim3(kThreads), 0, stream>>>(static_cast<const T *>(q), static_cast<const T *>(k_cache),
                                                                                     static_cast<const T *>(v_cache), block_tables, context_lens, q_start,
                                                                                     selected, static_cast<T *>(out), a);
    };
#define KVC_SELECTED(T, D)                                                          \
    do {                                                                            \
        if (a.group % 4 == 0) launch(pa_selected_valu_kernel<T, D, 4>, T(), 4);     \
        else if (a.group % 2 == 0) launch(pa_selected_valu_kernel<T, D, 2>, T(), 2); \
        else launch(pa_selected_valu_kernel<T, D, 1>, T(), 1);                      \
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
