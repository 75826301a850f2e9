// kvc_key_bounds_update: per channel the smallest and the largest key of every block that a batch's new tokens filled (gfx950),
//
//   bounds[block][kv head][0][d] = min_s K[block][kv head][s][d],   bounds[..][1][d] = max_s K[..][s][d],   NaN if one is.
//
// Exact in the cache's type: both are values of it.  Bound by memory: K of the filled blocks is read once.  One wavefront per
// (block, KV head): D * e / 16 lanes cover a token's row, 64 / that tokens per load.  Six requests, 8 heads of 128 in bf16, 280 MB of K
// and bounds: 54.8 us = 5.1 TB/s (a copy of 2 GiB moves 5.0 TB/s here; loads that leave K in the caches 62.3 us); 96 requests, one token each, 4.4 us, the launch.
//
// How many tokens are new only the device knows, so a sequence has a bounded number of workgroups, which take its blocks in turn: one per
// block that the longest can fill would be mostly empty ones in a batch of decode steps with one long prompt (256 requests, one of 8192
// new tokens: 56.0 us so, 90.8 us with a workgroup per block; the 280 MB above were 64.7 and 65.5 us).
#include "kvc_internal.h"
#include "pa_lanes.h"

namespace kvc {

namespace {

template <class T>
struct Word;  // 16 bytes of T
template <>
struct Word<float> {
    static constexpr int N = 4;
    __device__ static void get(const uint4 &w, float (&x)[4]) {
        x[0] = __uint_as_float(w.x);
        x[1] = __uint_as_float(w.y);
        x[2] = __uint_as_float(w.z);
        x[3] = __uint_as_float(w.w);
    }
    __device__ static uint4 put(const float (&x)[4]) {
        return uint4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
};
template <>
struct Word<uint16_t> {
    static constexpr int N = 8;
    __device__ static void get(const uint4 &w, float (&x)[8]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
    __device__ static uint4 put(const float (&x)[8]) {  // values of T: the upper halves are all of them
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]), 0x07060302u);
        return uint4{u[0], u[1], u[2], u[3]};
    }
};

// NaN if either is.  (A NaN of bf16 stays one: its upper half has a bit of the fraction, and none is made here.)
__device__ inline float least(float a, float b) { return a < b || a != a ? a : b; }
__device__ inline float most(float a, float b) { return a > b || a != a ? a : b; }

__device__ inline uint4 once(const uint4 *p) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)));
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) void key_bounds_kernel(const T *__restrict__ k_cache, T *__restrict__ bounds, const int32_t *__restrict__ block_tables,
                                                              const int32_t *__restrict__ context_lens, const int32_t *__restrict__ q_start,
                                                              int groups_per_seq, int num_kv_heads, int block_size_log2, int max_blocks_per_seq,
                                                              int num_pool_blocks) {
    constexpr int N = Word<T>::N, LR = D / N, TOKENS = 64 / LR;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int h = blockIdx.y * kWaves + wave;
    if (h >= num_kv_heads) return;
    const int n = blockIdx.x / groups_per_seq, bs = 1 << block_size_log2;
    const int ctx = context_lens[n], fresh = q_start ? q_start[n + 1] - q_start[n] : 1;
    if (fresh <= 0 || ctx < bs) return;
    const int c = lane % LR, t0 = lane / LR, end = min(ctx >> block_size_log2, max_blocks_per_seq);
    const int32_t *table = block_tables + int64_t(n) * max_blocks_per_seq;
    int j = (max(ctx - fresh, 0) >> block_size_log2) + int(blockIdx.x - n * groups_per_seq);
    int next = j < end ? table[j] : -1;
    for (; j < end; j += groups_per_seq) {
        const int block = next;
        next = j + groups_per_seq < end ? table[j + groups_per_seq] : -1;
        if (block < 0 || block >= num_pool_blocks) continue;
        const int64_t at = int64_t(block) * num_kv_heads + h;
        const uint4 *src = reinterpret_cast<const uint4 *>(k_cache + (at << block_size_log2) * D);
        float lo[N], hi[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            lo[i] = INFINITY;
            hi[i] = -INFINITY;
        }
        constexpr int U = 4;
        for (int t = 0; t < bs; t += U * TOKENS) {
            uint4 w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) w[u] = once(src + min(t + u * TOKENS + t0, bs - 1) * LR + c);  // past the end: the last one again
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x[N];
                Word<T>::get(w[u], x);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    lo[i] = least(lo[i], x[i]);
                    hi[i] = most(hi[i], x[i]);
                }
            }
        }
#pragma unroll
        for (int off = LR; off < 64; off <<= 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                lo[i] = least(lo[i], __shfl_xor(lo[i], off));
                hi[i] = most(hi[i], __shfl_xor(hi[i], off));
            }
        }
        uint4 *dst = reinterpret_cast<uint4 *>(bounds + at * 2 * D);
        if (t0 == 0) dst[c] = Word<T>::put(lo);
        if (t0 == 1) dst[LR + c] = Word<T>::put(hi);
    }
}

}  // namespace

constexpr int64_t kMostBoundsGroups = 8192;  // of all sequences, for each four KV heads

hipError_t launch_key_bounds(const void *k_cache, void *bounds, const int32_t *block_tables, const int32_t *context_lens, const int32_t *q_start,
                             const kvc_attn_desc &d, int block_size_log2, int max_query_len, hipStream_t stream) {
    // blocks that `max_query_len` tokens can fill
    const int64_t blocks = std::min<int64_t>((int64_t(max_query_len) >> block_size_log2) + 1, d.max_blocks_per_seq);
    const int64_t groups = std::min<int64_t>(blocks, (kMostBoundsGroups + d.num_seqs - 1) / d.num_seqs);
    const int64_t heads = (d.num_kv_heads + kWaves - 1) / kWaves;
    constexpr int64_t kMostGroups = (int64_t(1) << 32) / kThreads - 1;
    const int64_t most = kMostGroups / (groups * heads);
    if (most == 0 || heads > 65535) return hipErrorInvalidValue;
    for (int64_t n = 0; n < d.num_seqs; n += most) {
        const int64_t seqs = d.num_seqs - n < most ? d.num_seqs - n : most;
        const dim3 grid(unsigned(seqs * groups), unsigned(heads));
        auto launch = [&](auto kernel, auto type) {
            using T = decltype(type);
            kernel<<<grid, dim3(kThreads), 0, stream>>>(static_cast<const T *>(k_cache), static_cast<T *>(bounds), block_tables + n * d.max_blocks_per_seq,
                                                        context_lens + n, q_start ? q_start + n : nullptr, int(groups), d.num_kv_heads, block_size_log2,
                                                        d.max_blocks_per_seq, d.num_pool_blocks);
        };
        if (d.dtype == KVC_F32) {
            if (d.head_dim == 64) launch(key_bounds_kernel<float, 64>, float()); else launch(key_bounds_kernel<float, 128>, float());
        } else {
            if (d.head_dim == 64) launch(key_bounds_kernel<uint16_t, 64>, uint16_t()); else launch(key_bounds_kernel<uint16_t, 128>, uint16_t());
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace kvc
