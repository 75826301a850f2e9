// kvc_block_select: the blocks of its sequence that a query keeps (gfx950).
//
//   score(b) = max over the heads h of a KV head's group of sum_d max(q_hd * lo_bd, q_hd * hi_bd)
//
// with lo, hi the smallest and largest key of block b per channel: no token of b has a product q.k above it.  A row that sees nb blocks keeps
// all of them if they are no more than the budget, else the first keep_first, the last keep_last and of the others those of largest score.
//
// Scores are in 64 bits, so that which of two nearly equal blocks is kept does not hang on the order of a sum.  Channel by channel
// max(q lo, q hi) = (q (hi + lo) + |q| (hi - lo)) / 2: two multiply-adds on numbers made once for all heads, and no comparison
// (twice the score is as good).  What is not finite in a block's bounds or in the query makes the sum so, and such a score ranks
// above all others: the block is kept, and what it holds shows in the attention.
//
// First launch: scores as keys whose order as whole numbers is that of the scores.  Second: per (row, KV head) the keys' rank by
// digits of 8 bits, and the kept blocks in ascending order.
#include "cache_rows.h"
#include "kvc_internal.h"
#include "pa_lanes.h"

namespace kvc {

namespace {

template <class T>
struct Load;  // 16 bytes of T as doubles
template <>
struct Load<float> {
    static constexpr int N = 4;
    __device__ static void get(const uint4 &w, double (&x)[4]) {
        x[0] = __uint_as_float(w.x);
        x[1] = __uint_as_float(w.y);
        x[2] = __uint_as_float(w.z);
        x[3] = __uint_as_float(w.w);
    }
};
template <>
struct Load<uint16_t> {
    static constexpr int N = 8;
    __device__ static void get(const uint4 &w, double (&x)[8]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
};

__device__ inline uint64_t key_of(double s) {
    if (!__builtin_isfinite(s)) return ~uint64_t(0);
    const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);  // -0 is 0
    return u >> 63 ? ~u : u | uint64_t(1) << 63;
}

// A wavefront scores 64 / LR blocks at a time, LR lanes each; blockIdx.x = row * KV heads + KV head, blockIdx.y = share of the blocks.
template <class T, int D, int HEADS>
__global__ __launch_bounds__(kThreads) void block_scores_kernel(const T *__restrict__ q, const T *__restrict__ bounds, const int32_t *__restrict__ block_tables,
                                                                const int32_t *__restrict__ context_lens, const int32_t *__restrict__ q_start,
                                                                uint64_t *__restrict__ keys, SelectArgs a, int blocks_per_group) {
    constexpr int N = Load<T>::N, LR = D / N, TOGETHER = 64 / LR;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int row = blockIdx.x / a.num_kv_heads, kvh = blockIdx.x - row * a.num_kv_heads;
    int n, pos;
    if (!find_row(row, q_start, context_lens, a.num_seqs, a.max_context_len, &n, &pos) || pos < 0) return;
    const int nb = (pos >> a.block_size_log2) + 1;
    if (nb <= a.budget) return;
    const int first = a.keep_first + blockIdx.y * blocks_per_group, last = min(nb - a.keep_last, first + blocks_per_group);
    const int c = lane % LR, mine = lane / LR;
    const int32_t *table = block_tables + int64_t(n) * a.max_blocks_per_seq;
    uint64_t *out = keys + int64_t(blockIdx.x) * a.max_blocks;
    for (int h0 = 0; h0 < a.group; h0 += HEADS) {
        double x[HEADS][N];
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {  // heads past the group: the last one again
            const int64_t head = int64_t(row) * a.num_q_heads + kvh * a.group + min(h0 + h, a.group - 1);
            Load<T>::get(*reinterpret_cast<const uint4 *>(q + head * D + c * N), x[h]);
        }
        for (int b0 = first + wave * TOGETHER; b0 < last; b0 += kWaves * TOGETHER) {
            const int b = b0 + mine;
            const T *src = bounds + (int64_t(table[min(b, last - 1)]) * a.num_kv_heads + kvh) * 2 * D + c * N;
            double lo[N], hi[N], s[HEADS];
            Load<T>::get(*reinterpret_cast<const uint4 *>(src), lo);
            Load<T>::get(*reinterpret_cast<const uint4 *>(src + D), hi);
#pragma unroll
            for (int h = 0; h < HEADS; ++h) s[h] = 0.0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const double sum = hi[i] + lo[i], width = hi[i] - lo[i];
#pragma unroll
                for (int h = 0; h < HEADS; ++h) s[h] = fma(x[h][i], sum, fma(fabs(x[h][i]), width, s[h]));
            }
            uint64_t best = 0;
#pragma unroll
            for (int h = 0; h < HEADS; ++h) {
#pragma unroll
                for (int off = 1; off < LR; off <<= 1) s[h] += __shfl_xor(s[h], off);
                const uint64_t key = key_of(s[h]);
                best = key > best ? key : best;
            }
            if (c == 0 && b < last) {
                if (h0 > 0) {
                    const uint64_t before = out[b];
                    best = before > best ? before : best;
                }
                out[b] = best;
            }
        }
    }
}

__global__ __launch_bounds__(kThreads) void block_choose_kernel(const uint64_t *__restrict__ keys, const int32_t *__restrict__ context_lens,
                                                                const int32_t *__restrict__ q_start, int32_t *__restrict__ selected, SelectArgs a) {
    __shared__ uint32_t s_count[256], s_sums[kWaves], s_digit[2], s_before[2][kWaves];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int row = blockIdx.x / a.num_kv_heads;
    int n, pos;
    if (!find_row(row, q_start, context_lens, a.num_seqs, a.max_context_len, &n, &pos)) return;
    int32_t *out = selected + int64_t(blockIdx.x) * a.budget;
    const int nb = pos < 0 ? 0 : (pos >> a.block_size_log2) + 1;
    if (nb <= a.budget) {
        for (int i = tid; i < a.budget; i += kThreads) out[i] = i < nb ? i : -1;
        return;
    }
    keys += int64_t(blockIdx.x) * a.max_blocks;
    const int lo = a.keep_first, hi = nb - a.keep_last;  // lo <= b < hi compete
    // prefix, mask: the digits of the smallest key kept; left: keys to keep among those that agree in them
    uint64_t prefix = 0, mask = 0;
    uint32_t left = a.budget - a.keep_first - a.keep_last;
    const bool scored = left > 0;
    for (int shift = 56; scored && shift >= 0; shift -= 8) {
        s_count[tid] = 0;
        __syncthreads();
        for (int b = lo + tid; b < hi; b += kThreads) {
            const uint64_t key = keys[b];
            if ((key & mask) == prefix) atomicAdd(&s_count[255 - (uint32_t(key >> shift) & 255)], 1u);
        }
        __syncthreads();
        const uint32_t count = s_count[tid], incl = uint32_t(lanes::prefix_sum(int(count)));
        if (lane == 63) s_sums[wave] = incl;
        __syncthreads();
        uint32_t upto = incl;
        for (int w = 0; w < wave; ++w) upto += s_sums[w];
        if (upto >= left && upto - count < left) {  // one thread
            s_digit[0] = tid;
            s_digit[1] = upto - count;
        }
        __syncthreads();
        const uint32_t at = s_digit[0];
        left -= s_digit[1];
        prefix |= uint64_t(255 - at) << shift;
        mask |= uint64_t(255) << shift;
        const uint32_t here = s_count[at];
        __syncthreads();
        if (here == left) break;  // all that agree so far are kept
    }
    // Kept: what is above the prefix, and of what agrees with it the first `left`.  A wavefront takes consecutive blocks.
    const int share = (nb + kThreads - 1) / kThreads * 64, from = wave * share, to = min(from + share, nb);
    auto sort = [&](int b, bool *above, bool *equal) {
        *above = *equal = false;
        if (b >= to) return;
        if (b < lo || b >= hi) {
            *above = true;
            return;
        }
        if (!scored) return;
        const uint64_t key = keys[b] & mask;
        *above = key > prefix;
        *equal = key == prefix;
    };
    uint32_t above = 0, equal = 0;
    for (int b = from + lane; b - lane < to; b += 64) {
        bool x, y;
        sort(b, &x, &y);
        above += __popcll(__ballot(x));
        equal += __popcll(__ballot(y));
    }
    if (lane == 0) {
        s_before[0][wave] = above;
        s_before[1][wave] = equal;
    }
    __syncthreads();
    above = equal = 0;
    for (int w = 0; w < wave; ++w) {
        above += s_before[0][w];
        equal += s_before[1][w];
    }
    const uint64_t below = (uint64_t(1) << lane) - 1;
    for (int b = from + lane; b - lane < to; b += 64) {
        bool x, y;
        sort(b, &x, &y);
        const uint64_t xs = __ballot(x), ys = __ballot(y);
        const uint32_t above_me = above + __popcll(xs & below), equal_me = equal + __popcll(ys & below);
        if (x || (y && equal_me < left)) out[above_me + min(equal_me, left)] = b;
        above += __popcll(xs);
        equal += __popcll(ys);
    }
}

}  // namespace

hipError_t launch_block_select(const void *q, const void *bounds, const int32_t *block_tables, const int32_t *context_lens, const int32_t *q_start,
                               int32_t *selected, uint64_t *keys, const SelectArgs &a, int total_q, int dtype, int head_dim, hipStream_t stream) {
    const int64_t pairs = int64_t(total_q) * a.num_kv_heads;
    const int compete = a.max_blocks - a.keep_first - a.keep_last;
    if (a.max_blocks > a.budget && a.budget > a.keep_first + a.keep_last) {
        const int together = kWaves * 64 / (head_dim * (dtype == KVC_F32 ? 4 : 2) / 16);
        int64_t shares = std::min<int64_t>((compete + together - 1) / together, std::max<int64_t>(1, 8 * kNumCUs / pairs));
        const int per_group = int(((compete + shares - 1) / shares + together - 1) / together * together);
        shares = (compete + per_group - 1) / per_group;
        const dim3 grid{unsigned(pairs), unsigned(shares)};
        auto launch = [&](auto kernel, auto type) {
            using T = decltype(type);
            kernel<<<grid, dim3(kThreads), 0, stream>>>(static_cast<const T *>(q), static_cast<const T *>(bounds), block_tables, context_lens, q_start, keys, a,
                                                        per_group);
        };
#define KVC_SCORES(T, D)                                                                    \
    do {                                                                                    \
        if (a.group >= 5) launch(block_scores_kernel<T, D, 8>, T());                        \
        else if (a.group >= 3) launch(block_scores_kernel<T, D, 4>, T());                   \
        else if (a.group == 2) launch(block_scores_kernel<T, D, 2>, T());                   \
        else launch(block_scores_kernel<T, D, 1>, T());                                     \
    } while (0)
        if (dtype == KVC_F32) {
            if (head_dim == 64) KVC_SCORES(float, 64); else KVC_SCORES(float, 128);
        } else {
            if (head_dim == 64) KVC_SCORES(uint16_t, 64); else KVC_SCORES(uint16_t, 128);
        }
#undef KVC_SCORES
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    block_choose_kernel<<<dim3(unsigned(pairs)), dim3(kThreads), 0, stream>>>(keys, context_lens, q_start, selected, a);
    return hipGetLastError();
}

}  // namespace kvc
