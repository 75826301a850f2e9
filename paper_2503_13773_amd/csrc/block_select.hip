// kvc_block_select: the blocks of its sequence that a query keeps (gfx950).
//
//   score(b) = max over the heads h of a KV head's group of sum_d max(q_hd * lo_bd, q_hd * hi_bd)
//
// with lo, hi the smallest and largest key of block b per channel: no token of b has a product q.k above it.  A row that sees nb blocks keeps
// all of them if they are no more than the budget, else the first keep_first, the last keep_last and of the others those of largest score.
// Scores count in 64 bits, so that which of two nearly equal blocks is kept does not hang on the order of a sum.  What is not finite in a
// block's bounds or in the query makes the score so, and such a score ranks above all others: the block is kept, and what it holds shows
// in the attention.
//
// All scores in 64 bits are bound by the vector ALUs (32 long documents, 64 / 8 heads of 128: 116 us; 1000 rows of chunks, 16 / 4 heads
// of 64 in fp32: 166 us).  So the first launch takes them from the matrix cores, as
//
//   sum_d q+_d hi_d + q-_d lo_d,  q+ = max(q, 0), q- = min(q, 0)      (exact in the type of q)
//
// with fp32 sums, and beside them a bound on what these can be off: error <= kSlack * sum_d |q_d| max(|lo_d|, |hi_d|), the largest of a row
// E.  The second launch finds where the last kept score lies, T: blocks more than 2 E above T are kept and ones more than 2 E below are
// not, whatever the true scores are (the true last score is within E of T, each true score within E of its own).  Only the few in between are
// scored in 64 bits and ranked.  Rows where that settles too little (many equal scores, something not finite) are scored in 64 bits
// throughout.
#include <type_traits>

#include "cache_rows.h"
#include "kvc_internal.h"
#include "pa_mfma_tile.h"

namespace kvc {

namespace {

using mfma::bf16x8;
using mfma::floatx4;
using mfma::pack_bf16;

__device__ inline float first_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float second_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

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
            x[2 * i] = first_of(u[i]);
            x[2 * i + 1] = second_of(u[i]);
        }
    }
};

// ---- scores from the matrix cores

// An operand: 8 numbers of a lane.  bf16 as they are; fp32 as the sum of two bf16 values (2^-17 relative).
template <class T>
struct Operand;
template <>
struct Operand<uint16_t> {
    uint4 w;
    __device__ void load(const uint16_t *p) { w = *reinterpret_cast<const uint4 *>(p); }
    __device__ static uint32_t negative(uint32_t x) { return ((x >> 15) & 0x10001u) * 0xffffu; }
    __device__ Operand plus() const { return {uint4{w.x & ~negative(w.x), w.y & ~negative(w.y), w.z & ~negative(w.z), w.w & ~negative(w.w)}}; }
    __device__ Operand minus() const { return {uint4{w.x & negative(w.x), w.y & negative(w.y), w.z & negative(w.z), w.w & negative(w.w)}}; }
    // the larger size of two, number by number
    __device__ static bf16x8 sizes(const Operand &a, const Operand &b) {
        auto larger = [](uint32_t x, uint32_t y) {
            typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
            return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x & 0x7fff7fffu), __builtin_bit_cast(u16x2, y & 0x7fff7fffu)));
        };
        return __builtin_bit_cast(bf16x8, uint4{larger(a.w.x, b.w.x), larger(a.w.y, b.w.y), larger(a.w.z, b.w.z), larger(a.w.w, b.w.w)});
    }
    __device__ bf16x8 top() const { return __builtin_bit_cast(bf16x8, w); }
    __device__ static floatx4 multiply(const Operand &a, const Operand &b, floatx4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.top(), b.top(), c, 0, 0, 0);
    }
};
template <>
struct Operand<float> {
    float x[8];
    bf16x8 hi, lo;
    __device__ void load(const float *p) {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    __device__ void split() {
        uint32_t h[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
            l[i] = pack_bf16(x[2 * i] - first_of(h[i]), x[2 * i + 1] - second_of(h[i]));
        }
        hi = __builtin_bit_cast(bf16x8, uint4{h[0], h[1], h[2], h[3]});
        lo = __builtin_bit_cast(bf16x8, uint4{l[0], l[1], l[2], l[3]});
    }
    __device__ Operand plus() const {
        Operand o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.x[i] = x[i] < 0.f ? 0.f : x[i];  // NaN stays
        o.split();
        return o;
    }
    __device__ Operand minus() const {
        Operand o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.x[i] = x[i] < 0.f ? x[i] : 0.f;
        o.split();
        return o;
    }
    __device__ static bf16x8 sizes(const Operand &a, const Operand &b) {
        uint32_t s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            s[i] = pack_bf16(fmaxf(fabsf(a.x[2 * i]), fabsf(b.x[2 * i])), fmaxf(fabsf(a.x[2 * i + 1]), fabsf(b.x[2 * i + 1])));
        return __builtin_bit_cast(bf16x8, uint4{s[0], s[1], s[2], s[3]});
    }
    __device__ bf16x8 top() const { return hi; }
    __device__ static floatx4 multiply(const Operand &a, const Operand &b, floatx4 c) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.lo, b.hi, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.hi, b.lo, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.hi, b.hi, c, 0, 0, 0);
    }
};

// Error of a score over sum_d |q_d| max(|lo_d|, |hi_d|): the sums have 2 D products (fp32: three times that), each step loses at most 2^-23
// of what there is, counted twice; fp32 numbers are cut to 2^-17 each and the product of their lower parts (2^-18) is left out.
// The sum of sizes is itself computed in fp32 and, for fp32 numbers, from values rounded to 8 bits: within 2 % of what it stands for.
template <class T, int D>
constexpr float kSlack = 1.02f * (sizeof(T) == 2 ? (2 * D + 16) / 4194304.f : (6 * D + 16) / 4194304.f + 1.f / 32768.f);

__device__ inline float max_of(float a, float b) { return a != a || a > b ? a : b; }  // NaN stays

// Columns of a product are heads of rows of q: `heads` of them (a power of two, the group's last head again in place of what it lacks)
// times 16 / heads rows; GROUPS such sets of rows share the loads.  Rows of products are 16 blocks.  blockIdx.x = KV head + KV heads * tile of
// rows (tile_rows: one of a decode step, as many as there are columns for of chunks), blockIdx.y = share of the blocks.  Writes the scores of all rows of the tile, and per row and share the largest sum of sizes.
template <class T, int D, int GROUPS>
__global__ __launch_bounds__(kThreads) void block_scores_kernel(const T *__restrict__ q, const T *__restrict__ bounds, const int32_t *__restrict__ block_tables,
                                                                const int32_t *__restrict__ context_lens, const int32_t *__restrict__ q_start,
                                                                float *__restrict__ scores, float *__restrict__ sizes, SelectArgs a, int tile_rows) {
    constexpr int J = D / 32;
    using Op = Operand<T>;
    __shared__ float s_size[kWaves][GROUPS][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, quad = lane >> 4, r = lane & 15;
    const int tile = blockIdx.x / a.num_kv_heads, kvh = blockIdx.x - tile * a.num_kv_heads;
    const int set_rows = 16 >> a.heads_log2, my_row = r >> a.heads_log2, my_head = r & ((1 << a.heads_log2) - 1);
    const int tile_end = min(a.total_q, (tile + 1) * tile_rows);
    for (int row0 = tile * tile_rows, row1; row0 < tile_end; row0 = row1) {  // one sequence at a time
        int n, pos;
        row1 = row0 + 1;
        if (!find_row(row0, q_start, context_lens, a.num_seqs, a.max_context_len, &n, &pos)) continue;
        if (q_start) row1 = min(tile_end, q_start[n + 1]);
        pos = min(pos + (row1 - 1 - row0), a.max_context_len - 1);  // of the last row, which sees the most blocks
        const int nb = pos < 0 ? 0 : (pos >> a.block_size_log2) + 1;
        if (nb <= a.budget) continue;
        const int first = a.keep_first + blockIdx.y * a.share, last = min(nb - a.keep_last, first + a.share);
        const int32_t *table = block_tables + int64_t(n) * a.max_blocks_per_seq;
        float size[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) size[g] = 0.f;
        for (int h0 = 0; h0 < a.group; h0 += 16) {  // more than 16 heads: one set of 16 after the other
            Op plus[GROUPS][J], minus[GROUPS][J];
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const int64_t row = min(row0 + g * set_rows + my_row, row1 - 1);
                const T *src = q + (row * a.num_q_heads + kvh * a.group + min(h0 + my_head, a.group - 1)) * D + 8 * quad;
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    Op x;
                    x.load(src + 32 * j);
                    plus[g][j] = x.plus();
                    minus[g][j] = x.minus();
                }
            }
            int b0 = first + 16 * wave;
            int block = b0 < last ? table[min(b0 + r, last - 1)] : 0;
            for (; b0 < last; b0 += 16 * kWaves) {
                const T *src = bounds + (int64_t(block) * a.num_kv_heads + kvh) * 2 * D + 8 * quad;
                Op lo[J], hi[J];
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    lo[j].load(src + 32 * j);
                    hi[j].load(src + D + 32 * j);
                }
                block = table[min(b0 + 16 * kWaves + r, last - 1)];
                floatx4 s[GROUPS], up[GROUPS], down[GROUPS];
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) s[g] = up[g] = down[g] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const bf16x8 most = Op::sizes(lo[j], hi[j]);
                    if constexpr (sizeof(T) == 4) {
                        lo[j].split();
                        hi[j].split();
                    }
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) {
                        s[g] = Op::multiply(hi[j], plus[g][j], s[g]);
                        s[g] = Op::multiply(lo[j], minus[g][j], s[g]);
                        up[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(most, plus[g][j].top(), up[g], 0, 0, 0);
                        down[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(most, minus[g][j].top(), down[g], 0, 0, 0);
                    }
                }
                // lane (quad, r) holds blocks b0 + 4 quad + i of column r
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) size[g] = max_of(size[g], up[g][i] - down[g][i]);
                    floatx4 best = s[g];
                    for (int off = 1; off < 1 << a.heads_log2; off <<= 1) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) best[i] = max_of(best[i], __shfl_xor(best[i], off));
                    }
                    const int row = row0 + g * set_rows + my_row;
                    if (my_head == 0 && row < row1) {
                        float *dst = scores + (int64_t(row) * a.num_kv_heads + kvh) * a.stride + b0 - a.keep_first + 4 * quad;
                        if (h0 > 0) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) best[i] = max_of(dst[i], best[i]);
                        }
                        *reinterpret_cast<floatx4 *>(dst) = best;  // rows of `stride` have room for whole sets of blocks
                    }
                }
            }
        }
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
#pragma unroll
            for (int off = 16; off < 64; off <<= 1) size[g] = max_of(size[g], __shfl_xor(size[g], off));
            for (int off = 1; off < 1 << a.heads_log2; off <<= 1) size[g] = max_of(size[g], __shfl_xor(size[g], off));
            if (quad == 0) s_size[wave][g][r] = size[g];
        }
        __syncthreads();
        if (threadIdx.x < 16 * GROUPS) {
            const int g = threadIdx.x >> 4, row = row0 + g * set_rows + my_row;
            float x = s_size[0][g][r];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) x = max_of(x, s_size[w][g][r]);
            if (my_head == 0 && row < row1) sizes[(int64_t(row) * a.num_kv_heads + kvh) * gridDim.y + blockIdx.y] = x;
        }
        __syncthreads();
    }
}

// ---- the choice

// Order of numbers as order of whole numbers.
__device__ inline uint32_t key_of(float s) {
    const uint32_t u = __float_as_uint(s + 0.f);  // -0 is 0
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ inline float score_of(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }
__device__ inline uint64_t key_of(double s) {
    if (!__builtin_isfinite(s)) return ~uint64_t(0);
    const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
    return u >> 63 ? ~u : u | uint64_t(1) << 63;
}

// Scores in 64 bits of the blocks place(0) .. place(count - 1) of a row, given to put(i, key).  Channel by channel
// max(q lo, q hi) = (q (hi + lo) + |q| (hi - lo)) / 2, and twice the score is as good.
template <class T, int D, class Place, class Put>
__device__ inline void score_exactly(const T *q_heads, const T *bounds, const int32_t *table, int kvh, const SelectArgs &a, int count, Place place, Put put) {
    constexpr int N = Load<T>::N, LR = D / N, TOGETHER = 64 / LR;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane % LR;
    for (int i0 = wave * TOGETHER; i0 < count; i0 += kWaves * TOGETHER) {
        const int i = i0 + lane / LR;
        const T *src = bounds + (int64_t(table[place(min(i, count - 1))]) * a.num_kv_heads + kvh) * 2 * D + c * N;
        double sum[N], width[N];
        Load<T>::get(*reinterpret_cast<const uint4 *>(src), sum);
        Load<T>::get(*reinterpret_cast<const uint4 *>(src + D), width);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const double lo = sum[k], hi = width[k];
            sum[k] = hi + lo;
            width[k] = hi - lo;
        }
        uint64_t best = 0;
#pragma unroll 1
        for (int h = 0; h < a.group; ++h) {
            double x[N], s = 0.0;
            Load<T>::get(*reinterpret_cast<const uint4 *>(q_heads + int64_t(h) * D + c * N), x);
#pragma unroll
            for (int k = 0; k < N; ++k) s = fma(x[k], sum[k], fma(fabs(x[k]), width[k], s));
#pragma unroll
            for (int off = 1; off < LR; off <<= 1) s += __shfl_xor(s, off);
            const uint64_t key = key_of(s);
            best = key > best ? key : best;
        }
        if (c == 0 && i < count) put(i, best);
    }
}

// What a workgroup shares while it chooses for one (row, KV head).
constexpr int kBand = 512;  // blocks that it ranks by comparing each with each
struct Choice {
    uint32_t count[256], sums[kWaves], digit[2], before[2][kWaves], sure, band;
    float size;
    int wide;
    uint64_t keys[kBand];
    int places[kBand];
};

// Digit of the key at which the `left` largest of those counted in s.count end (slot 255 - digit): s.digit = slot, and how many lie above.
__device__ inline void find_digit(Choice &s, uint32_t left) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const uint32_t count = s.count[tid], incl = uint32_t(lanes::prefix_sum(int(count)));
    if (lane == 63) s.sums[wave] = incl;
    __syncthreads();
    uint32_t upto = incl;
    for (int w = 0; w < wave; ++w) upto += s.sums[w];
    if (upto >= left && upto - count < left) {  // one thread
        s.digit[0] = tid;
        s.digit[1] = upto - count;
    }
    __syncthreads();
}

// Writes, in ascending order, the blocks below nb that are kept: what(b) = 2 kept, 1 kept if among the first `left` of these, 0 not.
template <class What>
__device__ inline void write_kept(Choice &s, int nb, uint32_t left, int32_t *out, What what) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    // a wavefront takes consecutive blocks
    const int share = (nb + kThreads - 1) / kThreads * 64, from = wave * share, to = min(from + share, nb);
    uint32_t above = 0, equal = 0;
    for (int b = from + lane; b - lane < to; b += 64) {
        const int x = b < to ? what(b) : 0;
        above += __popcll(__ballot(x == 2));
        equal += __popcll(__ballot(x == 1));
    }
    if (lane == 0) {
        s.before[0][wave] = above;
        s.before[1][wave] = equal;
    }
    __syncthreads();
    above = equal = 0;
    for (int w = 0; w < wave; ++w) {
        above += s.before[0][w];
        equal += s.before[1][w];
    }
    const uint64_t below = (uint64_t(1) << lane) - 1;
    for (int b = from + lane; b - lane < to; b += 64) {
        const int x = b < to ? what(b) : 0;
        const uint64_t xs = __ballot(x == 2), ys = __ballot(x == 1);
        const uint32_t above_me = above + __popcll(xs & below), equal_me = equal + __popcll(ys & below);
        if (x == 2 || (x == 1 && equal_me < left)) out[above_me + min(equal_me, left)] = b;
        above += __popcll(xs);
        equal += __popcll(ys);
    }
}

// CAPACITY: scores that fit in LDS; rows with more competing blocks are scored in 64 bits throughout.
template <class T, int D, int CAPACITY>
__global__ __launch_bounds__(kThreads) void block_choose_kernel(const T *__restrict__ q, const T *__restrict__ bounds, const int32_t *__restrict__ block_tables,
                                                                const int32_t *__restrict__ context_lens, const int32_t *__restrict__ q_start,
                                                                const float *__restrict__ scores, const float *__restrict__ sizes, int shares,
                                                                uint64_t *__restrict__ all_keys, int32_t *__restrict__ selected, SelectArgs a) {
    __shared__ Choice s;
    __shared__ uint32_t s_keys[CAPACITY];
    const int tid = threadIdx.x, lane = tid & 63;
    const int row = blockIdx.x / a.num_kv_heads, kvh = blockIdx.x - row * a.num_kv_heads;
    int n, pos;
    if (!find_row(row, q_start, context_lens, a.num_seqs, a.max_context_len, &n, &pos)) return;
    int32_t *out = selected + int64_t(blockIdx.x) * a.budget;
    const int nb = pos < 0 ? 0 : (pos >> a.block_size_log2) + 1;
    if (nb <= a.budget) {
        for (int i = tid; i < a.budget; i += kThreads) out[i] = i < nb ? i : -1;
        return;
    }
    const int lo = a.keep_first, compete = nb - a.keep_last - a.keep_first;  // blocks lo .. lo + compete - 1 compete
    const uint32_t places = a.budget - a.keep_first - a.keep_last;           // for so many places: fewer than compete
    if (places == 0) {
        write_kept(s, nb, 0, out, [&](int b) { return b < lo || b >= lo + compete ? 2 : 0; });
        return;
    }
    const int32_t *table = block_tables + int64_t(n) * a.max_blocks_per_seq;
    const T *q_heads = q + (int64_t(row) * a.num_q_heads + kvh * a.group) * D;

    // ---- by the scores of the matrix cores
    bool settled = false;
    float bottom = 0.f, top = 0.f;  // scores above top are kept, ones below bottom are not
    uint32_t left = 0;              // places for those between
    if (compete <= CAPACITY) {
        if (tid == 0) {
            s.sure = s.band = 0;
            s.wide = 0;
        }
        float size = 0.f;
        for (int i = tid; i < shares; i += kThreads) {
            if (i * a.share >= compete) break;  // shares behind have not been written
            size = max_of(size, sizes[int64_t(blockIdx.x) * shares + i]);
        }
        const float *mine = scores + int64_t(blockIdx.x) * a.stride;
        uint32_t least = ~0u, most = 0;
        bool finite = true;
        for (int i = tid; i < compete; i += kThreads) {
            const float x = mine[i];
            finite &= __builtin_isfinite(x);
            const uint32_t key = key_of(x);
            s_keys[i] = key;
            least = min(least, key);
            most = max(most, key);
        }
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            size = max_of(size, __shfl_xor(size, off));
            least = min(least, uint32_t(__shfl_xor(int(least), off)));
            most = max(most, uint32_t(__shfl_xor(int(most), off)));
        }
        finite = __ballot(!finite) == 0;
        const int wave = tid >> 6;
        if (lane == 0) {
            s.count[wave] = least;
            s.count[4 + wave] = most;
            s.count[8 + wave] = __float_as_uint(finite ? size : INFINITY);
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            least = min(least, s.count[w]);
            most = max(most, s.count[4 + w]);
            const float other = __uint_as_float(s.count[8 + w]);
            size = w == 0 ? other : max_of(size, other);
        }
        __syncthreads();
        const float slack = kSlack<T, D> * size + 1e-30f;
        if (__builtin_isfinite(size) && size < 1e30f) {
            // the smallest kept key, to where what is left of its digits spans less than the slack
            int bits = most == least ? 0 : 32 - __builtin_clz(most ^ least);  // that differ
            uint32_t prefix = bits < 32 ? least >> bits << bits : 0, mask = bits < 32 ? ~0u << bits : 0;
            left = places;
            while (bits > 0) {
                const int shift = max(bits - 8, 0);
                s.count[tid] = 0;
                __syncthreads();
                for (int i = tid; i < compete; i += kThreads) {
                    const uint32_t key = s_keys[i];
                    if ((key & mask) == prefix) atomicAdd(&s.count[255 - ((key >> shift) & ((1u << (bits - shift)) - 1))], 1u);
                }
                __syncthreads();
                find_digit(s, left);
                left -= s.digit[1];
                prefix |= (255 - s.digit[0]) << shift;
                mask |= ((1u << (bits - shift)) - 1) << shift;
                bits = shift;
                __syncthreads();
                if (score_of(prefix | ~mask) - score_of(prefix) <= slack) break;
            }
            bottom = score_of(prefix) - 2.f * slack;
            top = score_of(prefix | ~mask) + 2.f * slack;
            // those between
            for (int i0 = 0; i0 < compete; i0 += kThreads) {
                const int i = i0 + tid;
                const float x = i < compete ? score_of(s_keys[i]) : -INFINITY;
                const uint64_t sure = __ballot(x > top);
                if (lane == 0 && sure) atomicAdd(&s.sure, uint32_t(__popcll(sure)));
                if (x >= bottom && x <= top && i < compete) {
                    const uint32_t at = atomicAdd(&s.band, 1u);
                    if (at < kBand) s.places[at] = lo + i;
                }
            }
            __syncthreads();
            left = places - s.sure;
            const int between = int(s.band);
            settled = between <= kBand;
            if (settled && uint32_t(between) != left) {
                score_exactly<T, D>(q_heads, bounds, table, kvh, a, between, [&](int i) { return s.places[i]; }, [&](int i, uint64_t key) { s.keys[i] = key; });
                __syncthreads();
                for (int i = tid; i < between; i += kThreads) {
                    const uint64_t key = s.keys[i];
                    const int place = s.places[i];
                    uint32_t ahead = 0;
                    for (int j = 0; j < between; ++j) ahead += s.keys[j] > key || (s.keys[j] == key && s.places[j] < place);
                    // kept or not from here on: a key above or below all others
                    s_keys[place - lo] = ahead < left ? ~0u : 0u;
                }
                __syncthreads();
            } else if (settled) {
                for (int i = tid; i < between; i += kThreads) s_keys[s.places[i] - lo] = ~0u;
                __syncthreads();
            }
        }
    }
    if (settled) {
        write_kept(s, nb, 0, out, [&](int b) {
            if (b < lo || b >= lo + compete) return 2;
            const uint32_t key = s_keys[b - lo];
            return key == ~0u || (key != 0 && score_of(key) > top) ? 2 : 0;
        });
        return;
    }

    // ---- all in 64 bits
    uint64_t *keys = all_keys + int64_t(blockIdx.x) * (a.stride / 2);  // where the scores were
    __syncthreads();
    score_exactly<T, D>(q_heads, bounds, table, kvh, a, compete, [&](int i) { return lo + i; }, [&](int i, uint64_t key) { keys[i] = key; });
    __threadfence_block();
    __syncthreads();
    // prefix, mask: the digits of the smallest key kept; left: places for those that agree in them
    uint64_t prefix = 0, mask = 0;
    left = places;
    for (int shift = 56; shift >= 0; shift -= 8) {
        s.count[tid] = 0;
        __syncthreads();
        for (int i = tid; i < compete; i += kThreads) {
            const uint64_t key = keys[i];
            if ((key & mask) == prefix) atomicAdd(&s.count[255 - (uint32_t(key >> shift) & 255)], 1u);
        }
        __syncthreads();
        find_digit(s, left);
        const uint32_t at = s.digit[0];
        left -= s.digit[1];
        prefix |= uint64_t(255 - at) << shift;
        mask |= uint64_t(255) << shift;
        const uint32_t here = s.count[at];
        __syncthreads();
        if (here == left) break;  // all that agree so far are kept
    }
    write_kept(s, nb, left, out, [&](int b) {
        if (b < lo || b >= lo + compete) return 2;
        const uint64_t key = keys[b - lo] & mask;
        return key > prefix ? 2 : key == prefix ? 1 : 0;
    });
}

}  // namespace

hipError_t launch_block_select(const void *q, const void *bounds, const int32_t *block_tables, const int32_t *context_lens, const int32_t *q_start,
                               int32_t *selected, void *workspace, const SelectArgs &a, int dtype, int head_dim, hipStream_t stream) {
    const int64_t pairs = int64_t(a.total_q) * a.num_kv_heads;
    float *scores = static_cast<float *>(workspace), *sizes = scores + pairs * a.stride;
    const int shares = a.shares;
    auto with_type = [&](auto type, auto dim) {
        using T = decltype(type);
        constexpr int D = decltype(dim)::value;
        const T *qp = static_cast<const T *>(q), *bp = static_cast<const T *>(bounds);
        if (shares > 0) {
            const int set_rows = 16 >> a.heads_log2;
            auto launch = [&](auto kernel, int rows) {
                const dim3 grid(unsigned((a.total_q + rows - 1) / rows * a.num_kv_heads), unsigned(shares));
                kernel<<<grid, dim3(kThreads), 0, stream>>>(qp, bp, block_tables, context_lens, q_start, scores, sizes, a, rows);
            };
            constexpr int kMore = sizeof(T) * D > 256 ? 1 : 2;  // what the registers hold
            if (q_start && kMore > 1) launch(block_scores_kernel<T, D, kMore>, set_rows * kMore);
            else launch(block_scores_kernel<T, D, 1>, q_start ? set_rows : 1);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        auto choose = [&](auto kernel) {
            kernel<<<dim3(unsigned(pairs)), dim3(kThreads), 0, stream>>>(qp, bp, block_tables, context_lens, q_start, scores, sizes, shares,
                                                                         static_cast<uint64_t *>(workspace), selected, a);
        };
        if (a.max_blocks <= 2048) choose(block_choose_kernel<T, D, 2048>); else choose(block_choose_kernel<T, D, 12288>);
        return hipGetLastError();
    };
    if (dtype == KVC_F32)
        return head_dim == 64 ? with_type(float(), std::integral_constant<int, 64>()) : with_type(float(), std::integral_constant<int, 128>());
    return head_dim == 64 ? with_type(uint16_t(), std::integral_constant<int, 64>()) : with_type(uint16_t(), std::integral_constant<int, 128>());
}

}  // namespace kvc
