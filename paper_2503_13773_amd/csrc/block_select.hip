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
// of 64 in fp32: 166 us).  So they come from the matrix cores, as
//
//   sum_d q+_d hi_d + q-_d lo_d,  q+ = max(q, 0), q- = min(q, 0)      (exact in the type of q)
//
// with fp32 sums, and beside them a bound on what these can be off: error <= kSlack * sum_d |q_d| max(|lo_d|, |hi_d|), the largest of a row
// E.  The choice finds where the last kept score lies, T: blocks more than 2 E above T are kept and ones more than 2 E below are
// not, whatever the true scores are (the true last score is within E of T, each true score within E of its own).  Only the few in between are
// scored in 64 bits and ranked.  Rows where that settles too little (many equal scores, something not finite) are scored in 64 bits
// throughout.
//
// Scores and choice are two launches.  A decode batch of at most 1024 (row, KV head) pairs and 2048 blocks has a workgroup or a few per
// pair and the last one to finish a pair's scores chooses at once, which saves the second launch.
//
// Bound: the bounds' bytes in a decode batch, read in pieces of 2 * D * e (32 long documents, 64 / 8 heads of 128, 172 MB:
// 44.6 us = 3.85 TB/s); the chain of dependent phases where there are few rows (one document of 30 011 tokens:
// 10.8 us, of which the choice is 4.5); products and LDS for chunks, whose rows share the bounds (1000 rows, 16 / 4 heads of 64 in fp32:
// 36 us of scores, 14 us of choice).
#include <type_traits>

#include "cache_rows.h"
#include "kvc_internal.h"
#include "lds_loads.h"
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

// An operand: 8 numbers of a lane.  bf16 as they are (the matrix cores keep subnormal numbers); fp32 as the sum of two bf16 values, 2^-17 relative
// or, below the normal numbers, 2^-134.  Bounds smaller than kSmallest count as that in the sum of sizes, whose share of slack (over 2^-14 of
// it) is more than they can lose; queries with numbers below 2^-100 are left to 64 bits.
constexpr float kSmallest = 0x1p-118f;
template <class T>
struct Operand;
template <>
struct Operand<uint16_t> {
    uint4 w;
    __device__ void load(const uint16_t *p) { w = *reinterpret_cast<const uint4 *>(p); }
    // from a stage's row, whose 16-byte chunk c lies at place(c)
    template <class Place>
    __device__ void load(const unsigned char *row, int first, Place place) { w = *reinterpret_cast<const uint4 *>(row + place(first / 8)); }
    __device__ bool too_small() const { return false; }
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
    __device__ void load(const float *p) { take(*reinterpret_cast<const float4 *>(p), *reinterpret_cast<const float4 *>(p + 4)); }
    __device__ void take(const float4 &a, const float4 &b) {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    template <class Place>
    __device__ void load(const unsigned char *row, int first, Place place) {
        take(*reinterpret_cast<const float4 *>(row + place(first / 4)), *reinterpret_cast<const float4 *>(row + place(first / 4 + 1)));
    }
    __device__ bool too_small() const {
        bool any = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) any |= x[i] != 0.f && fabsf(x[i]) < 0x1p-100f;
        return any;
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
            s[i] = pack_bf16(fmaxf(fmaxf(fabsf(a.x[2 * i]), fabsf(b.x[2 * i])), kSmallest), fmaxf(fmaxf(fabsf(a.x[2 * i + 1]), fabsf(b.x[2 * i + 1])), kSmallest));
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

// Largest over aligned groups of 1 << log2 lanes, up to 16: all of a group get it.
__device__ inline float over_heads(float x, int log2) {
    if (log2 > 0) x = max_of(x, lanes::permuted<lanes::kXor1>(x));
    if (log2 > 1) x = max_of(x, lanes::permuted<lanes::kXor2>(x));
    if (log2 > 2) x = max_of(x, lanes::permuted<lanes::kMirror8>(x));
    if (log2 > 3) x = max_of(x, lanes::permuted<lanes::kMirror16>(x));
    return x;
}

// ---- the choice

// Order of numbers as order of whole numbers.
__device__ inline uint64_t key_of(double s) {
    if (!__builtin_isfinite(s)) return ~uint64_t(0);
    const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);  // -0 is 0
    return u >> 63 ? ~u : u | uint64_t(1) << 63;
}

// x of another lane, both halves.
template <int CTRL>
__device__ inline double permuted(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, uint64_t(lanes::permuted<CTRL>(uint32_t(u >> 32))) << 32 | lanes::permuted<CTRL>(uint32_t(u)));
}
// Sum over aligned groups of LR lanes, 8, 16 or 32.
template <int LR>
__device__ inline double sum_over_lanes(double x) {
    x += permuted<lanes::kXor1>(x);
    x += permuted<lanes::kXor2>(x);
    x += permuted<lanes::kMirror8>(x);
    if constexpr (LR > 8) x += permuted<lanes::kMirror16>(x);
    if constexpr (LR > 16) x += __shfl_xor(x, 16);
    return x;
}

// A block's score for one head in 64 bits, by the LR lanes of a group.  Channel by channel
// max(q lo, q hi) = (q (hi + lo) + |q| (hi - lo)) / 2, and twice the score is as good.
template <class T, int D>
struct Exactly {
    static constexpr int N = Load<T>::N, LR = D / N;
    const T *q_heads, *bounds;  // of the row and KV head; of all blocks
    int num_kv_heads, kvh;
    __device__ uint64_t key(int block, int h) const {
        const int c = threadIdx.x % LR;
        const T *src = bounds + (int64_t(block) * num_kv_heads + kvh) * 2 * D + c * N;
        double lo[N], hi[N], x[N], s = 0.0;
        Load<T>::get(*reinterpret_cast<const uint4 *>(q_heads + int64_t(h) * D + c * N), x);
        Load<T>::get(*reinterpret_cast<const uint4 *>(src), lo);
        Load<T>::get(*reinterpret_cast<const uint4 *>(src + D), hi);
#pragma unroll
        for (int i = 0; i < N; ++i) s = fma(x[i], hi[i] + lo[i], fma(fabs(x[i]), hi[i] - lo[i], s));
        return key_of(sum_over_lanes<LR>(s));
    }
};


// What a workgroup shares while it chooses.
template <int WAVES, int MINE>
struct Choice {
    static constexpr int kBins = WAVES == 1 ? 256 : 1024;  // of the scores' range
    static constexpr int kBand = WAVES == 1 ? 128 : 512;   // blocks that are ranked by comparing each with each
    uint32_t bins[kBins], sums[WAVES], found[2], between;
    float stats[WAVES][3];
    uint32_t kept[MINE][WAVES], equal[MINE][WAVES];
    uint64_t keys[kBand];
    int places[kBand], blocks[kBand], won[kBand];
};

// What needs no scores: rows that keep all they see, and the blocks that are always kept.  Whether there is more to do, and then for the
// blocks lo .. lo + compete - 1 there are `places` places, fewer than that.
__device__ inline bool keep_the_ends(int32_t *out, int pos, const SelectArgs &a, int *compete, int *places) {
    const int nb = pos < 0 ? 0 : (pos >> a.block_size_log2) + 1;
    if (nb <= a.budget) {
        for (int i = threadIdx.x; i < a.budget; i += blockDim.x) out[i] = i < nb ? i : -1;
        return false;
    }
    *compete = nb - a.keep_last - a.keep_first;
    *places = a.budget - a.keep_last - a.keep_first;
    for (int i = threadIdx.x; i < a.keep_first + a.keep_last; i += blockDim.x)
        out[i < a.keep_first ? i : *places + i] = i < a.keep_first ? i : *compete + i;
    return *places > 0;
}

// The rest of a row and KV head's list.  x, blocks: scores and pool indices of blocks k * THREADS + tid of those that compete, size: the largest sum of sizes, of this thread's
// shares.  Rows with more competing blocks than THREADS * MINE are scored in 64 bits throughout.
template <class T, int D, int THREADS, int MINE>
__device__ inline void choose(Choice<THREADS / 64, MINE> &s, float (&x)[MINE], const int (&blocks)[MINE], float size, int row, int kvh, int compete, int places, const T *q,
                              const T *bounds, const int32_t *table, uint64_t *keys, int32_t *out, const SelectArgs &a) {
    constexpr int WAVES = THREADS / 64, kBins = Choice<WAVES, MINE>::kBins, kBand = Choice<WAVES, MINE>::kBand;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, lo = a.keep_first;
    out += lo;
    const Exactly<T, D> exactly = {q + (int64_t(row) * a.num_q_heads + kvh * a.group) * D, bounds, a.num_kv_heads, kvh};
    constexpr int LR = Exactly<T, D>::LR, kTeams = THREADS / LR;
    const int team = tid / LR;

    // Writes, in ascending order, the blocks of this pass over MINE * THREADS of them, from block `from` on, that are kept: what(k) = 2 kept,
    // 1 kept if among the first `left` of these (EQUAL).  kept, equal: how many there have been before.
    auto write_kept = [&](auto what, int from, int left, auto EQUAL, uint32_t &kept, uint32_t &equal) __attribute__((always_inline)) {
        constexpr bool kEqual = decltype(EQUAL)::value;
        static_assert(MINE * WAVES % 64 == 0 || MINE * WAVES <= 64, "counts of a lane");
        uint64_t xs[MINE], ys[MINE];
#pragma unroll
        for (int k = 0; k < MINE; ++k) {
            const int w = from + k * THREADS + tid < compete ? what(k) : 0;
            xs[k] = __ballot(w == 2);
            ys[k] = kEqual ? __ballot(w == 1) : 0;
            if (lane == 0) {
                s.kept[k][wave] = __popcll(xs[k]);
                if (kEqual) s.equal[k][wave] = __popcll(ys[k]);
            }
        }
        __syncthreads();
        // a lane sums what stands before (turn k, wavefront w) = entry k * WAVES + w, 64 entries at a time
        const uint64_t below = (uint64_t(1) << lane) - 1, bit = uint64_t(1) << lane;
        constexpr int kEntries = MINE * WAVES, kTurns = 64 / WAVES;
#pragma unroll
        for (int e0 = 0; e0 < kEntries; e0 += 64) {
            const uint32_t mine_x = e0 + lane < kEntries ? (&s.kept[0][0])[e0 + lane] : 0, mine_y = kEqual && e0 + lane < kEntries ? (&s.equal[0][0])[e0 + lane] : 0;
            const uint32_t sum_x = uint32_t(lanes::prefix_sum(int(mine_x))), sum_y = kEqual ? uint32_t(lanes::prefix_sum(int(mine_y))) : 0;
#pragma unroll
            for (int j = 0; j < kTurns; ++j) {
                const int k = e0 / WAVES + j;
                if (k >= MINE) break;
                const int at = j * WAVES + wave;
                const uint32_t x_before = kept + __builtin_amdgcn_readlane(sum_x - mine_x, at) + __popcll(xs[k] & below);
                const uint32_t y_before = kEqual ? equal + __builtin_amdgcn_readlane(sum_y - mine_y, at) + __popcll(ys[k] & below) : 0;
                if ((xs[k] & bit) || ((ys[k] & bit) && int(y_before) < left)) out[x_before + min(int(y_before), left)] = lo + from + k * THREADS + tid;
            }
            kept += __builtin_amdgcn_readlane(sum_x, 63);
            if (kEqual) equal += __builtin_amdgcn_readlane(sum_y, 63);
        }
    };
    uint32_t kept = 0, equal = 0;

    // ---- by the scores of the matrix cores
    if (compete <= THREADS * MINE) {
        float least = INFINITY, most = -INFINITY;
        bool finite = true;
#pragma unroll
        for (int k = 0; k < MINE; ++k) {
            if (k * THREADS + tid < compete) {
                finite &= __builtin_isfinite(x[k]);
                least = fminf(least, x[k]);
                most = fmaxf(most, x[k]);
            } else {
                x[k] = -INFINITY;
            }
        }
        least = lanes::over_wave(least, [](float u, float v) { return fminf(u, v); });
        most = lanes::wave_max(most);
        size = lanes::over_wave(size, max_of);
        if (__ballot(!finite)) size = INFINITY;
        if (lane == 0) {
            s.stats[wave][0] = least;
            s.stats[wave][1] = most;
            s.stats[wave][2] = size;
        }
#pragma unroll
        for (int i = 0; i < kBins / THREADS; ++i) s.bins[i * THREADS + tid] = 0;
        if (tid == 0) s.between = 0;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            least = fminf(least, s.stats[w][0]);
            most = fmaxf(most, s.stats[w][1]);
            size = max_of(size, s.stats[w][2]);
        }
        if (__builtin_isfinite(size) && size < 1e30f) {
            const float slack = kSlack<T, D> * size + 1e-30f;
            // The last kept score lies between least and most: narrowed down to a bin of a kBins-th of that, again while that leaves many
            // blocks and the bin is wide.  A bin holds what rounding says it holds; its borders are taken a millionth of the range wider.
            for (;;) {
                const float range = most - least, per_bin = kBins / range;
                // bins from the top, scores above `most` in the first
#pragma unroll
                for (int k = 0; k < MINE; ++k)
                    if (x[k] >= least) atomicAdd(&s.bins[kBins - 1 - int(fminf(fmaxf((x[k] - least) * per_bin, 0.f), float(kBins - 1)))], 1u);
                __syncthreads();
                constexpr int kEach = kBins / THREADS;
                uint32_t sum = 0;
#pragma unroll
                for (int i = 0; i < kEach; ++i) sum += s.bins[tid * kEach + i];
                const uint32_t incl = uint32_t(lanes::prefix_sum(int(sum)));
                if (lane == 63) s.sums[wave] = incl;
                __syncthreads();
                uint32_t upto = incl - sum;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) upto += w < wave ? s.sums[w] : 0;
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const uint32_t count = s.bins[tid * kEach + i];
                    if (upto < uint32_t(places) && upto + count >= uint32_t(places)) {  // one bin
                        s.found[0] = tid * kEach + i;
                        s.found[1] = count;
                    }
                    upto += count;
                }
                __syncthreads();
                const int bin = kBins - 1 - int(s.found[0]);
                const bool many = s.found[1] > 32;
                const float width = range * (1.f / kBins), wider = range * 1e-6f + fabsf(least) * 2.5e-7f;
                const float bottom = least + bin * width - wider;
                most = s.found[0] == 0 ? most : bottom + width + 2.f * wider;
                least = bottom;
                if (!many || !(width > slack) || s.found[0] == 0) break;
#pragma unroll
                for (int i = 0; i < kEach; ++i) s.bins[tid * kEach + i] = 0;
                __syncthreads();
            }
            const float bottom = least - 2.f * slack, top = most + 2.f * slack;  // above top: kept, below bottom: not
            int between[MINE], sure = 0;
#pragma unroll
            for (int k = 0; k < MINE; ++k) {
                between[k] = -1;
                sure += __popcll(__ballot(x[k] > top));
                if (x[k] >= bottom && x[k] <= top) {
                    between[k] = int(atomicAdd(&s.between, 1u));
                    if (between[k] < kBand) {
                        s.places[between[k]] = lo + k * THREADS + tid;
                        s.blocks[between[k]] = blocks[k];
                        s.keys[between[k]] = 0;
                    }
                }
            }
            if (lane == 0) s.sums[wave] = sure;
            __syncthreads();
            int left = places;  // for those between
#pragma unroll
            for (int w = 0; w < WAVES; ++w) left -= s.sums[w];
            const int band = int(s.between);
            if (band <= kBand) {
                if (band != left) {
                    // a team of LR lanes per block and head
                    for (int i = team; i < band * a.group; i += kTeams) {
                        const int at = i / a.group;
                        const uint64_t key = exactly.key(s.blocks[at], i - at * a.group);
                        if (tid % LR == 0) atomicMax(reinterpret_cast<unsigned long long *>(&s.keys[at]), static_cast<unsigned long long>(key));
                    }
                    __syncthreads();
                    for (int i = tid; i < band; i += THREADS) {
                        const uint64_t key = s.keys[i];
                        const int place = s.places[i];
                        int ahead = 0;
                        for (int j = 0; j < band; ++j) ahead += s.keys[j] > key || (s.keys[j] == key && s.places[j] < place);
                        s.won[i] = ahead < left;
                    }
                    __syncthreads();
                }
                write_kept([&](int k) { return (between[k] < 0 ? x[k] > top : band == left || s.won[between[k]]) ? 2 : 0; }, 0, 0, std::false_type(), kept, equal);
                return;
            }
        }
    }

    // ---- all in 64 bits
    __syncthreads();
    for (int i = team; i < compete; i += kTeams) {
        uint64_t best = 0;
#pragma unroll 1
        for (int h = 0; h < a.group; ++h) {
            const uint64_t key = exactly.key(table[lo + i], h);
            best = key > best ? key : best;
        }
        if (tid % LR == 0) keys[i] = best;
    }
    __threadfence_block();
    // prefix, mask: the digits of the smallest key kept; left: places for those that agree in them
    uint64_t prefix = 0, mask = 0;
    int left = places;
    constexpr int kDigit = THREADS < 256 ? 6 : 8, kDigits = 1 << kDigit;
    for (int bits = 64; bits > 0;) {
        const int shift = max(bits - kDigit, 0);
        const uint32_t last = (1u << (bits - shift)) - 1;
        if (tid < kDigits) s.bins[tid] = 0;
        __syncthreads();
        for (int i = tid; i < compete; i += THREADS) {
            const uint64_t key = keys[i];
            if ((key & mask) == prefix) atomicAdd(&s.bins[last - (uint32_t(key >> shift) & last)], 1u);
        }
        __syncthreads();
        uint32_t count = 0, incl = 0;
        if (tid < kDigits) {
            count = s.bins[tid];
            incl = uint32_t(lanes::prefix_sum(int(count)));
            if (lane == 63) s.sums[wave] = incl;
        }
        __syncthreads();
        if (tid < kDigits) {
            int before = int(incl - count);
            for (int w = 0; w < wave; ++w) before += s.sums[w];
            if (before < left && before + int(count) >= left) {  // one thread
                s.found[0] = tid;
                s.found[1] = before;
            }
        }
        __syncthreads();
        const uint32_t at = s.found[0];
        left -= int(s.found[1]);
        prefix |= uint64_t(last - at) << shift;
        mask |= uint64_t(last) << shift;
        bits = shift;
        const int here = int(s.bins[at]);
        __syncthreads();
        if (here == left) break;  // all that agree so far are kept
    }
    for (int from = 0; from < compete; from += MINE * THREADS) {
        write_kept([&](int k) {
            const uint64_t key = keys[from + k * THREADS + tid] & mask;
            return key > prefix ? 2 : key == prefix ? 1 : 0;
        }, from, left, std::true_type(), kept, equal);
        __syncthreads();
    }
}

// Columns of a product are heads of rows of q: `heads` of them (a power of two, the group's last head again in place of what it lacks)
// times 16 / heads rows; GROUPS such sets of rows share the loads.  Rows of products are 16 blocks.  blockIdx.x = KV head + KV heads * tile of
// rows (tile_rows: one of a decode step, as many as there are columns for of chunks), blockIdx.y = share of the blocks.  Writes the scores of all
// rows of the tile, and per row and share the largest sum of sizes.
// MINE > 0 (tiles of one row): the workgroup that finishes a row and KV head's last share chooses for it, MINE blocks a thread at most.  Scores and
// sizes travel by device-scope accesses; each workgroup waits for its own and counts itself; nobody waits for anybody.  A single share's
// scores stay in LDS.
template <class T, int D, int GROUPS, int THREADS, int MINE>
__global__ __launch_bounds__(THREADS, sizeof(T) == 2 && MINE > 0 ? 4 : 1) void block_scores_kernel(const T *__restrict__ q, const T *__restrict__ bounds, const int32_t *__restrict__ block_tables,
                                                                const int32_t *__restrict__ context_lens, const int32_t *__restrict__ q_start,
                                                                float *__restrict__ scores, float *__restrict__ sizes, int32_t *__restrict__ counters,
                                                                int32_t *__restrict__ selected, SelectArgs a, int tile_rows) {
    constexpr int J = D / 32, WAVES = THREADS / 64;
    constexpr bool HERE = MINE > 0;
    using Op = Operand<T>;
    __shared__ float s_size[WAVES][GROUPS][16];
    using Chosen = std::conditional_t<HERE, Choice<WAVES, HERE ? MINE : 1>, int>;
    // Bounds of 16 blocks per wavefront, afterwards what the choice shares.  A decode step's rows share no blocks: whole rows of bounds go straight into
    // LDS, past the caches, those of the next blocks under the products of these.  (Loads in the operands' layout touch 16 lines each: 32 long
    // documents 54.6 us so, through LDS 48.8, and past the caches 44.6; rows of chunks read bounds again and gain nothing, 49.6 and 49.3;
    // sets of fp32 of 128 are more than LDS holds for enough wavefronts.)
    constexpr int kRecord = 2 * D * int(sizeof(T)), kSet = 16 * kRecord, kChunks = kRecord / 16, kLoads = kSet / 1024;
    constexpr bool STAGED = GROUPS == 1 && kRecord <= 512;  // with GROUPS == 1 chunks have rows of 1024 bytes
    constexpr int kStage = STAGED ? WAVES * kSet : 0;
    __shared__ __attribute__((aligned(1024))) unsigned char s_stage[kStage > int(sizeof(Chosen)) ? kStage : sizeof(Chosen)];
    Chosen &s_choice = *reinterpret_cast<Chosen *>(s_stage);
    __shared__ float s_scores[HERE ? THREADS * MINE : 1];
    __shared__ float s_whole_size;
    __shared__ int s_last;
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
        if constexpr (HERE) {
            int compete, places;
            if (blockIdx.y == 0) keep_the_ends(selected + (int64_t(row0) * a.num_kv_heads + kvh) * a.budget, pos, a, &compete, &places);
            if (nb > a.budget && int(blockIdx.y) * a.share >= nb - a.keep_last - a.keep_first) continue;
        }
        if (nb <= a.budget) continue;
        const int first = a.keep_first + blockIdx.y * a.share, last = min(nb - a.keep_last, first + a.share);
        const int32_t *table = block_tables + int64_t(n) * a.max_blocks_per_seq;
        const bool whole = HERE && nb - a.keep_last - a.keep_first <= a.share;  // one share is all there is
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
                    if (x.too_small()) size[g] = INFINITY;
                    plus[g][j] = x.plus();
                    minus[g][j] = x.minus();
                }
            }
            int b0 = first + 16 * wave;
            int block = b0 < last ? table[min(b0 + r, last - 1)] : 0;
            // chunk c of row R of a stage lies at c ^ R: 16 rows' chunks of one index fall into 16 places of 256 bytes
            unsigned char *const stage = s_stage + (STAGED ? wave * kSet : 0);
            const uint32_t lds = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(reinterpret_cast<uintptr_t>(stage)))));
            auto issue = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int row = i * (64 / kChunks) + lane / kChunks, from = __shfl(block, row);
                    load_to_lds<false>(reinterpret_cast<const unsigned char *>(bounds) + (int64_t(from) * a.num_kv_heads + kvh) * kRecord +
                                          ((lane % kChunks ^ row) << 4), lds + 1024 * i);
                }
            };
            if (STAGED && b0 < last) {
                issue();
                block = table[min(b0 + 16 * WAVES + r, last - 1)];
            }
            for (; b0 < last; b0 += 16 * WAVES) {
                const T *src = bounds + (int64_t(block) * a.num_kv_heads + kvh) * 2 * D + 8 * quad;
                Op lo[J], hi[J];
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    if constexpr (STAGED) {
                        if (j == 0) wait_for_loads<0>();
                        const unsigned char *const row = stage + r * kRecord;
                        auto place = [&](int c) __attribute__((always_inline)) { return (c ^ r) << 4; };
                        lo[j].load(row, 8 * quad + 32 * j, place);
                        hi[j].load(row, 8 * quad + 32 * j + D, place);
                    } else {
                        lo[j].load(src + 32 * j);
                        hi[j].load(src + D + 32 * j);
                    }
                }
                if constexpr (STAGED) {
                    wait_for_lds();
                    if (b0 + 16 * WAVES < last) {
                        issue();
                        block = table[min(b0 + 32 * WAVES + r, last - 1)];
                    }
                } else {
                    block = table[min(b0 + 16 * WAVES + r, last - 1)];
                }
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
#pragma unroll
                    for (int i = 0; i < 4; ++i) best[i] = over_heads(best[i], a.heads_log2);
                    const int row = row0 + g * set_rows + my_row;
                    if (my_head == 0 && row < row1) {
                        float *dst = scores + (int64_t(row) * a.num_kv_heads + kvh) * a.stride + b0 - a.keep_first + 4 * quad;
                        if (h0 > 0) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float other = HERE && whole ? s_scores[b0 - a.keep_first + 4 * quad + i]
                                                    : HERE        ? __hip_atomic_load(dst + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)
                                                                  : dst[i];
                                best[i] = max_of(other, best[i]);
                            }
                        }
                        // rows of `stride` have room for whole sets of blocks
                        if (HERE && whole) {
                            *reinterpret_cast<floatx4 *>(s_scores + (b0 - a.keep_first + 4 * quad)) = best;
                        } else if constexpr (HERE) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) __hip_atomic_store(dst + i, best[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        } else {
                            *reinterpret_cast<floatx4 *>(dst) = best;
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            size[g] = lanes::over_rows(size[g], max_of);
            size[g] = over_heads(size[g], a.heads_log2);
            if (quad == 0) s_size[wave][g][r] = size[g];
        }
        __syncthreads();
        if (threadIdx.x < 16 * GROUPS) {
            const int g = threadIdx.x >> 4, row = row0 + g * set_rows + my_row;
            float x = s_size[0][g][r];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) x = max_of(x, s_size[w][g][r]);
            if (my_head == 0 && row < row1) {
                float *dst = sizes + (int64_t(row) * a.num_kv_heads + kvh) * gridDim.y + blockIdx.y;
                if (HERE && whole) s_whole_size = x;
                else if (HERE) __hip_atomic_store(dst, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                else *dst = x;
            }
        }
        if constexpr (HERE) {
            const int compete = nb - a.keep_last - a.keep_first, shares = (compete + a.share - 1) / a.share;
            const int64_t pair = int64_t(row0) * a.num_kv_heads + kvh;
            float *mine = scores + pair * a.stride;
            float x[MINE], most = 0.f;
            int blocks[MINE];
            if (!whole) {
                // the count may become visible only after the scores: every wavefront waits for its own stores, then all meet
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                if (threadIdx.x == 0) s_last = __hip_atomic_fetch_add(counters + pair * a.counter_step, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == shares - 1;
                __syncthreads();
                if (!s_last) return;
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");  // the fetches stay behind the count
                if (threadIdx.x == 0) __hip_atomic_store(counters + pair * a.counter_step, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            } else {
                __syncthreads();
            }
#pragma unroll
            for (int k = 0; k < MINE; ++k) {
                const int i = k * THREADS + int(threadIdx.x);
                blocks[k] = table[min(a.keep_first + i, nb - 1)];
                x[k] = whole ? s_scores[i] : __hip_atomic_load(mine + min(i, a.stride - 1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            if (whole) {
                most = s_whole_size;
            } else {
                for (int i = threadIdx.x; i < shares; i += THREADS)
                    most = max_of(most, __hip_atomic_load(sizes + pair * gridDim.y + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
            }
            choose<T, D, THREADS, MINE>(s_choice, x, blocks, most, row0, kvh, compete, a.budget - a.keep_last - a.keep_first, q, bounds, table,
                                                reinterpret_cast<uint64_t *>(mine), selected + pair * a.budget, a);
            return;
        }
        __syncthreads();
    }
}

// A launch of its own, a workgroup per row and KV head.
template <class T, int D, int THREADS, int MINE>
__global__ __launch_bounds__(THREADS) void block_choose_kernel(const T *__restrict__ q, const T *__restrict__ bounds, const int32_t *__restrict__ block_tables,
                                                               const int32_t *__restrict__ context_lens, const int32_t *__restrict__ q_start,
                                                               float *__restrict__ scores, const float *__restrict__ sizes, int32_t *__restrict__ selected,
                                                               SelectArgs a) {
    __shared__ Choice<THREADS / 64, MINE> s;
    const int tid = threadIdx.x, row = blockIdx.x / a.num_kv_heads, kvh = blockIdx.x - row * a.num_kv_heads;
    // the scores are asked for before it is known how many there are: there is room for `stride` of them
    float x[MINE], size = 0.f;
    float *mine = scores + int64_t(blockIdx.x) * a.stride;
    if (a.shares > 0) {
#pragma unroll
        for (int k = 0; k < MINE; ++k) x[k] = mine[min(k * THREADS + tid, a.stride - 1)];
    }
    int n, pos, compete, places;
    if (!find_row(row, q_start, context_lens, a.num_seqs, a.max_context_len, &n, &pos)) return;
    int32_t *out = selected + int64_t(blockIdx.x) * a.budget;
    if (!keep_the_ends(out, pos, a, &compete, &places)) return;
    const int32_t *table = block_tables + int64_t(n) * a.max_blocks_per_seq;
    int blocks[MINE];
#pragma unroll
    for (int k = 0; k < MINE; ++k) blocks[k] = table[min(a.keep_first + k * THREADS + tid, (pos >> a.block_size_log2))];
    for (int i = tid; i * a.share < compete; i += THREADS) size = max_of(size, sizes[int64_t(blockIdx.x) * a.shares + i]);
    choose<T, D, THREADS, MINE>(s, x, blocks, size, row, kvh, compete, places, q, bounds, table, reinterpret_cast<uint64_t *>(mine), out, a);
}

}  // namespace

hipError_t launch_block_select(const void *q, const void *bounds, const int32_t *block_tables, const int32_t *context_lens, const int32_t *q_start,
                               int32_t *selected, void *workspace, const SelectArgs &a, int dtype, int head_dim, hipStream_t stream) {
    const int64_t pairs = int64_t(a.total_q) * a.num_kv_heads;
    auto *counters = static_cast<int32_t *>(workspace);
    float *scores = reinterpret_cast<float *>(static_cast<char *>(workspace) + kWorkspaceHeaderBytes), *sizes = scores + pairs * a.stride;
    auto with_type = [&](auto type, auto dim) {
        using T = decltype(type);
        constexpr int D = decltype(dim)::value;
        const T *qp = static_cast<const T *>(q), *bp = static_cast<const T *>(bounds);
        if (a.shares > 0) {
            constexpr int kSets = select_sets(sizeof(T) == 4 ? KVC_F32 : KVC_BF16, D);
            auto launch = [&](auto kernel, int rows, int threads) {
                const dim3 grid(unsigned((a.total_q + rows - 1) / rows * a.num_kv_heads), unsigned(a.shares));
                kernel<<<grid, dim3(threads), 0, stream>>>(qp, bp, block_tables, context_lens, q_start, scores, sizes, counters, selected, a, rows);
            };
            const int set_rows = 16 >> a.heads_log2;
            if (a.choose_here && a.max_blocks <= kSmallChoice) launch(block_scores_kernel<T, D, 1, 256, 2>, 1, 256);
            else if (a.choose_here) launch(block_scores_kernel<T, D, 1, 512, 4>, 1, 512);
            else if (a.total_q > a.num_seqs) launch(block_scores_kernel<T, D, kSets, kThreads, 0>, set_rows * kSets, kThreads);
            else launch(block_scores_kernel<T, D, 1, kThreads, 0>, 1, kThreads);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess || a.choose_here) return e;
        }
        auto choose_by = [&](auto kernel, int threads) {
            kernel<<<dim3(unsigned(pairs)), dim3(threads), 0, stream>>>(qp, bp, block_tables, context_lens, q_start, scores, sizes, selected, a);
        };
        // Many rows fill the device with small workgroups: a wavefront each up to 512 blocks (1000 rows, 4 KV heads, both launches, 46.6 us, 256
        // threads each 52.6; 24 rows, 2 KV heads, up to 190 blocks, 16.4 and 14.4), 256 threads up to 2048 (182 rows, 16 KV heads, up to 746 blocks
        // 29.6 us, 512 threads 34.6).
        const bool many = pairs > 4 * kNumCUs;
        if (a.max_blocks <= kSmallChoice && many) choose_by(block_choose_kernel<T, D, 64, 8>, 64);
        else if (a.max_blocks <= kSmallChoice) choose_by(block_choose_kernel<T, D, 256, 2>, 256);
        else if (a.max_blocks <= kSelectHereBlocks && many) choose_by(block_choose_kernel<T, D, 256, 8>, 256);
        else if (a.max_blocks <= kSelectHereBlocks) choose_by(block_choose_kernel<T, D, 512, 4>, 512);
        else choose_by(block_choose_kernel<T, D, 1024, 16>, 1024);
        return hipGetLastError();
    };
    if (dtype == KVC_F32)
        return head_dim == 64 ? with_type(float(), std::integral_constant<int, 64>()) : with_type(float(), std::integral_constant<int, 128>());
    return head_dim == 64 ? with_type(uint16_t(), std::integral_constant<int, 64>()) : with_type(uint16_t(), std::integral_constant<int, 128>());
}

}  // namespace kvc
