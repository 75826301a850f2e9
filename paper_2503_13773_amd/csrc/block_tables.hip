// kvc_block_tables_extend: blocks from a free list for the new tokens of every sequence, and the slot, position and sequence of
// every new token (gfx950).  With need_n the blocks that sequence n lacks, new_n its new tokens,
//
//   F_n = sum_{i<n} need_i,  R_n = sum_{i<n} new_i;   granted: need_n = 0 or F_n + need_n <= num_free, and R_n + new_n <= max_rows
//   Q_n = new_n if granted, else 0;   row sum_{i<n} Q_i + j of the maps is token ctx_n + j
//
// Bound: latency for an iteration's batch (lengths, scans, a table entry, the store), memory for large maps (16 bytes a row).  One launch up to
// 2048 sequences: every workgroup sums the lengths for itself, which are few, and takes its share of table entries and rows, so no
// workgroup waits for another.  64 sequences, one token each, 4.4 us; 1500 sequences, 1.05 M rows, 9.1-9.5 us (a search over all sequences and
// three dependent loads for every row by itself: 15.4 us; the 17 MB that are written take 3.4 us).
//
// A refusal for want of blocks refuses everybody behind who needs one, and one for want of rows everybody behind who brings any
// (the sums count refused sequences too), so the blocks dealt out are the front of the free list, in order.
#include "kvc_internal.h"
#include "pa_lanes.h"

namespace kvc {

namespace {

// Sums stop at 2^31 - 1, which is more than either limit (the host refuses larger ones).
__device__ inline uint32_t add_saturated(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }

// Inclusive scan over the lanes of a wavefront.
template <class Op>
__device__ inline uint32_t scan_wave(uint32_t x, Op op) {
    using namespace lanes;
    x = op(x, permuted<kShr + 1>(x));
    x = op(x, permuted<kShr + 2>(x));
    x = op(x, permuted<kShr + 4>(x));
    x = op(x, permuted<kShr + 8>(x));
    x = op(x, permuted<kBcast15, 0xa>(x));
    return op(x, permuted<kBcast31, 0xc>(x));
}

// Exclusive scan over the workgroup of two numbers per thread, starting from (and moving on) the carries.
template <int WAVES, class Op>
__device__ inline void scan_group(uint32_t &a, uint32_t &b, uint32_t &carry_a, uint32_t &carry_b, uint32_t (&s_sums)[2][WAVES], Op op) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint32_t ia = scan_wave(a, op), ib = scan_wave(b, op);
    if (lane == 63) {
        s_sums[0][wave] = ia;
        s_sums[1][wave] = ib;
    }
    __syncthreads();
    // lane w: the sum over wavefronts 0 .. w
    const uint32_t wa = scan_wave(lane < WAVES ? s_sums[0][lane] : 0u, op), wb = scan_wave(lane < WAVES ? s_sums[1][lane] : 0u, op);
    const uint32_t before_a = wave > 0 ? __builtin_amdgcn_readlane(wa, __builtin_amdgcn_readfirstlane(wave - 1)) : 0u;
    const uint32_t before_b = wave > 0 ? __builtin_amdgcn_readlane(wb, __builtin_amdgcn_readfirstlane(wave - 1)) : 0u;
    const uint32_t pa = uint32_t(__shfl_up(int(ia), 1)), pb = uint32_t(__shfl_up(int(ib), 1));
    a = op(op(carry_a, before_a), lane > 0 ? pa : 0u);
    b = op(op(carry_b, before_b), lane > 0 ? pb : 0u);
    carry_a = op(carry_a, __builtin_amdgcn_readlane(wa, WAVES - 1));
    carry_b = op(carry_b, __builtin_amdgcn_readlane(wb, WAVES - 1));
    __syncthreads();
}

// What a pass over sequences base .. base + kThreads * ITEMS - 1 leaves in LDS for each of them: its first row, the first of the blocks dealt out to it
// (one more entry than sequences), its length and the blocks it had.
template <int THREADS, int ITEMS>
struct Pass {
    static constexpr int kSeqs = THREADS * ITEMS;
    uint32_t rows[kSeqs + 1], first[kSeqs + 1], sums[2][THREADS / 64];
    int ctx[kSeqs], held[kSeqs];
};
struct Carries { uint32_t need, rows, dealt, taken; };

// Writes what is known per sequence where `write`.
template <int THREADS, int ITEMS>
__device__ inline void scan_pass(const TableArgs &t, int base, Carries &c, Pass<THREADS, ITEMS> &s, bool write) {
    const int first = base + threadIdx.x * ITEMS;
    int ctx[ITEMS], held[ITEMS] = {}, fresh[ITEMS];
    uint32_t need[ITEMS], rows[ITEMS], sum_need = 0, sum_rows = 0;
    auto saturated = [](uint32_t a, uint32_t b) { return add_saturated(a, b); };
    auto plain = [](uint32_t a, uint32_t b) { return a + b; };
    auto load = [&](const int32_t *p, int (&x)[ITEMS]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) x[k] = p[min(first + k, t.num_seqs - 1)];
    };
    load(t.context_lens, ctx);
    load(t.new_lens, fresh);
    if (t.held_blocks) load(t.held_blocks, held);
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        need[k] = rows[k] = 0;
        if (!t.held_blocks) held[k] = (ctx[k] + (1 << t.block_size_log2) - 1) >> t.block_size_log2;
        const int tokens = t.max_blocks_per_seq << t.block_size_log2;  // at most 2^30
        if (first + k < t.num_seqs && fresh[k] > 0 && ctx[k] >= 0 && ctx[k] <= tokens && fresh[k] <= tokens - ctx[k] && held[k] >= 0 &&
            held[k] <= t.max_blocks_per_seq) {
            rows[k] = fresh[k];
            need[k] = max(0, ((ctx[k] + fresh[k] - 1) >> t.block_size_log2) + 1 - held[k]);
        }
        sum_need = add_saturated(sum_need, need[k]);
        sum_rows = add_saturated(sum_rows, rows[k]);
    }
    scan_group(sum_need, sum_rows, c.need, c.rows, s.sums, saturated);
    uint32_t sum_dealt = 0, sum_taken = 0;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        sum_need = add_saturated(sum_need, need[k]);
        sum_rows = add_saturated(sum_rows, rows[k]);
        if (!((need[k] == 0 || sum_need <= uint32_t(t.num_free)) && sum_rows <= uint32_t(t.max_rows))) need[k] = rows[k] = 0;
        sum_dealt += rows[k];
        sum_taken += need[k];
    }
    scan_group(sum_dealt, sum_taken, c.dealt, c.taken, s.sums, plain);
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const int n = first + k;
        if (n < t.num_seqs) {
            s.rows[n - base] = sum_dealt;
            s.first[n - base] = sum_taken;
            s.ctx[n - base] = ctx[k];
            s.held[n - base] = held[k];
            if (write) {
                t.q_start[n] = int(sum_dealt);
                t.context_lens_out[n] = ctx[k] + int(rows[k]);
                if (t.held_blocks_out) t.held_blocks_out[n] = held[k] + int(need[k]);
            }
            sum_dealt += rows[k];
            sum_taken += need[k];
        }
    }
    const int count = min(Pass<THREADS, ITEMS>::kSeqs, t.num_seqs - base);
    if (threadIdx.x == 0) {
        s.rows[count] = c.dealt;
        s.first[count] = c.taken;
    }
}

// Largest i in [lo, hi) with s[i] <= x, where s[lo] <= x and x < s[hi].
__device__ inline int place_of(const uint32_t *s, int lo, int hi, uint32_t x) {
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}
// The same over [0, count) for an x that all lanes share, up to 64 * 64 entries: 64 at a time.
__device__ inline int place_of_all(const uint32_t *s, int count, uint32_t x) {
    const int lane = threadIdx.x & 63, stride = (count + 63) >> 6;
    const int at = lane * stride;
    const int base = (__popcll(__ballot(at < count && s[min(at, count)] <= x)) - 1) * stride;
    return base + __popcll(__ballot(lane < stride && base + lane < count && s[min(base + lane, count)] <= x)) - 1;
}

__device__ inline void write_row(const TableArgs &t, int64_t i, int n, int pos, int block) {
    t.slot_map[i] = block < 0 ? -1 : (int64_t(block) << t.block_size_log2) + (pos & ((1 << t.block_size_log2) - 1));
    if (t.positions) t.positions[i] = pos;
    if (t.row_seqs) t.row_seqs[i] = n;
}

// All sequences in one pass.  A wavefront takes 64 * U rows at a time.
template <int THREADS, int ITEMS, int U>
__global__ __launch_bounds__(THREADS) void block_tables_extend_kernel(TableArgs t) {
    constexpr int WAVES = THREADS / 64, kRowsAtOnce = 64 * U;
    __shared__ Pass<THREADS, ITEMS> s;
    Carries c = {0, 0, 0, 0};
    if (t.num_seqs > 0) scan_pass(t, 0, c, s, blockIdx.x == 0);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        t.q_start[t.num_seqs] = int(c.dealt);
        if (t.taken) *t.taken = int(c.taken);
    }
    __syncthreads();
    // A wavefront takes table entries and rows that lie together: the sequences they can belong to are found once for all of them.
    const int lane = threadIdx.x & 63, wave = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = gridDim.x * WAVES;
    auto range = [&](const uint32_t *starts, uint32_t from, uint32_t to, int *first, int *end) __attribute__((always_inline)) {
        *first = place_of_all(starts, t.num_seqs, from);
        *end = starts[*first + 1] > to ? *first + 1 : place_of_all(starts, t.num_seqs, to) + 1;
    };
    for (int64_t i0 = int64_t(wave) * kRowsAtOnce; i0 < t.max_rows; i0 += int64_t(waves) * kRowsAtOnce) {
        int first = 0, end = 0;
        if (i0 < c.dealt) range(s.rows, uint32_t(i0), uint32_t(min(i0 + kRowsAtOnce, int64_t(c.dealt)) - 1), &first, &end);
        int n_of[U], seq[U], pos[U], block[U];
#pragma unroll
        for (int u = 0; u < U; ++u) n_of[u] = first;
        for (int left = end - first; left > 1;) {  // the largest with rows[n] <= i, for all U rows of a lane at once
            const int half = left >> 1;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (s.rows[n_of[u] + half] <= uint32_t(i0) + 64 * u + lane) n_of[u] += half;
            left -= half;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + 64 * u + lane;
            seq[u] = pos[u] = block[u] = -1;
            if (i < c.dealt) {
                const int n = n_of[u], held = s.held[n];
                seq[u] = n;
                pos[u] = s.ctx[n] + int(i - s.rows[n]);
                const int b = pos[u] >> t.block_size_log2;
                block[u] = b < held ? t.block_tables[int64_t(n) * t.max_blocks_per_seq + b] : t.free_blocks[s.first[n] + (b - held)];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + 64 * u + lane < t.max_rows) write_row(t, i0 + 64 * u + lane, seq[u], pos[u], block[u]);
    }
    for (int64_t e0 = int64_t(wave) * 64; e0 < c.taken; e0 += int64_t(waves) * 64) {
        int first, end;
        range(s.first, uint32_t(e0), uint32_t(min(e0 + 64, int64_t(c.taken)) - 1), &first, &end);
        const int64_t e = e0 + lane;
        if (e < c.taken) {
            const int n = place_of(s.first, first, end, uint32_t(e));
            t.block_tables[int64_t(n) * t.max_blocks_per_seq + s.held[n] + (e - s.first[n])] = t.free_blocks[e];
        }
    }
}

// More sequences: one workgroup sums and fills the tables, a second launch fills the maps.
constexpr int kSumThreads = 1024;
using SumPass = Pass<kSumThreads, 2>;
__global__ __launch_bounds__(kSumThreads) void block_tables_sum_kernel(TableArgs t) {
    __shared__ SumPass s;
    Carries c = {0, 0, 0, 0};
    for (int base = 0; base < t.num_seqs; base += SumPass::kSeqs) {
        const uint32_t taken = c.taken;
        scan_pass(t, base, c, s, true);
        __syncthreads();
        for (uint32_t e = taken + threadIdx.x; e < c.taken; e += kSumThreads) {
            const int i = place_of(s.first, 0, min(SumPass::kSeqs, t.num_seqs - base), e);
            t.block_tables[int64_t(base + i) * t.max_blocks_per_seq + s.held[i] + (e - s.first[i])] = t.free_blocks[e];
        }
        __syncthreads();  // the next pass writes what is read here
    }
    if (threadIdx.x == 0) {
        t.q_start[t.num_seqs] = int(c.dealt);
        if (t.taken) *t.taken = int(c.taken);
    }
}
__global__ __launch_bounds__(kThreads) void block_tables_map_kernel(TableArgs t) {
    const int64_t stride = int64_t(gridDim.x) * kThreads;
    const uint32_t *starts = reinterpret_cast<const uint32_t *>(t.q_start);
    const uint32_t dealt = starts[t.num_seqs];
    for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < t.max_rows; i += stride) {
        if (i >= dealt) {
            write_row(t, i, -1, -1, -1);
            continue;
        }
        const int n = place_of(starts, 0, t.num_seqs, uint32_t(i));
        const int pos = t.context_lens[n] + int(i - starts[n]);
        write_row(t, i, n, pos, t.block_tables[int64_t(n) * t.max_blocks_per_seq + (pos >> t.block_size_log2)]);
    }
}

}  // namespace

hipError_t launch_block_tables_extend(const TableArgs &t, hipStream_t stream) {
    auto grid_of = [&](int64_t share, int most) { return dim3(unsigned(std::min<int64_t>(std::max<int64_t>((t.max_rows + share - 1) / share, 1), most))); };
    if (t.num_seqs <= SumPass::kSeqs) {
        // Workgroups that sum many sequences are large and no more than the compute units: they all read the same lengths, which is what
        // four times as many of a quarter the size spent their time on (1500 sequences 6 to 12 us of 18).
        // A wavefront takes 64 rows where the workgroups of the launch have enough of them, else 256 at a time.
#define KVC_EXTEND(THREADS, ITEMS, GROUPS)                                                                                              \
    do {                                                                                                                                \
        if (t.max_rows <= int64_t(GROUPS) * THREADS / 4)                                                                                \
            block_tables_extend_kernel<THREADS, ITEMS, 1><<<grid_of(THREADS, GROUPS), dim3(THREADS), 0, stream>>>(t);                   \
        else                                                                                                                            \
            block_tables_extend_kernel<THREADS, ITEMS, 4><<<grid_of(4 * THREADS, GROUPS), dim3(THREADS), 0, stream>>>(t);               \
    } while (0)
        if (t.num_seqs <= kThreads) KVC_EXTEND(kThreads, 1, 4 * kNumCUs);
        else if (t.num_seqs <= kSumThreads) KVC_EXTEND(kSumThreads, 1, kNumCUs);
        else KVC_EXTEND(kSumThreads, 2, kNumCUs);
#undef KVC_EXTEND
        return hipGetLastError();
    }
    block_tables_sum_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(t);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || t.max_rows == 0) return e;
    block_tables_map_kernel<<<grid_of(4 * kThreads, 4 * kNumCUs), dim3(kThreads), 0, stream>>>(t);
    return hipGetLastError();
}

}  // namespace kvc
