// kvc_block_tables_extend: blocks from a free list for the new tokens of every sequence, and the slot, position and sequence of
// every new token (gfx950).  With need_n the blocks that sequence n lacks, new_n its new tokens,
//
//   F_n = sum_{i<n} need_i,  R_n = sum_{i<n} new_i;   granted: need_n = 0 or F_n + need_n <= num_free, and R_n + new_n <= max_rows
//   Q_n = new_n if granted, else 0;   row sum_{i<n} Q_i + j of the maps is token ctx_n + j
//
// A refusal for want of blocks refuses everybody behind who needs one, and one for want of rows everybody behind who brings any
// (the sums count refused sequences too), so the blocks dealt out are the front of the free list, in order.
#include "kvc_internal.h"
#include "pa_lanes.h"

namespace kvc {

namespace {

constexpr int kItems = 4;                       // sequences per thread and pass
constexpr int kPass = kThreads * kItems;        // sequences per pass

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
template <class Op>
__device__ inline void scan_group(uint32_t &a, uint32_t &b, uint32_t &carry_a, uint32_t &carry_b, uint32_t (&s_sums)[2][kWaves], Op op) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint32_t ia = scan_wave(a, op), ib = scan_wave(b, op);
    if (lane == 63) {
        s_sums[0][wave] = ia;
        s_sums[1][wave] = ib;
    }
    __syncthreads();
    uint32_t ba = carry_a, bb = carry_b;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) {
            a = op(ba, uint32_t(__shfl_up(int(ia), 1)) * (lane > 0));
            b = op(bb, uint32_t(__shfl_up(int(ib), 1)) * (lane > 0));
        }
        ba = op(ba, s_sums[0][w]);
        bb = op(bb, s_sums[1][w]);
    }
    carry_a = ba;
    carry_b = bb;
    __syncthreads();
}

__device__ inline int blocks_held(const TableArgs &t, int n, int ctx) {
    return t.held_blocks ? t.held_blocks[n] : (ctx + (1 << t.block_size_log2) - 1) >> t.block_size_log2;
}

// One pass over sequences base .. base + kPass - 1.  Leaves in s_rows / s_first the first row and the first of the dealt-out blocks of each
// (one more entry than sequences), and writes what is known per sequence where `write`.
struct Carries { uint32_t need, rows, dealt, taken; };
__device__ inline void scan_pass(const TableArgs &t, int base, Carries &c, uint32_t (&s_sums)[2][kWaves], uint32_t *s_rows, uint32_t *s_first,
                                 bool write) {
    const int first = base + threadIdx.x * kItems;
    int ctx[kItems], held[kItems];
    uint32_t need[kItems], rows[kItems], sum_need = 0, sum_rows = 0;
    auto saturated = [](uint32_t a, uint32_t b) { return add_saturated(a, b); };
    auto plain = [](uint32_t a, uint32_t b) { return a + b; };
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int n = first + k;
        ctx[k] = held[k] = 0;
        need[k] = rows[k] = 0;
        if (n < t.num_seqs) {
            ctx[k] = t.context_lens[n];
            const int fresh = t.new_lens[n];
            held[k] = blocks_held(t, n, ctx[k]);
            const int tokens = t.max_blocks_per_seq << t.block_size_log2;  // at most 2^30
            if (fresh > 0 && ctx[k] >= 0 && ctx[k] <= tokens && fresh <= tokens - ctx[k] && held[k] >= 0 && held[k] <= t.max_blocks_per_seq) {
                rows[k] = fresh;
                need[k] = max(0, ((ctx[k] + fresh - 1) >> t.block_size_log2) + 1 - held[k]);
            }
        }
        sum_need = add_saturated(sum_need, need[k]);
        sum_rows = add_saturated(sum_rows, rows[k]);
    }
    scan_group(sum_need, sum_rows, c.need, c.rows, s_sums, saturated);
    uint32_t sum_dealt = 0, sum_taken = 0;
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        sum_need = add_saturated(sum_need, need[k]);
        sum_rows = add_saturated(sum_rows, rows[k]);
        if (!((need[k] == 0 || sum_need <= uint32_t(t.num_free)) && sum_rows <= uint32_t(t.max_rows))) need[k] = rows[k] = 0;
        sum_dealt += rows[k];
        sum_taken += need[k];
    }
    scan_group(sum_dealt, sum_taken, c.dealt, c.taken, s_sums, plain);
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int n = first + k;
        if (n < t.num_seqs) {
            s_rows[n - base] = sum_dealt;
            s_first[n - base] = sum_taken;
            if (write) {
                t.q_start[n] = int(sum_dealt);
                t.context_lens_out[n] = ctx[k] + int(rows[k]);
                if (t.held_blocks_out) t.held_blocks_out[n] = held[k] + int(need[k]);
            }
            sum_dealt += rows[k];
            sum_taken += need[k];
        }
    }
    const int count = min(kPass, t.num_seqs - base);
    if (threadIdx.x == 0) {
        s_rows[count] = c.dealt;
        s_first[count] = c.taken;
    }
}

// Largest i < count with s[i] <= x, for s[0] <= x < s[count].
__device__ inline int place_of(const uint32_t *s, int count, uint32_t x) {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ inline void write_row(const TableArgs &t, int64_t i, int n, int pos, int block) {
    t.slot_map[i] = block < 0 ? -1 : (int64_t(block) << t.block_size_log2) + (pos & ((1 << t.block_size_log2) - 1));
    if (t.positions) t.positions[i] = pos;
    if (t.row_seqs) t.row_seqs[i] = n;
}

// Up to kWholeSeqs sequences: every workgroup sums for itself and takes its share of the table entries and rows.
constexpr int kWholeSeqs = 4 * kPass;
__global__ __launch_bounds__(kThreads) void block_tables_extend_kernel(TableArgs t) {
    __shared__ uint32_t s_rows[kWholeSeqs + 1], s_first[kWholeSeqs + 1], s_sums[2][kWaves];
    Carries c = {0, 0, 0, 0};
    for (int base = 0; base < t.num_seqs; base += kPass) scan_pass(t, base, c, s_sums, s_rows + base, s_first + base, blockIdx.x == 0);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        t.q_start[t.num_seqs] = int(c.dealt);
        if (t.taken) *t.taken = int(c.taken);
    }
    __syncthreads();
    const int stride = gridDim.x * kThreads, me = blockIdx.x * kThreads + threadIdx.x;
    for (int64_t e = me; e < c.taken; e += stride) {
        const int n = place_of(s_first, t.num_seqs, uint32_t(e));
        t.block_tables[int64_t(n) * t.max_blocks_per_seq + blocks_held(t, n, t.context_lens[n]) + (e - s_first[n])] = t.free_blocks[e];
    }
    for (int64_t i = me; i < t.max_rows; i += stride) {
        if (i >= c.dealt) {
            write_row(t, i, -1, -1, -1);
            continue;
        }
        const int n = place_of(s_rows, t.num_seqs, uint32_t(i));
        const int ctx = t.context_lens[n], held = blocks_held(t, n, ctx);
        const int pos = ctx + int(i - s_rows[n]), b = pos >> t.block_size_log2;
        write_row(t, i, n, pos, b < held ? t.block_tables[int64_t(n) * t.max_blocks_per_seq + b] : t.free_blocks[s_first[n] + (b - held)]);
    }
}

// More sequences: one workgroup sums and fills the tables, a second launch fills the maps.
__global__ __launch_bounds__(kThreads) void block_tables_sum_kernel(TableArgs t) {
    __shared__ uint32_t s_rows[kPass + 1], s_first[kPass + 1], s_sums[2][kWaves];
    Carries c = {0, 0, 0, 0};
    for (int base = 0; base < t.num_seqs; base += kPass) {
        const uint32_t taken = c.taken;
        scan_pass(t, base, c, s_sums, s_rows, s_first, true);
        __syncthreads();
        for (uint32_t e = taken + threadIdx.x; e < c.taken; e += kThreads) {
            const int i = place_of(s_first, min(kPass, t.num_seqs - base), e), n = base + i;
            t.block_tables[int64_t(n) * t.max_blocks_per_seq + blocks_held(t, n, t.context_lens[n]) + (e - s_first[i])] = t.free_blocks[e];
        }
        __syncthreads();  // the next pass writes s_rows and s_first
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
        const int n = place_of(starts, t.num_seqs, uint32_t(i));
        const int pos = t.context_lens[n] + int(i - starts[n]);
        write_row(t, i, n, pos, t.block_tables[int64_t(n) * t.max_blocks_per_seq + (pos >> t.block_size_log2)]);
    }
}

}  // namespace

hipError_t launch_block_tables_extend(const TableArgs &t, hipStream_t stream) {
    const int64_t share = 4 * kThreads;
    const int grid = int(std::min<int64_t>(std::max<int64_t>((t.max_rows + share - 1) / share, 1), 4 * kNumCUs));
    if (t.num_seqs <= kWholeSeqs) {
        block_tables_extend_kernel<<<dim3(grid), dim3(kThreads), 0, stream>>>(t);
        return hipGetLastError();
    }
    block_tables_sum_kernel<<<dim3(1), dim3(kThreads), 0, stream>>>(t);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || t.max_rows == 0) return e;
    block_tables_map_kernel<<<dim3(grid), dim3(kThreads), 0, stream>>>(t);
    return hipGetLastError();
}

}  // namespace kvc
