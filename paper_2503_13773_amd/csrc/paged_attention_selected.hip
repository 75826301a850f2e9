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
//
// Bound: memory in a decode batch (32 long documents, 64 / 8 heads of 128 in bf16, 128 blocks of 16 each, 269 MB: 45.6 us = 5.9 TB/s; a
// copy of 2 GiB moves 5.0 TB/s here); launch and the join for a single row (9.4 us); LDS and the issue of instructions for chunks, whose rows
// read the same blocks again from L2 (1000 rows, 32 / 8 heads of 64, 1024 tokens each: 91-93 us, 2.1 GB through LDS).
#include "cache_rows.h"
#include "kvc_internal.h"
#include "lds_loads.h"
#include "pa_partials.h"

namespace kvc {

namespace {

using namespace mfma;

constexpr int kWindow = 512;  // list entries whose places are held in LDS at a time (vector ALUs)

// ---- bf16 on the matrix cores, up to 16 heads of a KV head (blocks of 4 tokens and more)
//
// A tile is 32 tokens.  With lane = 16 * quad + r:
//   S[token][head]   = K . Q^T    per 16 tokens HD / 32 v_mfma_f32_16x16x32_bf16: lane holds scores of tokens 16 h + 4 quad + i of head r
//   O^T[dim][head]  += V^T . P^T  per 16 dims one such product over the 32 tokens, depth slot 8 quad + 4 h + i = token 16 h + 4 quad + i,
//                                 which is how the weights lie already; lane holds dims 16 b + 4 quad + i of head r
// K and V rows go straight from the cache into LDS, 16 bytes a lane, into a stage that the wavefront has for itself: no barrier, and a
// stage is filled again as soon as its operands are in registers, K of the next tile under the softmax of this one.  Which 16 bytes a
// lane asks for makes the image free of bank conflicts: chunk c of K's row R at c ^ (R / 2 % 8) (heads of 64) or c ^ (R % 16); 32-byte
// granule g of V's row R, which transposing reads take 16 rows at a time, at (g + R / 2) % 4 or (g + R) % 8.
//
// A lane's own loads in the operands' layout touch 64 lines per instruction, one per lane, and the vector cache takes one a cycle: 1000
// rows of chunks, 32 / 8 heads of 64, 1024 tokens each: 172 us so, 387 cycles of it per tile and compute unit; through LDS 93 us.

template <int HD>
struct Stage {
    static constexpr int kTokens = 32, kRowBytes = HD * 2, kBytes = kTokens * kRowBytes;  // of K, and of V
    static constexpr int kLoads = kBytes / 1024, kRows = 1024 / kRowBytes;                // instructions for each, rows of one
    static constexpr int kChunks = kRowBytes / 16;
    __device__ static int k_place(int row, int chunk) { return row * kRowBytes + ((chunk ^ (HD == 64 ? (row >> 1) & 7 : row & 15)) << 4); }
    __device__ static int v_place(int row, int granule) {
        return row * kRowBytes + (HD == 64 ? (granule + (row >> 1)) & 3 : (granule + row) & 7) * 32;
    }
    // where in its row the lane of a load finds what belongs at 16 bytes * lane of the kilobyte that load i fills
    __device__ static int k_source(int lane, int i) {
        const int row = i * kRows + lane / kChunks;
        return ((lane % kChunks) ^ (HD == 64 ? (row >> 1) & 7 : row & 15)) << 4;
    }
    __device__ static int v_source(int lane, int i) {
        const int row = i * kRows + lane / kChunks, place = lane % kChunks;
        return (((place >> 1) - (HD == 64 ? row >> 1 : row)) & (HD == 64 ? 3 : 7)) * 32 + (place & 1) * 16;
    }
};

// Softmax state of up to 16 heads in one wavefront: lane (quad, r) holds dims 16 b + 4 quad + i of head r in acc[b][i].
template <int HD>
struct State {
    floatx4 acc[HD / 16];
    float m, l;  // largest scaled score so far (base 2); sum of the weights, of this lane's tokens until finish()
    __device__ void reset() {
#pragma unroll
        for (int b = 0; b < HD / 16; ++b) acc[b] = floatx4{0.f, 0.f, 0.f, 0.f};
        m = -FLT_MAX;  // not -inf: scores of -inf weigh nothing then, instead of -inf - -inf
        l = 0.f;
    }
    __device__ void finish() { l = lanes::sum_over_rows(l); }
};

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
// one unit; 64 >> units_log2 tiles are known at a time.  UNIFORM: the rows of a load lie in one unit (blocks of 8 tokens and more at
// head_dim 64, all at 128).  AGAIN: rows near this one read the same blocks, so loads leave them in L2 (else they
// pass through it).
// `stage`: K and V of a tile, this wavefront's own.
template <int HD, bool UNIFORM, bool AGAIN>
__device__ inline bool attend_list(State<HD> &st, const bf16x8 (&qb)[HD / 32], const uint16_t *__restrict__ k_cache, const uint16_t *__restrict__ v_cache,
                                   const ListOf &list, float scale_log2e, int tile0, int tiles, int first, int step, unsigned char *stage) {
    using G = Stage<HD>;
    typedef short v4i16 __attribute__((ext_vector_type(4)));
    typedef v4i16 __attribute__((address_space(3))) * lds_v4i16_ptr;
    constexpr int kLoads = G::kLoads, kRows = G::kRows;
    const int lane = threadIdx.x & 63, quad = lane >> 4, r = lane & 15;
    const int unit_log2 = list.unit_log2, units_log2 = 5 - unit_log2;
    const uint32_t unit_bytes = uint32_t(G::kRowBytes) << unit_log2, in_rows = uint32_t(lane / G::kChunks) * G::kRowBytes;
    unsigned char *const s_k = stage, *const s_v = stage + G::kBytes;
    const uint32_t lds_k = uniform(int(uint32_t(reinterpret_cast<uintptr_t>(s_k)))), lds_v = lds_k + G::kBytes;
    const unsigned char *const k_bytes = reinterpret_cast<const unsigned char *>(k_cache), *const v_bytes = reinterpret_cast<const unsigned char *>(v_cache);
    bool any = false;
    for (int from = first; from < tiles; from += step << (6 - units_log2)) {
        const int mine = from + step * (lane >> units_log2);
        int2 e = {0, 0};
        if (mine < tiles) e = list.unit(((tile0 + mine) << units_log2) + (lane & ((1 << units_log2) - 1)));
        const uint64_t there = __ballot(e.y > 0);
        if (there == 0) continue;
        any = true;
        const int count = ((63 - __builtin_clzll(there)) >> units_log2) + 1;
        auto issue = [&](const unsigned char *cache, uint32_t lds, int i, auto source) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int row = j * kRows;  // of the tile, the load's first
                if constexpr (UNIFORM) {
                    const uint32_t unit = __builtin_amdgcn_readlane(e.x, (i << units_log2) + (row >> unit_log2));
                    load_to_lds<AGAIN>(cache + uint64_t(unit) * unit_bytes + uint32_t(row & ((1 << unit_log2) - 1)) * G::kRowBytes, in_rows + source(lane, j),
                                       lds + 1024 * j);
                } else {
                    const int mine = row + lane / G::kChunks;
                    const uint32_t unit = __shfl(e.x, (i << units_log2) + (mine >> unit_log2));
                    load_to_lds<AGAIN>(cache + uint64_t(unit) * unit_bytes + uint32_t(mine & ((1 << unit_log2) - 1)) * G::kRowBytes + source(lane, j), lds + 1024 * j);
                }
            }
        };
        auto issue_k = [&](int i) __attribute__((always_inline)) { issue(k_bytes, lds_k, i, G::k_source); };
        auto issue_v = [&](int i) __attribute__((always_inline)) { issue(v_bytes, lds_v, i, G::v_source); };
        // Q is waited for here: inside the loop the wait would be for the loads of tiles too
#pragma unroll
        for (int j = 0; j < HD / 32; ++j) asm volatile("" ::"v"(qb[j]));
        issue_k(0);
        issue_v(0);
        for (int i = 0; i < count; ++i) {
            const bool more = i + 1 < count;
            // how many of this lane's tokens 16 h + 4 quad .. + 3 count; full: all of every lane's
            int limit[2];
            bool full = true;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int token = 16 * h + 4 * quad;
                if (unit_log2 >= 4) {
                    const int counts = __builtin_amdgcn_readlane(e.y, (i << units_log2) + ((16 * h) >> unit_log2)) - ((16 * h) & ((1 << unit_log2) - 1));
                    full &= counts >= 16;
                    limit[h] = min(max(counts - 4 * quad, 0), 4);
                } else {
                    limit[h] = min(max(__shfl(e.y, (i << units_log2) + (token >> unit_log2)) - (token & ((1 << unit_log2) - 1)), 0), 4);
                    full &= __ballot(limit[h] < 4) == 0;
                }
            }
            wait_for_loads<kLoads>();  // all but V's
            bf16x8 ka[2][HD / 32];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < HD / 32; ++j) ka[h][j] = *reinterpret_cast<const bf16x8 *>(s_k + G::k_place(16 * h + r, 4 * j + quad));
            wait_for_lds();
            if (more) issue_k(i + 1);
            float sv[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < HD / 32; ++j) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[h][j], qb[j], s, 0, 0, 0);
#pragma unroll
                for (int t = 0; t < 4; ++t) sv[4 * h + t] = s[t] * scale_log2e;
            }
            if (!full) {
#pragma unroll
                for (int t = 0; t < 8; ++t)
                    if ((t & 3) >= limit[t >> 2]) sv[t] = -INFINITY;
            }
            const float mx = lanes::max_over_rows(fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7]))));
            const float m_new = fmaxf(st.m, mx), alpha = __builtin_amdgcn_exp2f(st.m - m_new);
            st.m = m_new;
            // Weights go into the product as a sum of two bf16 values (upper bits and rounded rest, 2^-16 relative), the sum takes them in fp32.
            // The upper part is cut off and the rest made positive by 2^-23 of the weight (a factor that all weights share), so that an infinity in V
            // keeps its sign, which a rest of 0 or of the other sign would turn into NaN.
            float sum = 0.f;
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const float p0 = __builtin_amdgcn_exp2f(sv[2 * t] - m_new), p1 = __builtin_amdgcn_exp2f(sv[2 * t + 1] - m_new);
                sum += p0 + p1;
                const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
                hi[t] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
                lo[t] = pack_bf16(__builtin_fmaf(p0, 1.f + FLT_EPSILON, -__uint_as_float(u0 & 0xffff0000u)),
                                  __builtin_fmaf(p1, 1.f + FLT_EPSILON, -__uint_as_float(u1 & 0xffff0000u)));
            }
            st.l = fmaf(st.l, alpha, sum);
            if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
                for (int b = 0; b < HD / 16; ++b) st.acc[b] *= alpha;
            }
            const bf16x8 ph = __builtin_bit_cast(bf16x8, uint4{hi[0], hi[1], hi[2], hi[3]}), pl = __builtin_bit_cast(bf16x8, uint4{lo[0], lo[1], lo[2], lo[3]});
            if (more) wait_for_loads<kLoads>(); else wait_for_loads<0>();  // all but K of the next tile
            uint2 va[HD / 16][2];  // lanes 4 k .. 4 k + 3 of a quad point at 16 dims of its token k and get a dim each of all four
#pragma unroll
            for (int b = 0; b < HD / 16; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    va[b][h] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(s_v + G::v_place(16 * h + 4 * quad + (r >> 2), b) + 8 * (r & 3))));
            wait_for_lds();
            if (more) issue_v(i + 1);
            if (!full) {  // what does not count may hold anything
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t x = (limit[h] > 0 ? 0xffffu : 0u) | (limit[h] > 1 ? 0xffff0000u : 0u), y = (limit[h] > 2 ? 0xffffu : 0u) | (limit[h] > 3 ? 0xffff0000u : 0u);
#pragma unroll
                    for (int b = 0; b < HD / 16; ++b) va[b][h] = uint2{va[b][h].x & x, va[b][h].y & y};
                }
            }
#pragma unroll
            for (int b = 0; b < HD / 16; ++b) {
                const bf16x8 v = __builtin_bit_cast(bf16x8, uint4{va[b][0].x, va[b][0].y, va[b][1].x, va[b][1].y});
                st.acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, ph, st.acc[b], 0, 0, 0);
                st.acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pl, st.acc[b], 0, 0, 0);
            }
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
    __shared__ __attribute__((aligned(1024))) unsigned char s_stage[kWaves][2 * Stage<HD>::kBytes];
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, quad = lane >> 4, r = lane & 15;
    const int group = blockIdx.x / a.num_kv_heads, row = group * kWaves + wave;
    if (row >= a.total_q) return;
    const Unit u(a, q_start, context_lens, row, blockIdx.x - group * a.num_kv_heads, blockIdx.y);
    if (!u.there) return;
    uint16_t *dst = out + (int64_t(row) * a.num_q_heads + u.head0 + r) * HD + 4 * quad;
    State<HD> st;
    st.reset();
    bool any = false;
    if (u.pos >= 0) {
        bf16x8 qb[HD / 32];
        load_q_operand(qb, q + (int64_t(row) * a.num_q_heads + u.head0 + (r < u.heads ? r : 0)) * HD, quad, r < u.heads);
        any = attend_list<HD, UNIFORM, true>(st, qb, k_cache, v_cache, list_of(a, u, selected, block_tables), a.scale_log2e, 0, a.tiles, 0, 1,
                                              s_stage[wave]);
    }
    st.finish();
    if (r >= u.heads) return;
    const float inv = 1.0f / st.l;
#pragma unroll
    for (int b = 0; b < HD / 16; ++b) {
        const uint2 w = {pack_bf16(st.acc[b][0] * inv, st.acc[b][1] * inv), pack_bf16(st.acc[b][2] * inv, st.acc[b][3] * inv)};
        *reinterpret_cast<uint2 *>(dst + 16 * b) = any ? w : uint2{0u, 0u};
    }
}

// A workgroup per part of a unit's list; blockIdx.x = KV head + KV heads * row, blockIdx.y = chunk of heads, blockIdx.z = part.
template <int HD, bool UNIFORM, bool AGAIN, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void pa_selected_mfma_kernel(
    const uint16_t *__restrict__ q, const uint16_t *__restrict__ k_cache, const uint16_t *__restrict__ v_cache, const int32_t *__restrict__ block_tables,
    const int32_t *__restrict__ context_lens, const int32_t *__restrict__ q_start, const int32_t *__restrict__ selected, uint16_t *__restrict__ out,
    Workspace ws, SelectedArgs a) {
    // tiles while the wavefronts stream, what they and the parts exchange afterwards (a state is HD / 4 vectors of 16 heads: as large as a stage)
    __shared__ __attribute__((aligned(1024))) unsigned char s_stage[WAVES][2 * Stage<HD>::kBytes];
    float4 (*const s_acc)[16 * HD / 4] = reinterpret_cast<float4 (*)[16 * HD / 4]>(s_stage);
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
    bf16x8 qb[HD / 32];
    load_q_operand(qb, q + (int64_t(row) * a.num_q_heads + u.head0 + (r < u.heads ? r : 0)) * HD, quad, r < u.heads);
    State<HD> st;
    st.reset();
    const int tile0 = part * a.tiles_per_part;
    const bool any = attend_list<HD, UNIFORM, AGAIN>(st, qb, k_cache, v_cache, list_of(a, u, selected, block_tables), a.scale_log2e, tile0,
                                              min(a.tiles_per_part, a.tiles - tile0), wave, WAVES, s_stage[wave]);
    st.finish();
    // a wavefront or part without a token says so with a maximum of -inf (with tokens it is -FLT_MAX at least)
    __syncthreads();  // the stages are no longer needed
#pragma unroll
    for (int b = 0; b < HD / 16; ++b) s_acc[wave][(4 * b + quad) * 16 + r] = __builtin_bit_cast(float4, st.acc[b]);
    if (quad == 0) s_ml[wave][r] = float2{any ? st.m : -INFINITY, st.l};
    __syncthreads();
    const int vecs = u.heads * HD / 4;
    const int64_t slot0 = (int64_t(blockIdx.x) * gridDim.y + blockIdx.y) * parts;
    const uint32_t slots = uint32_t(gridDim.x * gridDim.y) * parts, slot_vecs = 16 * HD / 4;
    const __amdgpu_buffer_rsrc_t acc_buf = raw_buffer(ws.acc, parts > 1 ? slots * slot_vecs * 16u : 0u), ml_buf = raw_buffer(ws.ml, parts > 1 ? slots * 16u * 8u : 0u);
    // vector f of the output: dims 4 d .. 4 d + 3 of a head
    auto place = [&](int f, int *head) __attribute__((always_inline)) {
        *head = f / (HD / 4);
        return f % (HD / 4) * 16 + *head;
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
    int32_t *const counter = ws.cnt + (blockIdx.x * gridDim.y + blockIdx.y) * a.counter_step;
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
// op over the lanes that hold the same dims of the wavefront's tokens, LR apart.
template <int LR, class Op>
__device__ inline float over_tokens(float x, Op op) {
    if constexpr (LR <= 8) x = op(x, lanes::permuted<lanes::kRor8>(x));
    if constexpr (LR <= 16) {
        const lanes::Pair<float> a = lanes::pair_of<16>(x);
        x = op(a.first, a.second);
    }
    const lanes::Pair<float> b = lanes::pair_of<32>(x);
    return op(b.first, b.second);
}
// exp(d) for d <= 0, as a power of two: the rounding of the product moves a weight by 2^-24 of its own exponent, 3e-8 of the largest weight
// at most.  An expf is fifteen instructions, and the lanes of a token all compute the same one.
__device__ inline float weight_of(float d) { return __builtin_amdgcn_exp2f(d * 1.44269504088896340736f); }
__device__ inline void store_device(float *p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline float load_device(const float *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Grid as above, the chunk of heads HEADS of them.
template <class T, int D, int HEADS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void pa_selected_valu_kernel(const T *__restrict__ q, const T *__restrict__ k_cache, const T *__restrict__ v_cache,
                                                                    const int32_t *__restrict__ block_tables, const int32_t *__restrict__ context_lens,
                                                                    const int32_t *__restrict__ q_start, const int32_t *__restrict__ selected,
                                                                    T *__restrict__ out, Workspace ws, SelectedArgs a) {
    constexpr int N = Vec<T>::N, LR = D / N, TOKENS = 64 / LR, U = 4;
    __shared__ int2 s_entry[kWindow];  // pool index of a block, tokens of it that count
    __shared__ int s_last;
    __shared__ float s_m[kMaxSelectedParts][HEADS], s_l[kMaxSelectedParts][HEADS], s_acc[WAVES][HEADS][D];  // of the wavefronts; m, l of the parts
    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, c = lane % LR, tg = lane / LR;
    const int row = blockIdx.x / a.num_kv_heads, parts = a.parts, part = blockIdx.z;
    const Unit u(a, q_start, context_lens, row, blockIdx.x - row * a.num_kv_heads, blockIdx.y);
    if (!u.there) return;
    T *dst = out + (int64_t(row) * a.num_q_heads + u.head0) * D;
    if (u.pos < 0) {
        if (part == 0)
            for (int i = tid; i < HEADS * D; i += (64 * WAVES)) dst[i] = T(0);
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
        for (int i = tid; i < min(kWindow, end - e0); i += (64 * WAVES)) {
            const int b = list[e0 + i];
            const int named = table[min(max(b, 0), a.max_blocks_per_seq - 1)];  // without waiting for the position
            const bool there = b >= 0 && b <= own;
            s_entry[i] = int2{there ? named : own_block, there ? min(u.pos + 1 - (b << bs_log2), 1 << bs_log2) : 0};
            if (there) last = i + 1;
        }
        if (last > 0) atomicMax(&s_last, last);
        __syncthreads();
        const int tokens = s_last << bs_log2;
        any |= tokens > 0;
        for (int t0 = wave * TOKENS * U; t0 < tokens; t0 += WAVES * TOKENS * U) {
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
                const float alpha = weight_of(m[h] - top);
                m[h] = top;
                l[h] *= alpha;
#pragma unroll
                for (int j = 0; j < N; ++j) acc[h][j] *= alpha;
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const float p = weight_of(s[i] - top);
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
        const float top = over_tokens<LR>(m[h], [](float u, float v) { return fmaxf(u, v); }), mine = weight_of(m[h] - top);
        auto add = [](float u, float v) { return u + v; };
        l[h] = over_tokens<LR>(l[h] * mine, add);
#pragma unroll
        for (int i = 0; i < N; ++i) acc[h][i] = over_tokens<LR>(acc[h][i] * mine, add);
        m[h] = top;
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
    for (int f = tid; f < HEADS * D; f += (64 * WAVES)) {
        const int h = f / D, d = f % D;
        float M = -FLT_MAX, L = 0.f, A = 0.f;
        for (int w = 0; w < WAVES; ++w) M = fmaxf(M, s_m[w][h]);
        for (int w = 0; w < WAVES; ++w) {
            const float wgt = weight_of(s_m[w][h] - M);
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
    if (tid == 0) s_last = __hip_atomic_fetch_add(ws.cnt + unit * a.counter_step, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
    __syncthreads();
    if (!s_last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    if (tid == 0) __hip_atomic_store(ws.cnt + unit * a.counter_step, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int i = tid; i < parts * HEADS; i += (64 * WAVES)) {
        s_m[i / HEADS][i % HEADS] = load_device(ws.ml + (slot0 * HEADS + i) * 2);
        s_l[i / HEADS][i % HEADS] = load_device(ws.ml + (slot0 * HEADS + i) * 2 + 1);
    }
    __syncthreads();
    for (int f = tid; f < HEADS * D; f += (64 * WAVES)) {
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
                const float wgt = s_m[p0 + j][h] == -INFINITY ? 0.f : weight_of(s_m[p0 + j][h] - M);
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
        const bool uniform = head_dim == 128 || a.unit_log2 >= 3;  // the rows of a load are in one unit
        if (a.wave_per_unit) {
            const dim3 waves(unsigned((a.total_q + kWaves - 1) / kWaves) * unsigned(a.num_kv_heads), chunks);
            auto launch = [&](auto kernel) { kernel<<<waves, dim3(kThreads), 0, stream>>>(qp, kp, vp, block_tables, context_lens, q_start, selected, op, a); };
            if (head_dim == 64) uniform ? launch(pa_selected_wave_kernel<64, true>) : launch(pa_selected_wave_kernel<64, false>);
            else launch(pa_selected_wave_kernel<128, true>);
        } else {
            auto launch = [&](auto kernel) {
                kernel<<<grid, dim3(64 * a.waves), 0, stream>>>(qp, kp, vp, block_tables, context_lens, q_start, selected, op, ws, a);
            };
#define KVC_PARTS(HD, UNIFORM)                                                                                                     \
    do {                                                                                                                           \
        if (a.waves == 8) a.again ? launch(pa_selected_mfma_kernel<HD, UNIFORM, true, 8>) : launch(pa_selected_mfma_kernel<HD, UNIFORM, false, 8>); \
        else a.again ? launch(pa_selected_mfma_kernel<HD, UNIFORM, true, 4>) : launch(pa_selected_mfma_kernel<HD, UNIFORM, false, 4>);               \
    } while (0)
            if (head_dim == 64) { if (uniform) KVC_PARTS(64, true); else KVC_PARTS(64, false); }
            else KVC_PARTS(128, true);
#undef KVC_PARTS
        }
        return hipGetLastError();
    }
    auto launch = [&](auto kernel, auto type) {
        using T = decltype(type);
        kernel<<<grid, dim3(64 * a.waves), 0, stream>>>(static_cast<const T *>(q), static_cast<const T *>(k_cache), static_cast<const T *>(v_cache), block_tables,
                                                    context_lens, q_start, selected, static_cast<T *>(out), ws, a);
    };
#define KVC_SELECTED_WAVES(T, D, HEADS)                                                       \
    do {                                                                                      \
        if (a.waves == 16) launch(pa_selected_valu_kernel<T, D, HEADS, 16>, T());             \
        else launch(pa_selected_valu_kernel<T, D, HEADS, 4>, T());                            \
    } while (0)
#define KVC_SELECTED(T, D)                                                                    \
    do {                                                                                      \
        if (a.heads_per_chunk == 4) KVC_SELECTED_WAVES(T, D, 4);                              \
        else if (a.heads_per_chunk == 2) KVC_SELECTED_WAVES(T, D, 2);                         \
        else KVC_SELECTED_WAVES(T, D, 1);                                                     \
    } while (0)
    if (dtype == KVC_F32) {
        if (head_dim == 64) KVC_SELECTED(float, 64); else KVC_SELECTED(float, 128);
    } else {
        if (head_dim == 64) KVC_SELECTED(uint16_t, 64); else KVC_SELECTED(uint16_t, 128);
    }
#undef KVC_SELECTED
#undef KVC_SELECTED_WAVES
    return hipGetLastError();
}

}  // namespace kvc
