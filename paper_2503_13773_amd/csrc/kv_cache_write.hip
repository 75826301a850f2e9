// kvc_kv_cache_write: K and V of many new tokens into the slots that a slot map names (gfx950): the write that precedes the
// attention of a prompt, a chunk of one, or a batch of any mixture.  A copy: bound by memory, 4 * rows * Hkv * D * e bytes.
// 12 000 tokens of 32 heads of 128 in bf16, 394 MB: 75 us = 5.25 TB/s (a copy of 2 GiB moves 5.0 TB/s here); 4 x 512 tokens of 8 heads,
// 17 MB: 4.4 us, the launch and one pass to memory.
//
// One 16-byte word of K and one of V per lane.  A row's words are consecutive in k_new / v_new (rows may lie apart, as views into
// a fused projection do) and land in runs of D * e bytes, one per KV head.
#include "kvc_internal.h"

namespace kvc {

namespace {

__global__ __launch_bounds__(kThreads) void kv_cache_write_kernel(const uint4 *__restrict__ k_new, const uint4 *__restrict__ v_new, int64_t k_stride,
                                                                  int64_t v_stride, uint4 *__restrict__ k_cache, uint4 *__restrict__ v_cache,
                                                                  const int64_t *__restrict__ slot_map, int num_rows, int chunks, int per_group,
                                                                  int num_kv_heads, int words_log2, int block_size_log2, int64_t num_slots) {
    const int words = num_kv_heads << words_log2;
    const int64_t item = blockIdx.x;
    int64_t row;
    int i;  // word of the row
    if (chunks == 1) {
        const int local = threadIdx.x / words;
        row = item * per_group + local;
        i = threadIdx.x - local * words;
        if (local >= per_group || row >= num_rows) return;
    } else {
        row = item / chunks;
        i = int(item - row * chunks) * kThreads + threadIdx.x;
        if (i >= words) return;
    }
    const int64_t slot = slot_map[row];
    if (slot < 0 || slot >= num_slots) return;
    const uint4 k = k_new[row * k_stride + i], v = v_new[row * v_stride + i];
    const int64_t line = (((slot >> block_size_log2) * num_kv_heads + (i >> words_log2)) << block_size_log2) + (slot & ((1 << block_size_log2) - 1));
    const int64_t dst = (line << words_log2) + (i & ((1 << words_log2) - 1));
    k_cache[dst] = k;
    v_cache[dst] = v;
}

}  // namespace

hipError_t launch_cache_write(const void *k_new, const void *v_new, int64_t k_row_words, int64_t v_row_words, void *k_cache, void *v_cache,
                              const int64_t *slot_map, int num_rows, int num_kv_heads, int row_bytes, int block_size_log2,
                              int64_t num_slots, hipStream_t stream) {
    int words_log2 = 0;  // 16-byte words of a head's row: 8, 16 or 32
    while ((16 << words_log2) < row_bytes) ++words_log2;
    const int64_t words = int64_t(num_kv_heads) << words_log2;
    const int64_t chunks = (words + kThreads - 1) / kThreads, per_group = words <= kThreads ? kThreads / words : 1;
    // a launch holds fewer than 2^32 threads: more rows than fit go in several
    constexpr int64_t kMostGroups = (int64_t(1) << 32) / kThreads - 1;
    const int64_t most = kMostGroups / chunks * per_group;
    if (most == 0) return hipErrorInvalidValue;  // the words of one row alone
    for (int64_t n = 0; n < num_rows; n += most) {
        const int64_t rows = num_rows - n < most ? num_rows - n : most;
        const int64_t grid = (rows + per_group - 1) / per_group * chunks;
        kv_cache_write_kernel<<<dim3(unsigned(grid)), dim3(kThreads), 0, stream>>>(
            static_cast<const uint4 *>(k_new) + n * k_row_words, static_cast<const uint4 *>(v_new) + n * v_row_words, k_row_words, v_row_words,
            static_cast<uint4 *>(k_cache), static_cast<uint4 *>(v_cache), slot_map + n, int(rows), int(chunks), int(per_group), num_kv_heads,
            words_log2, block_size_log2, num_slots);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace kvc
