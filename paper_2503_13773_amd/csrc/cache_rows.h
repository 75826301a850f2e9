// What the kernels over the cache's blocks share: which sequence a query row belongs to and where it stands.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kvc {

// Row `row` of a batch: sequence n, position pos (the row sees tokens 0 .. pos), pos < 0: nothing.  Without q_start
// row n is the last position of sequence n.  False: the row belongs to no sequence.
__device__ inline bool find_row(int row, const int32_t *q_start, const int32_t *context_lens, int num_seqs, int max_context_len, int *n,
                                int *pos) {
    if (!q_start) {
        *n = row;
        *pos = min(context_lens[row], max_context_len) - 1;
        return true;
    }
    int lo = 0, hi = num_seqs;  // largest n with q_start[n] <= row: sequences without rows are skipped
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (q_start[mid] <= row) lo = mid; else hi = mid;
    }
    const int first = q_start[lo], last = q_start[lo + 1];
    if (row < first || row >= last) return false;
    *n = lo;
    *pos = min(context_lens[lo] - (last - row), max_context_len - 1);
    return true;
}

}  // namespace kvc
