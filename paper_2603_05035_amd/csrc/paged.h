// The paged cache of keys and values and a batch of sequences, as the kernels see them.
#pragma once

#include "gelo_internal.h"

namespace gelo {

// Which sequence row `row` belongs to: the number of entries row_start[1 .. n_seqs] that are at most `row` (a binary search would be a chain
// of dependent loads; a wave reads 64 entries at once).  n_seqs where the row lies behind all of them.  All lanes active.
__device__ __forceinline__ int sequence_of_row(const int32_t* __restrict__ row_start, int n_seqs, int row) {
    const int lane = threadIdx.x & 63;
    int s = 0;
    for (int i0 = 0; i0 < n_seqs; i0 += 64) {
        const bool below = i0 + lane < n_seqs && row_start[i0 + lane + 1] <= row;
        const int n = __popcll(__ballot(below));
        s += n;
        if (n < 64) break;
    }
    return s;
}

// The rows a sequence brings: rows first ... first + count - 1 of the batch, whatever row_start holds.
struct NewRows { int first, count; };
__device__ __forceinline__ NewRows rows_of_sequence(const SeqBatch& b, int s) {
    if (!b.row_start) return NewRows{s, 1};
    const int first = max(b.row_start[s], 0), end = max(min(b.row_start[s + 1], b.n_rows), 0);        // (a difference of two such fits in 32 bits)
    return NewRows{first, min(max(end - first, 0), b.max_rows)};
}

// kv_len of a sequence.  Below zero means as little as zero does, but positions reckoned from it could leave 32 bits and come out beyond the cache.
__device__ __forceinline__ int length_of_sequence(const SeqBatch& b, int s) { return max(b.kv_len[s], 0); }

}  // namespace gelo
