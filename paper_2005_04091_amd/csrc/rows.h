// Rows of a batch whose sequences have one token each (internal header, host and device).
#pragma once

#include <hip/hip_runtime.h>

namespace {

// The sequence, which is the token, of a row of a batch without q_start; -1 for a row without tokens. Sequence b
// starts at token b, so its row is b/q_block + b: behind the rows of each q_block sequences lies one without tokens, and
// behind the last sequence's there can be more. With a q_block of 1 rows are tokens.
__host__ __device__ inline int sequence_of_row(int row, int q_block, int sequences) {
    if (q_block > 1) {
        const int turn = row / (q_block + 1);
        if (row - turn * (q_block + 1) == q_block) return -1;
        row -= turn;
    }
    return row < sequences ? row : -1;
}

}  // namespace
