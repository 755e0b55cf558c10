// The rows of a batch whose tables, lengths and masks are device data, as the kernels read and check them.
#ifndef TREEKV_ROWS_H
#define TREEKV_ROWS_H

#include <hip/hip_runtime.h>
#include <cstdint>

#include "internal.h"

namespace tkv {

struct RowTokens {
    int q0, L;
    bool ok;  // inside the batch
};
__device__ __forceinline__ RowTokens row_tokens(const tkv_draft_batch& b, int r) {
    RowTokens t;
    t.q0 = b.q_indptr[r];
    const int64_t n = static_cast<int64_t>(b.q_indptr[r + 1]) - t.q0;
    t.ok = t.q0 >= 0 && t.q0 <= b.n_qtok && n >= 1 && n <= b.max_q && n <= b.n_qtok - t.q0;
    t.L = t.ok ? static_cast<int>(n) : 0;
    return t;
}

struct RowTable {
    int first, n;  // its entries
    bool ok;       // inside the array, and no more than the batch allows
};
__device__ __forceinline__ RowTable row_table(const int32_t* indptr, int r, int n_entries, int most) {
    RowTable t;
    t.first = indptr[r];
    const int64_t n = static_cast<int64_t>(indptr[r + 1]) - t.first;
    t.ok = t.first >= 0 && t.first <= n_entries && n >= 0 && n <= most && n <= n_entries - t.first;
    t.n = t.ok ? static_cast<int>(n) : 0;
    return t;
}

// Length of a table's entry, 0 if it is no block of the pool or its length none of a block's.
__device__ __forceinline__ int entry_len(const int32_t* blocks, const int32_t* block_len, int num_blocks, int at, int& id) {
    id = blocks[at];
    if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(num_blocks)) return 0;
    const int len = block_len[id];
    return len >= 1 && len <= kBlock ? len : 0;
}

// Sum over the lanes before this one; total: over all.  All lanes are active.  By data-parallel moves: sums within the rows of
// 16 lanes, then row 0's to row 1 and row 2's to row 3, then the first half's to the second.
__device__ __forceinline__ int wave_before(int v, int& total) {
    int incl = v;
    incl += __builtin_amdgcn_update_dpp(0, incl, 0x111, 0xf, 0xf, true);   // row_shr:1
    incl += __builtin_amdgcn_update_dpp(0, incl, 0x112, 0xf, 0xf, true);   // row_shr:2
    incl += __builtin_amdgcn_update_dpp(0, incl, 0x114, 0xf, 0xf, true);   // row_shr:4
    incl += __builtin_amdgcn_update_dpp(0, incl, 0x118, 0xf, 0xf, true);   // row_shr:8
    incl += __builtin_amdgcn_update_dpp(0, incl, 0x142, 0xa, 0xf, false);  // row_bcast:15
    incl += __builtin_amdgcn_update_dpp(0, incl, 0x143, 0xc, 0xf, false);  // row_bcast:31
    total = __builtin_amdgcn_readlane(incl, 63);
    return incl - v;
}

// The same over a workgroup of W waves; part: W words of LDS, free again after the next barrier of the caller's.
template <int W>
__device__ __forceinline__ int group_before(int v, int& total, int* part) {
    const int wid = threadIdx.x >> 6;
    int mine;
    int at = wave_before(v, mine);
    if ((threadIdx.x & 63) == 0) part[wid] = mine;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        at += w < wid ? part[w] : 0;
        total += part[w];
    }
    return at;
}

}  // namespace tkv

#endif
