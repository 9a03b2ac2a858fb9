// The work plan of a ragged batch, shared by the decode kernels.
#pragma once

#include "atf_internal.hpp"

namespace atf {

// Keys of ragged row r that its query reaches (the clamps keep every read inside the
// row's cache): min(n_k_rows[r], q_pos_rows[r] + 1), within [0, n_k].
__device__ __forceinline__ int ragged_valid(const DecodeParams& p, int r) {
    const int nk = min(max(p.n_k_rows[r], 0), p.n_k);
    const int qp = min(max(p.q_pos_rows[r], 0), 0x7FFFFFFD);
    return min(nk, qp + 1);
}

// Work plan of a ragged batch, the same in every wave that computes it: the batch's
// causal keys are cut into spans of `span` tokens (about total / p.splits, a multiple
// of the workgroup's token step `step`), each row into ceil(n_valid / span) items of its own
// keys, items numbered row by row.  Returns the row of `item` (or -1 past the last
// item) and its first token; with `plan` set, also writes the index of each row's
// first item and the item count at plan[B].
__device__ inline int ragged_item(const DecodeParams& p, int item, int step, int& t_first,
                                  int64_t& span, int32_t* plan) {
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int r0 = 0; r0 < p.batch; r0 += 64) {
        int64_t nv = r0 + lane < p.batch ? ragged_valid(p, r0 + lane) : 0;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) nv += __shfl_xor(nv, o);
        total += nv;
    }
    span = (total + p.splits - 1) / p.splits;
    span = (span + step - 1) / step * step;
    if (span < step) span = step;
    int row = -1, first = 0;
    int before = 0;  // items of the rows below r0
    for (int r0 = 0; r0 < p.batch; r0 += 64) {
        const int r = r0 + lane;
        const int cnt = r < p.batch ? int((ragged_valid(p, r) + span - 1) / span) : 0;
        int incl = cnt;  // inclusive prefix over the wave's rows
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(incl, o);
            if (lane >= o) incl += y;
        }
        incl += before;
        if (plan != nullptr && r < p.batch) plan[r] = incl - cnt;
        const uint64_t hit = __ballot(item < incl);
        if (row < 0 && hit != 0) {
            const int l = __builtin_ctzll(hit);
            row = r0 + l;
            first = item - __shfl(incl - cnt, l);
        }
        before = __shfl(incl, 63);
    }
    if (plan != nullptr && lane == 0) plan[p.batch] = before;
    t_first = int(int64_t(first) * span);
    return row;
}

}  // namespace atf
