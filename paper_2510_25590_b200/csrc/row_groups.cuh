// Live rows of ragged groups, numbered through: what a kernel that goes over rows in any number of blocks plans from the ranges in
// device memory.  Row v of the live ones is in the group g with first[g] <= v < first[g + 1], at begin[g] + v - first[g].
#pragma once

#include "common.cuh"
#include "grouped_plan.cuh"

namespace regione {

constexpr int kMaxRowGroups = 512;

struct RowGroups {
    int first[kMaxRowGroups + 1];
    int begin[kMaxRowGroups];
};

// Fills the table (one warp adds up, then a barrier of the block), from L2, since a kernel may do so before it has waited for the one
// in front of it.  No more rows are counted than the buffer has, which ranges without a
// common row do not reach: numbers stay within 32 bits, whatever the ranges are.
__device__ __forceinline__ int fill_row_groups(RowGroups* t, const int32_t* row_begin, const int32_t* row_end, int groups, int cap,
                                               bool reports, int32_t* dev_status) {
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        int at = 0;
        for (int g0 = 0; g0 < groups; g0 += 32) {
            const int g = g0 + lane;
            int begin = 0, rows = 0;
            bool in = true;
            if (g < groups) in = cut_range(__ldcg(row_begin + g), __ldcg(row_end + g), cap, begin, rows);
            int sum = rows;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, sum, d);
                if (lane >= d) sum += up;
            }
            if (g < groups) {
                t->begin[g] = begin;
                t->first[g] = min(at + sum - rows, cap);
            }
            at += __shfl_sync(0xffffffffu, sum, 31);
            if (reports && (!in || at > cap)) record_status(dev_status, REGIONE_DEV_BOUNDS);
            at = min(at, cap);
        }
        if (lane == 0) t->first[groups] = at;
    }
    __syncthreads();
    return t->first[groups];
}

// The group of live row v, which is not smaller than at the last call; `g` is where that one was.
__device__ __forceinline__ int group_of(const RowGroups* t, int v, int g) {
    while (t->first[g + 1] <= v) ++g;
    return g;
}

}  // namespace regione
