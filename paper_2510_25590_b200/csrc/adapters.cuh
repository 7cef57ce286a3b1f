// What the product with low-rank adapters (adapters.cu) asks of the grouped products (grouped.cu).
#pragma once

#include "common.cuh"

namespace regione {

// A sum u = x A^T goes into the product with B as bf16 operands that add up to it.  No part is zero unless the sum is, and all have its sign, so
// that times an infinite element of B they are what the sum is: an infinity, and NaN only where u is 0.  lead_part takes the first of the parts
// that are still to come off `rest`; the last is what is left, to be rounded.  Two parts hold u to 2^-15 of it, three (3 x 8 bits) are the
// 24 of fp32.
__device__ __forceinline__ float lead_part(float& rest, bool last) {
    const float cut = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
    const float part = last ? rest : cut == rest ? 0.5f * rest : cut;
    if (!isinf(rest)) rest -= part;
    return part;
}

struct AdapterCall {
    const uint16_t* x;
    long long x_stride;
    const uint16_t *w, *bias;                         // [n_weights, N, K], [n_weights, N] or NULL
    const uint16_t *a, *b;                            // [n_adapters, rank, K], [n_adapters, N, rank]
    const float* scale;                               // [n_adapters] or NULL
    const int32_t* adapter;                           // [groups]
    const int32_t *row_begin, *row_end;
    int n_adapters, rank, rows_cap, groups, n_weights, K, N, activation;
    uint16_t* out;
    long long out_stride;
    int32_t* dev_status;
};

// Arguments that all grouped products have in common.
int check_grouped(const void* x, const void* w, const void* bias, const void* begin, const void* end, int rows_cap, int groups,
                  int n_weights, int K, int N, int activation, const void* out, long long out_stride);

// Parts of u between the two launches of many rows.  Outputs of 17408 rows (rank 64, GELU) are then as far from 64 bits as those of a product in
// fp32, 1.665e-3, which is their own rounding; with one part 1.80e-3, at 390 us instead of 398.  A third takes 412 and changes nothing there.
constexpr int kSumParts = 2;

// u[r, :] = s_a x[r] A_a^T, rows of groups with an adapter; part i of row r is row i rows_cap + r of u
int adapters_into(const AdapterCall& c, uint16_t* u, cudaStream_t st);
// out[r, :] = act(x[r] W_i^T + u[r] B_a^T + bias_i)
int adapters_tail(const AdapterCall& c, const uint16_t* u, cudaStream_t st);
// out[r, :] = act(x[r] W_i^T + addend[r, :] + bias_i), groups of a set whose ranges touch taken as one
int adapters_joined(const AdapterCall& c, const float* addend, cudaStream_t st);

}  // namespace regione
