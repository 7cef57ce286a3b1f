// What the product with low-rank adapters (adapters.cu) asks of the grouped products (grouped.cu).
#pragma once

#include "common.cuh"

namespace regione {

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

// u[r, :] = s_a x[r] A_a^T, rows of groups with an adapter
int adapters_into(const AdapterCall& c, uint16_t* u, cudaStream_t st);
// out[r, :] = act(x[r] W_i^T + u[r] B_a^T + bias_i)
int adapters_tail(const AdapterCall& c, const uint16_t* u, cudaStream_t st);
// out[r, :] = act(x[r] W_i^T + addend[r, :] + bias_i), groups of a set whose ranges touch taken as one
int adapters_joined(const AdapterCall& c, const float* addend, cudaStream_t st);

}  // namespace regione
