// Product of ragged groups of rows with the weight set of their group, and beside it the low-rank adapter of the group
// (regione_adapter_matmul):
//
//     out[r, :] = act(x[r] W_i^T + bias_i + s_a (x[r] A_a^T) B_a^T),   r in group g,  i = g mod n_weights,  a = adapter[g]
//
// The paper names no such operator; edits of one batch that each bring an adapter of their own share everything else.
//
// Groups of many rows: the tensor core does all of it.  u = s_a x A_a^T first, as a grouped product whose weight set is the adapter
// (bound by one pass over x), rounded to bf16 because the tensor core takes it as an operand: a relative 2^-9 of the adapter's part.
// Then the product with W, whose tiles go on behind the chunks of K with those of the rank, u against B_a into the same
// accumulators: the adapter's part is never rounded, written or read on its own.
//
// Groups of a row or two (a token each): tiles of their own would read W once per group.  The adapters' part comes first here, in
// fp32, by this file's kernel: a cluster of eight CTAs has a group, each CTA an eighth of K for the first factor (partial sums
// meet over distributed shared memory, added in the order of the CTAs) and an eighth of N for the second.  It is bound by reading A and B.  The
// product with W then takes groups that lie side by side as one and adds that part in its epilogue.
#include "adapters.cuh"
#include "grouped_plan.cuh"
#include "sm100_ptx.cuh"

#include <algorithm>

namespace regione {

constexpr int kMaxRank = 256;
constexpr int kPartCtas = 8, kPartThreads = 256, kPartRows = 4;

__device__ __forceinline__ void fma8(const uint4& a, const uint4& b, float& sum) {
    sum = fmaf(bf16_lo(a.x), bf16_lo(b.x), sum); sum = fmaf(bf16_hi(a.x), bf16_hi(b.x), sum);
    sum = fmaf(bf16_lo(a.y), bf16_lo(b.y), sum); sum = fmaf(bf16_hi(a.y), bf16_hi(b.y), sum);
    sum = fmaf(bf16_lo(a.z), bf16_lo(b.z), sum); sum = fmaf(bf16_hi(a.z), bf16_hi(b.z), sum);
    sum = fmaf(bf16_lo(a.w), bf16_lo(b.w), sum); sum = fmaf(bf16_hi(a.w), bf16_hi(b.w), sum);
}

// addend[r, :] = s_a (x[r] A_a^T) B_a^T for the rows of every group, zeros without an adapter.
__global__ void __launch_bounds__(kPartThreads) adapter_part_kernel(const __grid_constant__ AdapterCall p, float* __restrict__ addend) {
    __shared__ __align__(16) float partial[2][kPartRows][kMaxRank], u[kPartRows][kMaxRank];
    grid_dependency_wait();
    grid_launch_dependents();
    const int g = blockIdx.x / kPartCtas, cta = blockIdx.x % kPartCtas, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int begin, rows;
    const bool in = cut_range(p.row_begin[g], p.row_end[g], p.rows_cap, begin, rows);
    int a = p.adapter[g];
    const bool exists = a >= -1 && a < p.n_adapters;
    if ((!in || !exists) && cta == 0 && threadIdx.x == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
    if (!exists) a = -1;
    const int n0 = p.N / 8 * cta / kPartCtas * 8, n1 = p.N / 8 * (cta + 1) / kPartCtas * 8;       // features of this CTA
    if (a < 0) {                                      // (the whole cluster)
        for (int r = 0; r < rows; ++r)
            for (int f = n0 + threadIdx.x * 4; f < n1; f += kPartThreads * 4)
                *reinterpret_cast<float4*>(addend + (size_t)(begin + r) * p.N + f) = make_float4(0.f, 0.f, 0.f, 0.f);
        return;
    }
    const int k0 = p.K / 8 * cta / kPartCtas, k1 = p.K / 8 * (cta + 1) / kPartCtas;               // pieces of 8 of K
    const float scale = p.scale != nullptr ? p.scale[a] : 1.0f;
    for (int r0 = 0, turn = 0; r0 < rows; r0 += kPartRows, turn ^= 1) {
        const int live = min(kPartRows, rows - r0);
        const uint16_t* x = p.x + (size_t)(begin + r0) * p.x_stride;
        for (int j = warp; j < p.rank; j += kPartThreads / 32) {
            const uint16_t* row = p.a + ((size_t)a * p.rank + j) * p.K;
            float sum[kPartRows] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
            for (int k = k0 + lane; k < k1; k += 32) {
                const uint4 w = ldg128(row + k * 8);
#pragma unroll
                for (int r = 0; r < kPartRows; ++r)
                    if (r < live) fma8(w, ldg128(x + r * p.x_stride + k * 8), sum[r]);
            }
#pragma unroll
            for (int r = 0; r < kPartRows; ++r) {
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], d);
                if (lane == 0) partial[turn][r][j] = sum[r];
            }
        }
        ptx::cluster_sync();
        for (int i = threadIdx.x; i < kPartRows * (p.rank / 4); i += kPartThreads) {
            const int r = i / (p.rank / 4), j = 4 * (i - r * (p.rank / 4));
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int c = 0; c < kPartCtas; ++c) {
                const float4 part = ptx::ld_cluster_f4(ptx::map_rank(ptx::smem_addr(&partial[turn][r][j]), c));
                sum.x += part.x; sum.y += part.y; sum.z += part.z; sum.w += part.w;
            }
            *reinterpret_cast<float4*>(&u[r][j]) = make_float4(sum.x * scale, sum.y * scale, sum.z * scale, sum.w * scale);
        }
        __syncthreads();
        for (int f = n0 + threadIdx.x; f < n1; f += kPartThreads) {
            const uint16_t* row = p.b + ((size_t)a * p.N + f) * p.rank;
            float y[kPartRows] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int j = 0; j < p.rank; j += 8) {
                const uint4 w = ldg128(row + j);
                const float v[8] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y), bf16_lo(w.z), bf16_hi(w.z), bf16_lo(w.w), bf16_hi(w.w)};
#pragma unroll
                for (int r = 0; r < kPartRows; ++r) {
                    const float4 lo = *reinterpret_cast<const float4*>(&u[r][j]), hi = *reinterpret_cast<const float4*>(&u[r][j + 4]);
                    y[r] = fmaf(v[0], lo.x, y[r]); y[r] = fmaf(v[1], lo.y, y[r]); y[r] = fmaf(v[2], lo.z, y[r]); y[r] = fmaf(v[3], lo.w, y[r]);
                    y[r] = fmaf(v[4], hi.x, y[r]); y[r] = fmaf(v[5], hi.y, y[r]); y[r] = fmaf(v[6], hi.z, y[r]); y[r] = fmaf(v[7], hi.w, y[r]);
                }
            }
#pragma unroll
            for (int r = 0; r < kPartRows; ++r)
                if (r < live) addend[(size_t)(begin + r0 + r) * p.N + f] = y[r];
        }
        __syncthreads();                              // (u is written again)
    }
    ptx::cluster_sync();                              // (no CTA leaves while another may read its sums)
}

// Whether the groups are of so few rows that the adapters' part is summed up apart.
static bool few_rows(int rows_cap, int groups) { return (long long)rows_cap <= 16LL * groups; }

static size_t adapter_workspace(int rows_cap, int groups, int N, int rank) {
    const size_t bytes = few_rows(rows_cap, groups) ? (size_t)rows_cap * N * sizeof(float) : (size_t)rows_cap * rank * sizeof(uint16_t);
    return (bytes + 255) & ~(size_t)255;
}

}  // namespace regione

using namespace regione;

extern "C" size_t regione_adapter_matmul_workspace(int rows_cap, int groups, int K, int N, int rank) {
    if (rows_cap < 0 || groups < 0 || K < 1 || N < 1 || rank < 1 || rank > kMaxRank) return 0;
    return adapter_workspace(rows_cap, groups, N, rank);
}

extern "C" int regione_adapter_matmul(const regione_bf16* x, int64_t x_stride, const regione_bf16* w, const regione_bf16* bias,
                                      const regione_bf16* a, const regione_bf16* b, const float* scale, const int32_t* adapter,
                                      int n_adapters, int rank, const int32_t* row_begin, const int32_t* row_end, int rows_cap,
                                      int groups, int n_weights, int K, int N, int activation, regione_bf16* out, int64_t out_stride,
                                      void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    const int rc = check_grouped(x, w, bias, row_begin, row_end, rows_cap, groups, n_weights, K, N, activation, out, out_stride);
    if (rc != REGIONE_OK) return rc;
    if (!a || !b || (groups && !adapter) || !aligned16(a) || !aligned16(b) || n_adapters < 1 || rank < 1 || x_stride < K) return REGIONE_INVALID_ARG;
    if (K % 8 || x_stride % 8 || x_stride > (1LL << 32) || rank % 8 || rank > kMaxRank || n_adapters > 65536) return REGIONE_UNSUPPORTED;
    if (rows_cap == 0 || groups == 0) return REGIONE_OK;
    if (!workspace || workspace_bytes < adapter_workspace(rows_cap, groups, N, rank)) return REGIONE_WORKSPACE_TOO_SMALL;
    if (!aligned16(workspace)) return REGIONE_INVALID_ARG;
    const AdapterCall c = {x, x_stride, w, bias, a, b, scale, adapter, row_begin, row_end, n_adapters, rank, rows_cap, groups, n_weights, K, N,
                           activation, out, out_stride, dev_status};
    cudaStream_t st = (cudaStream_t)stream;
    if (!few_rows(rows_cap, groups)) {
        const int into = adapters_into(c, (uint16_t*)workspace, st);
        return into == REGIONE_OK ? adapters_tail(c, (const uint16_t*)workspace, st) : into;
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = dim3(groups * kPartCtas);
    cfg.blockDim = dim3(kPartThreads);
    cfg.stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kPartCtas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = launch_counted(&cfg, adapter_part_kernel, c, (float*)workspace);
    if (e != cudaSuccess) return launch_status(e);
    return adapters_joined(c, (const float*)workspace, st);
}
