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
// fp32, by this file's kernel: a cluster of eight CTAs has eight rows with the same adapter, each CTA an eighth of K for the first factor
// (partial sums meet over distributed shared memory, added in the order of the CTAs) and an eighth of N for the second.  It is
// bound by the latency of its steps and by reading A and B.  The product with W, which runs beside it, takes groups that lie side by
// side as one and adds that part in its epilogue.
#include "adapters.cuh"
#include "grouped_plan.cuh"
#include "sm100_ptx.cuh"

#include <algorithm>

namespace regione {

constexpr int kMaxRank = 256, kMaxAdapterGroups = 512;
constexpr int kPartCtas = 8, kPartThreads = 256, kPartWarps = kPartThreads / 32, kPartRows = 8;

// D = A B + D of 16 x 16 by 16 x 8 bf16 numbers.  (Eight rows at a time: the tensor core's large tiles would stand almost empty.)
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 32 elements of the contraction, of which a lane has the eight of its place among four in one load: in which order they are added does not
// matter as long as both operands have the same.  lo, hi: rows l / 4 and l / 4 + 8 of A; b: row l / 4 of B.
__device__ __forceinline__ void mma_32(float (&d)[4], const uint4& lo, const uint4& hi, const uint4& b) {
    mma_16x8x16(d, lo.x, hi.x, lo.y, hi.y, b.x, b.y);
    mma_16x8x16(d, lo.z, hi.z, lo.w, hi.w, b.z, b.w);
}

// What two numbers are above those that they were rounded to.  (Infinite ones: nothing.)
__device__ __forceinline__ uint32_t rest_of(float x, float y, uint32_t rounded) {
    const float a = bf16_lo(rounded), b = bf16_hi(rounded);
    return pack_bf16x2(isinf(a) ? 0.f : x - a, isinf(b) ? 0.f : y - b);
}

struct PartMemory {
    float sums[2][kPartRows][kMaxRank];               // this CTA's part of u = x A^T, in turns
    float parts[kPartWarps * 16][kPartRows + 1];      // of a warp, before the warps with the same ranks are added
    uint16_t u_hi[kPartRows][kMaxRank + 8], u_lo[kPartRows][kMaxRank + 8];
    int begin[kMaxAdapterGroups], first[kMaxAdapterGroups + 1];      // the adapter's groups: their rows, numbered through
    int warp_rows[kPartWarps], warp_groups[kPartWarps];
    int place, groups;                                // of this cluster's group among them, how many
};

// addend[r, :] = s_a (x[r] A_a^T) B_a^T for the rows of every group, zeros without an adapter.  A cluster to a group, or `subs`; the clusters
// of all groups with an adapter deal its rows out eight at a time, so that A and B are read once for eight rows wherever those are.
__global__ void __launch_bounds__(kPartThreads) adapter_part_kernel(const __grid_constant__ AdapterCall p, float* __restrict__ addend, int subs) {
    __shared__ __align__(16) PartMemory m;
    grid_dependency_wait();
    grid_launch_dependents();
    const int cluster = blockIdx.x / kPartCtas, cta = blockIdx.x % kPartCtas, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = cluster / subs, sub = cluster - g * subs;
    int begin, rows;
    const bool in = cut_range(p.row_begin[g], p.row_end[g], p.rows_cap, begin, rows);
    int a = p.adapter[g];
    const bool exists = a >= -1 && a < p.n_adapters;
    if ((!in || !exists) && cta == 0 && threadIdx.x == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
    if (!exists) a = -1;
    const int n0 = p.N / 8 * cta / kPartCtas * 8, n1 = p.N / 8 * (cta + 1) / kPartCtas * 8;       // features of this CTA
    if (a < 0) {                                      // (the whole cluster)
        for (int r = sub; r < rows; r += subs)
            for (int f = n0 + threadIdx.x * 4; f < n1; f += kPartThreads * 4)
                *reinterpret_cast<float4*>(addend + (size_t)(begin + r) * p.N + f) = make_float4(0.f, 0.f, 0.f, 0.f);
        return;
    }
    const uint16_t* factor_b = p.b + ((size_t)a * p.N + n0) * p.rank;
    if (threadIdx.x == 0 && n1 > n0)                  // (read in the second half; contiguous)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(factor_b), "r"((n1 - n0) * p.rank * 2) : "memory");

    // ---- the groups with this adapter, in order ----------------------------------------------------------------------------------
    {
        constexpr int kEach = kMaxAdapterGroups / kPartThreads;
        int of_begin[kEach], of_rows[kEach], mine = 0, mine_rows = 0;
        bool same[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int other = threadIdx.x * kEach + i;
            same[i] = other < p.groups && p.adapter[other] == a;
            of_begin[i] = of_rows[i] = 0;
            if (same[i]) cut_range(p.row_begin[other], p.row_end[other], p.rows_cap, of_begin[i], of_rows[i]);
            mine += same[i];
            mine_rows += of_rows[i];
        }
        int at = mine, at_rows = mine_rows;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, at, d), up_rows = __shfl_up_sync(0xffffffffu, at_rows, d);
            if (lane >= d) { at += up; at_rows += up_rows; }
        }
        if (lane == 31) { m.warp_groups[warp] = at; m.warp_rows[warp] = at_rows; }
        __syncthreads();
        for (int w = 0; w < warp; ++w) { at += m.warp_groups[w]; at_rows += m.warp_rows[w]; }
        if (threadIdx.x == kPartThreads - 1) {
            m.groups = at;
            m.first[at] = min(at_rows, p.rows_cap);   // (more only where ranges overlap)
        }
        at -= mine;
        at_rows -= mine_rows;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (same[i]) {
                m.begin[at] = of_begin[i];
                m.first[at] = min(at_rows, p.rows_cap);
                if (threadIdx.x * kEach + i == g) m.place = at;
                ++at;
                at_rows += of_rows[i];
            }
        __syncthreads();
    }
    const int total = m.first[m.groups];
    const int k0 = p.K / 8 * cta / kPartCtas, k1 = p.K / 8 * (cta + 1) / kPartCtas;               // pieces of 8 of K
    const float scale = p.scale != nullptr ? p.scale[a] : 1.0f;
    const int tiles = (p.rank + 15) / 16, k_parts = tiles >= kPartWarps ? 1 : kPartWarps / tiles;  // warps that share 16 ranks
    const int piece = lane & 3, row_of = lane >> 2;
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    int turn = 0;
    for (long long c = m.place * subs + sub; c * kPartRows < total; c += m.groups * subs, turn ^= 1) {
        auto buffer_row = [&](int i) {                // of the i-th row of this round, -1 behind the last
            const int v = (int)(c * kPartRows) + i;
            if (v >= total) return -1;
            int lo = 0, hi = m.groups - 1;            // the last group whose first row is not behind v
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (m.first[mid] <= v) lo = mid; else hi = mid - 1;
            }
            return m.begin[lo] + v - m.first[lo];
        };
        // ---- u = x A^T over this CTA's part of K ---------------------------------------------------------------------------
        const int from = buffer_row(row_of);
        const uint16_t* x = p.x + (size_t)max(from, 0) * p.x_stride;
        for (int tile0 = 0; tile0 < tiles; tile0 += kPartWarps / k_parts) {
            const int tile = tile0 + warp / k_parts, k_part = warp % k_parts;
            float d[4] = {0.f, 0.f, 0.f, 0.f};
            if (tile < tiles && warp / k_parts < kPartWarps / k_parts) {
                const int j = tile * 16 + row_of;
                const uint16_t* lo = p.a + ((size_t)a * p.rank + j) * p.K;
                const uint16_t* hi = lo + (size_t)8 * p.K;
                const bool in_lo = j < p.rank, in_hi = j + 8 < p.rank;
#pragma unroll 4
                for (int k = k0 + k_part * 4 + piece; k < k1 + piece; k += 4 * k_parts) {         // (all lanes as often: k - piece is the warp's)
                    const bool in_k = k < k1;
                    mma_32(d, in_k && in_lo ? ldg128(lo + k * 8) : none, in_k && in_hi ? ldg128(hi + k * 8) : none,
                           in_k && from >= 0 ? ldg128(x + k * 8) : none);
                }
            }
            // ranks row_of, row_of + 8 of the tile; rows 2 piece, 2 piece + 1
#pragma unroll
            for (int i = 0; i < 4; ++i) m.parts[warp * 16 + row_of + 8 * (i >> 1)][2 * piece + (i & 1)] = d[i];
            __syncthreads();
            for (int i = threadIdx.x; i < kPartWarps / k_parts * 16 * kPartRows; i += kPartThreads) {
                const int r = i & (kPartRows - 1), q = i / kPartRows, of = q >> 4, j = (tile0 + of) * 16 + (q & 15);
                float sum = 0.f;
                for (int w = 0; w < k_parts; ++w) sum += m.parts[(of * k_parts + w) * 16 + (q & 15)][r];
                if (j < p.rank) m.sums[turn][r][j] = sum;
            }
            if (tile0 + kPartWarps / k_parts < tiles) __syncthreads();
        }
        ptx::cluster_sync();
        // ---- the CTAs' parts, in their order; u as the sum of two bf16 numbers, 2^-16 off -----------------------------------------
        for (int i = threadIdx.x; i < kPartRows * (p.rank / 4); i += kPartThreads) {
            const int r = i / (p.rank / 4), j = 4 * (i - r * (p.rank / 4));
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int q = 0; q < kPartCtas; ++q) {
                const float4 part = ptx::ld_cluster_f4(ptx::map_rank(ptx::smem_addr(&m.sums[turn][r][j]), q));
                sum.x += part.x; sum.y += part.y; sum.z += part.z; sum.w += part.w;
            }
            sum.x *= scale; sum.y *= scale; sum.z *= scale; sum.w *= scale;
            const uint32_t h0 = pack_bf16x2(sum.x, sum.y), h1 = pack_bf16x2(sum.z, sum.w);
            *reinterpret_cast<uint2*>(&m.u_hi[r][j]) = make_uint2(h0, h1);
            *reinterpret_cast<uint2*>(&m.u_lo[r][j]) = make_uint2(rest_of(sum.x, sum.y, h0), rest_of(sum.z, sum.w, h1));
        }
        __syncthreads();
        // ---- times B^T, 16 features to a warp at a time ------------------------------------------------------------------------------
        const int to0 = buffer_row(2 * piece), to1 = buffer_row(2 * piece + 1);
#pragma unroll 2
        for (int f0 = warp * 16; f0 < n1 - n0; f0 += kPartWarps * 16) {
            const uint16_t* lo = factor_b + (size_t)(f0 + row_of) * p.rank;
            const uint16_t* hi = lo + 8 * p.rank;
            const bool in_hi = f0 + 8 < n1 - n0;      // (features come in eights)
            float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int j0 = 0; j0 < p.rank; j0 += 32) {
                const int j = j0 + piece * 8;
                const bool in_j = j < p.rank;
                const uint4 b_lo = in_j ? ldg128(lo + j) : none, b_hi = in_j && in_hi ? ldg128(hi + j) : none;
                mma_32(d, b_lo, b_hi, in_j ? *reinterpret_cast<const uint4*>(&m.u_hi[row_of][j]) : none);
                mma_32(d, b_lo, b_hi, in_j ? *reinterpret_cast<const uint4*>(&m.u_lo[row_of][j]) : none);
            }
            const int f = n0 + f0 + row_of;
            if (to0 >= 0) addend[(size_t)to0 * p.N + f] = d[0];
            if (to1 >= 0) addend[(size_t)to1 * p.N + f] = d[1];
            if (to0 >= 0 && in_hi) addend[(size_t)to0 * p.N + f + 8] = d[2];
            if (to1 >= 0 && in_hi) addend[(size_t)to1 * p.N + f + 8] = d[3];
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
    const int subs = std::max(1, std::min(4, (rows_cap + groups * kPartRows - 1) / (groups * kPartRows)));
    cfg.gridDim = dim3(groups * subs * kPartCtas);
    cfg.blockDim = dim3(kPartThreads);
    cfg.stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kPartCtas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = launch_counted(&cfg, adapter_part_kernel, c, (float*)workspace, subs);
    if (e != cudaSuccess) return launch_status(e);
    return adapters_joined(c, (const float*)workspace, st);
}
