// Product of ragged groups of rows with the weight set of their group, and beside it the low-rank adapter of the group
// (regione_adapter_matmul):
//
//     out[r, :] = act(x[r] W_i^T + bias_i + s_a (x[r] A_a^T) B_a^T),   r in group g,  i = g mod n_weights,  a = adapter[g]
//
// The paper names no such operator; edits of one batch that each bring an adapter of their own share everything else.
//
// Groups of many rows: the tensor core does all of it.  u = s_a x A_a^T first, as a grouped product whose weight set is the adapter
// (bound by one pass over x), left as two bf16 numbers that add up to it (lead_part), because the tensor core takes it as an operand and one
// would be off by 2^-8.  Then the product with W, whose tiles go on behind the chunks of K with those of the rank, both parts of u against
// B_a into the same accumulators: the adapter's part is never written or read on its own.  17408 rows, K 2048, N 8192, rank 64, GELU: 398 us,
// the tensor core at the power limit (355 without adapters); 4 x 1101 rows, N 6144, rank 32: 94 (83).
//
// Groups of a row or two (a token each): tiles of their own would read W once per group.  The adapters' part comes first here, in
// fp32, by this file's kernel: a cluster of eight CTAs has eight rows with the same adapter, each CTA an eighth of K for the first factor
// (partial sums meet over distributed shared memory, added in the order of the CTAs) and an eighth of N for the second.  It is
// bound by the latency of its steps (7 to 10 us) and by reading A and B.  The product with W, which runs beside it, takes groups that lie side by
// side as one and adds that part in its epilogue.  64 rows, K 2048, N 6144, rank 16, 24 adapters: 17.8 us, of which the product on its own
// takes 11.
#include "adapters.cuh"
#include "grouped_plan.cuh"
#include "sm100_ptx.cuh"

#include <algorithm>

namespace regione {

constexpr int kMaxRank = 256, kMaxAdapterGroups = 512;
constexpr int kPartCtas = 8, kPartThreads = 256, kPartWarps = kPartThreads / 32, kPartRows = 8;
constexpr int kPartSums = 3;                          // bf16 numbers that u is taken apart into: all of its 24 bits (0.2 us of 18 more than two)

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

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

struct PartMemory {
    float sums[kPartRows][kMaxRank];                  // this CTA's part of u = x A^T
    float parts[kPartWarps * 16][kPartRows + 1];      // of a warp, before the warps with the same ranks are added
    uint16_t u[kPartSums][kPartRows][kMaxRank + 8];
    int begin_of[kMaxAdapterGroups], rows_of[kMaxAdapterGroups], adapter_of[kMaxAdapterGroups];      // of all groups
    int begin[kMaxAdapterGroups], first[kMaxAdapterGroups + 1];      // the adapter's groups: their rows, numbered through
    int warp_rows[kPartWarps], warp_groups[kPartWarps];
    int place, groups;                                // of this cluster's group among them, how many
};

// addend[r, :] = s_a (x[r] A_a^T) B_a^T for the rows of every group, zeros without an adapter.  There are `subs` clusters to a group; those of
// all groups with an adapter deal its rows out eight at a time, so that A and B are read once for eight rows wherever those are, and most
// clusters have nothing to do where many groups share few adapters.  (Few clusters that go through the groups take longer, 256 groups
// with 24 adapters 48 us instead of 37: which of them have rows is uneven.)  72 registers leave room for the product beside it.
__global__ void __launch_bounds__(kPartThreads, 3) adapter_part_kernel(const __grid_constant__ AdapterCall p, float* __restrict__ addend, int subs) {
    __shared__ __align__(16) PartMemory m;
    grid_dependency_wait();
    grid_launch_dependents();
    const int cta = blockIdx.x % kPartCtas, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kEach = kMaxAdapterGroups / kPartThreads;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int g = threadIdx.x * kEach + i;
        int a = -1, begin = 0, rows = 0;
        if (g < p.groups) {
            a = p.adapter[g];
            const bool in = cut_range(p.row_begin[g], p.row_end[g], p.rows_cap, begin, rows);
            const bool exists = a >= -1 && a < p.n_adapters;
            if ((!in || !exists) && blockIdx.x == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
            if (!exists) a = -1;
        }
        m.adapter_of[g] = a;
        m.begin_of[g] = begin;
        m.rows_of[g] = rows;
    }
    __syncthreads();
    const int n0 = p.N / 8 * cta / kPartCtas * 8, n1 = p.N / 8 * (cta + 1) / kPartCtas * 8;       // features of this CTA
    const int k0 = p.K / 8 * cta / kPartCtas, k1 = p.K / 8 * (cta + 1) / kPartCtas;               // pieces of 8 of K
    const int tiles = (p.rank + 15) / 16, k_parts = tiles >= kPartWarps ? 1 : kPartWarps / tiles;  // warps that share 16 ranks
    const int piece = lane & 3, row_of = lane >> 2;
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    bool entered = false;
    const int item = blockIdx.x / kPartCtas;
    const int g = item / subs, sub = item - g * subs, a = m.adapter_of[g];
    if (a < 0) {                                      // (the whole cluster)
        for (int r = sub; r < m.rows_of[g]; r += subs)
            for (int f = n0 + threadIdx.x * 4; f < n1; f += kPartThreads * 4)
                *reinterpret_cast<float4*>(addend + (size_t)(m.begin_of[g] + r) * p.N + f) = make_float4(0.f, 0.f, 0.f, 0.f);
        return;
    }
    // ---- the groups with this adapter, in order ----------------------------------------------------------------------------------
    {
        int mine = 0, mine_rows = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (m.adapter_of[threadIdx.x * kEach + i] == a) {
                ++mine;
                mine_rows += m.rows_of[threadIdx.x * kEach + i];
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
        for (int i = 0; i < kEach; ++i) {
            const int other = threadIdx.x * kEach + i;
            if (m.adapter_of[other] == a) {
                m.begin[at] = m.begin_of[other];
                m.first[at] = min(at_rows, p.rows_cap);
                if (other == g) m.place = at;
                ++at;
                at_rows += m.rows_of[other];
            }
        }
        __syncthreads();
    }
    const uint16_t* factor_b = p.b + ((size_t)a * p.N + n0) * p.rank;
    const float scale = p.scale != nullptr ? p.scale[a] : 1.0f;
    const int total = m.first[m.groups];
    const long long first_eight = m.place * subs + sub;
    if (first_eight * kPartRows < total && threadIdx.x == 0 && n1 > n0)      // (read in the second half; contiguous)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(factor_b), "r"((n1 - n0) * p.rank * 2) : "memory");
    for (long long c = first_eight; c * kPartRows < total; c += m.groups * subs) {
        auto buffer_row = [&](int i) {                // of the i-th of the eight rows, -1 behind the last
            const int v = (int)(c * kPartRows) + i;
            if (v >= total) return -1;
            int lo = 0, hi = m.groups - 1;            // the last group whose first row is not behind v
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (m.first[mid] <= v) lo = mid; else hi = mid - 1;
            }
            return m.begin[lo] + v - m.first[lo];
        };
        if (entered) cluster_wait();                  // (all have read what this CTA left for the eight before)
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
                constexpr int kBatch = 2;             // loads of a lane, of each operand, that are on their way at one time
                for (int k = k0 + k_part * 4; k < k1; k += kBatch * 4 * k_parts) {
                    uint4 v_lo[kBatch], v_hi[kBatch], v_x[kBatch];        // (all loads of a batch ahead of its products)
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) {
                        const int at = k + i * 4 * k_parts + piece;
                        const bool in_k = at < k1;
                        v_lo[i] = in_k && in_lo ? ldg128(lo + at * 8) : none;
                        v_hi[i] = in_k && in_hi ? ldg128(hi + at * 8) : none;
                        v_x[i] = in_k && from >= 0 ? ldg128(x + at * 8) : none;
                    }
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) mma_32(d, v_lo[i], v_hi[i], v_x[i]);
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
                if (j < p.rank) m.sums[r][j] = sum;
            }
            if (tile0 + kPartWarps / k_parts < tiles) __syncthreads();
        }
        cluster_arrive();
        cluster_wait();
        entered = true;
        // ---- the CTAs' parts, in their order; u as the sum of three bf16 numbers ---------------------------------------------------
        for (int i = threadIdx.x; i < kPartRows * (p.rank / 4); i += kPartThreads) {
            const int r = i / (p.rank / 4), j = 4 * (i - r * (p.rank / 4));
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int q = 0; q < kPartCtas; ++q) {
                const float4 part = ptx::ld_cluster_f4(ptx::map_rank(ptx::smem_addr(&m.sums[r][j]), q));
                sum.x += part.x; sum.y += part.y; sum.z += part.z; sum.w += part.w;
            }
            sum.x *= scale; sum.y *= scale; sum.z *= scale; sum.w *= scale;
#pragma unroll
            for (int o = 0; o < kPartSums; ++o) {
                const bool last = o + 1 == kPartSums;
                const float x0 = lead_part(sum.x, last), x1 = lead_part(sum.y, last), x2 = lead_part(sum.z, last), x3 = lead_part(sum.w, last);
                *reinterpret_cast<uint2*>(&m.u[o][r][j]) = make_uint2(pack_bf16x2(x0, x1), pack_bf16x2(x2, x3));
            }
        }
        cluster_arrive();
        __syncthreads();
        // ---- times B^T, 16 features to a warp at a time ------------------------------------------------------------------------------
        const int to0 = buffer_row(2 * piece), to1 = buffer_row(2 * piece + 1);
        for (int f0 = warp * 16; f0 < n1 - n0; f0 += kPartWarps * 32) {                    // two tiles of 16 features at one time
            float d[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
            for (int j0 = 0; j0 < p.rank; j0 += 64) {
                uint4 v[2][2][2];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int f = f0 + t * kPartWarps * 16, j = j0 + 32 * i + piece * 8;
                        const uint16_t* at = factor_b + (size_t)(f + row_of) * p.rank + j;
                        v[t][i][0] = j < p.rank && f < n1 - n0 ? ldg128(at) : none;
                        v[t][i][1] = j < p.rank && f + 8 < n1 - n0 ? ldg128(at + 8 * p.rank) : none;   // (features come in eights)
                    }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int j = j0 + 32 * i + piece * 8;
#pragma unroll
                    for (int o = 0; o < kPartSums; ++o) {
                        const uint4 u = j < p.rank ? *reinterpret_cast<const uint4*>(&m.u[o][row_of][j]) : none;
#pragma unroll
                        for (int t = 0; t < 2; ++t) mma_32(d[t], v[t][i][0], v[t][i][1], u);
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int f = f0 + t * kPartWarps * 16 + 8 * (i >> 1), to = i & 1 ? to1 : to0;
                    if (to >= 0 && f < n1 - n0) addend[(size_t)to * p.N + n0 + f + row_of] = d[t][i];
                }
        }
        __syncthreads();                              // (u is written again)
    }
    if (entered) cluster_wait();                      // (no CTA leaves while another may read its sums)
}

// Whether the groups are of so few rows that the adapters' part is summed up apart: 32 on average where all have one weight set, since tiles
// are shared then (16 groups of 16 rows, 2048 x 6144, rank 16: 26 us against 57; of 64 rows 57 and 59; 4096 x 4096, rank 64, of 64 rows 78
// and 72; one group of 1900 rows beside 63 single ones 108 and 246, since each of those would be a tile), 8 where sets take turns and
// there are rarely rows to share (16 groups of 8 rows: 53 us against 57, of 32 rows 62 and 58).
static bool few_rows(int rows_cap, int groups, int n_weights) { return rows_cap <= (n_weights == 1 ? 32LL : 8LL) * groups; }

// For either form, and for calls of fewer rows and groups, which may be of the other one.
static size_t adapter_workspace(int rows_cap, int groups, int N, int rank) {
    const size_t few = std::min<size_t>(rows_cap, 32 * (size_t)groups);
    return (std::max(few * N * sizeof(float), (size_t)rows_cap * rank * kSumParts * sizeof(uint16_t)) + 255) & ~(size_t)255;
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
    if (!few_rows(rows_cap, groups, n_weights)) {
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
