// Layer normalisation of ragged groups of rows, behind the gated residual update of a transformer block, and its backward pass
// (regione_layer_norm, regione_layer_norm_backward).
//
// The paper takes the model's blocks as given and states neither.  Rows are in ranges that only the device knows, as the grouped
// products have them: text and image rows of every request have a scale, a shift and a gate of their own (the modulation of a
// denoising step), or all rows share a weight and a bias.
//
//   z = x + gate r (rounded to bf16: the row that x_out keeps is the row that is normalised)
//   m = mean z, s = 1 / sqrt(mean (z - m)^2 + eps), h = (z - m) s, y = h w + b, w = weight or 1 + weight
//
//   a = dy w,  dz = dz_in + s (a - mean a - h mean (a h)),  dr = gate dz
//   dweight = sum dy h,  dbias = sum dy,  dgate = sum dz r   over the rows of the groups that have the set
//
// Both are bound by device memory.  Forward: a warp has a row (128 threads where rows are few, 256 where they are long), all of its
// loads in flight before the first is used; the row stays in registers as bf16, so that the mean of the squared distances is taken
// from the mean itself and not as a difference of two sums.  Parameters are read again for every row and come from L1.
// Backward: a block has a contiguous share of the rows and a thread the same eight columns of all of them, whose sums it keeps in
// registers; two sums a row cross the block (one barrier), the next row's loads are on their way meanwhile.  Where a share
// passes from one group to the next the sums go to a slot of the workspace, and a second kernel adds the slots of a set in the
// order of the rows: results do not depend on timing.  All arithmetic in fp32.
#include "row_groups.cuh"

#include <algorithm>

namespace regione {

constexpr int kNormMaxC = 8192;

struct NormArgs {
    const uint16_t *x, *r, *gate, *weight, *bias;     // gate, weight, bias [n_sets, C], set_stride apart, or NULL
    long long x_stride, r_stride, set_stride;
    const int32_t *row_begin, *row_end;
    int groups, rows_cap, n_sets, C;
    float one;                                        // added to the weight: 1 where it is a modulation's scale
    float eps;
    uint16_t *x_out, *out;
    long long x_out_stride, out_stride;
    float *mean, *rstd;                               // [rows_cap] or NULL
    int32_t* dev_status;
};

struct NormGradArgs {
    const uint16_t *x, *dy, *dz, *r, *gate, *weight;
    long long x_stride, dy_stride, dz_stride, r_stride, set_stride;
    const float *mean, *rstd;
    const int32_t *row_begin, *row_end;
    int groups, rows_cap, n_sets, C;
    float one;
    uint16_t *dx, *dr;
    long long dx_stride, dr_stride;
    float* sums;                                      // workspace: [slot][3][C]
    float *dweight, *dbias, *dgate;                   // [n_sets, C] or NULL
    int32_t* dev_status;
};

// Read once, and possibly the buffer that is written: not through the path of read-only data.
__device__ __forceinline__ uint4 ld_once128(const void* p) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}
__device__ __forceinline__ void widen8(const uint4& w, float (&x)[8]) {
    x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
    x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
}
__device__ __forceinline__ uint4 round8(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
}

// The sum over the W warps of a row; `part`: W places that nothing else uses until the next barrier but one.
template <int W> __device__ __forceinline__ float row_sum(float x, float* part) {
    x = warp_sum(x);
    if constexpr (W > 1) {
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
        __syncthreads();
        x = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) x += part[i];
    }
    return x;
}

// W warps to a row (1: eight rows to a block), P pieces of 8 columns to a thread.
template <int W, int P, bool RES>
__global__ void __launch_bounds__(W == 1 ? 256 : W * 32) layer_norm_kernel(const __grid_constant__ NormArgs p) {
    __shared__ RowGroups table;
    __shared__ float part[2][W];
    constexpr int kTeams = W == 1 ? 8 : 1, kThreads = W * 32;
    grid_dependency_wait();
    grid_launch_dependents();
    const int total = fill_row_groups(&table, p.row_begin, p.row_end, p.groups, p.rows_cap, blockIdx.x == 0, p.dev_status);
    const int team = W == 1 ? threadIdx.x >> 5 : 0, t = W == 1 ? threadIdx.x & 31 : threadIdx.x;
    const float inv = 1.0f / p.C;
    int g = 0;
    for (int v = blockIdx.x * kTeams + team; v < total; v += gridDim.x * kTeams) {
        g = group_of(&table, v, g);
        const size_t row = (size_t)(table.begin[g] + v - table.first[g]);
        const size_t set = (size_t)(g % p.n_sets) * p.set_stride;
        uint4 z[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int c = (i * kThreads + t) * 8;
            z[i] = make_uint4(0u, 0u, 0u, 0u);
            if (c < p.C) z[i] = ld_once128(p.x + row * p.x_stride + c);
        }
        float sum = 0.f;
        if constexpr (RES) {
            uint4 r[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int c = (i * kThreads + t) * 8;
                r[i] = make_uint4(0u, 0u, 0u, 0u);
                if (c < p.C) r[i] = ld_once128(p.r + row * p.r_stride + c);
            }
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int c = (i * kThreads + t) * 8;
                if (c >= p.C) continue;
                uint4 gate = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);      // ones
                if (p.gate != nullptr) gate = ldg128(p.gate + set + c);
                float a[8], b[8], q[8];
                widen8(z[i], a); widen8(r[i], b); widen8(gate, q);
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] = fmaf(q[e], b[e], a[e]);
                z[i] = round8(a);
                *reinterpret_cast<uint4*>(p.x_out + row * p.x_out_stride + c) = z[i];
            }
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float a[8];
            widen8(z[i], a);
            sum += ((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7]));
        }
        const float mean = row_sum<W>(sum, part[0]) * inv;
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if ((i * kThreads + t) * 8 >= p.C) continue;
            float a[8];
            widen8(z[i], a);
#pragma unroll
            for (int e = 0; e < 8; ++e) sq = fmaf(a[e] - mean, a[e] - mean, sq);
        }
        const float rstd = rsqrtf(fmaf(row_sum<W>(sq, part[W > 1]), inv, p.eps));
        if (t == 0) {
            if (p.mean != nullptr) p.mean[row] = mean;
            if (p.rstd != nullptr) p.rstd[row] = rstd;
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int c = (i * kThreads + t) * 8;
            if (c >= p.C) continue;
            float a[8], w[8], b[8];
            widen8(z[i], a);
            if (p.weight != nullptr) widen8(ldg128(p.weight + set + c), w);
            else for (int e = 0; e < 8; ++e) w[e] = 1.0f - p.one;
            if (p.bias != nullptr) widen8(ldg128(p.bias + set + c), b);
            else for (int e = 0; e < 8; ++e) b[e] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] = fmaf((a[e] - mean) * rstd, w[e] + p.one, b[e]);
            *reinterpret_cast<uint4*>(p.out + row * p.out_stride + c) = round8(a);
        }
    }
}

// Rows to a block's share: the same in both kernels of the backward pass.
__host__ __device__ __forceinline__ int norm_share(int total, int blocks) { return total > 0 ? (total + blocks - 1) / blocks : 1; }

template <int T, bool RES>
__global__ void __launch_bounds__(T, T <= 256 ? 2 : 1) layer_norm_backward_kernel(const __grid_constant__ NormGradArgs p) {
    __shared__ RowGroups table;
    __shared__ float2 part[2][T / 32];
    constexpr bool kAhead = T < 1024;                 // room for the next row's loads in registers
    grid_dependency_wait();
    grid_launch_dependents();
    const int total = fill_row_groups(&table, p.row_begin, p.row_end, p.groups, p.rows_cap, blockIdx.x == 0, p.dev_status);
    const int share = norm_share(total, gridDim.x);
    const long long v0 = (long long)blockIdx.x * share;
    if (v0 >= total) return;
    const int v1 = (int)min((long long)total, v0 + share);
    const int c = threadIdx.x * 8, warps = blockDim.x >> 5;
    const bool live = c < p.C;
    const float inv = 1.0f / p.C;
    int g = group_of(&table, (int)v0, 0), ahead_g = g;
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    uint4 x, dy, dz = none, r = none;
    float mean, rstd;
    auto fetch = [&](int v, uint4& x, uint4& dy, uint4& dz, uint4& r, float& mean, float& rstd) {
        ahead_g = group_of(&table, v, ahead_g);
        const size_t row = (size_t)(table.begin[ahead_g] + v - table.first[ahead_g]);
        x = dy = none;
        mean = p.mean[row];
        rstd = p.rstd[row];
        if (!live) return;
        x = ld_once128(p.x + row * p.x_stride + c);
        dy = ld_once128(p.dy + row * p.dy_stride + c);
        if constexpr (RES) {
            if (p.dz != nullptr) dz = ld_once128(p.dz + row * p.dz_stride + c);
            r = ld_once128(p.r + row * p.r_stride + c);
        } else {
            if (p.dz != nullptr) dz = ld_once128(p.dz + row * p.dz_stride + c);
        }
    };
    float dw[8], db[8], dg[8];
    uint4 weight = none, gate = none;
    auto enter = [&] {                                // a new group: its parameters, no sums yet
        const size_t set = (size_t)(g % p.n_sets) * p.set_stride;
        const uint32_t one = p.one != 0.f ? 0u : 0x3f803f80u;
        weight = make_uint4(one, one, one, one);
        if (p.weight != nullptr && live) weight = ldg128(p.weight + set + c);
        if (RES && live) gate = ldg128(p.gate + set + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[e] = db[e] = dg[e] = 0.f;
    };
    auto leave = [&] {
        if (!live) return;
        float* to = p.sums + (size_t)(blockIdx.x + g) * 3 * p.C + c;
        auto put = [&](float* at, const float (&s)[8]) {
            reinterpret_cast<float4*>(at)[0] = make_float4(s[0], s[1], s[2], s[3]);
            reinterpret_cast<float4*>(at)[1] = make_float4(s[4], s[5], s[6], s[7]);
        };
        put(to, dw);
        put(to + p.C, db);
        if (RES) put(to + 2 * p.C, dg);
    };
    enter();
    fetch((int)v0, x, dy, dz, r, mean, rstd);
    for (int v = (int)v0; v < v1; ++v) {
        if (v >= table.first[g + 1]) {
            leave();
            g = group_of(&table, v, g);
            enter();
        }
        if (!kAhead && v > v0) fetch(v, x, dy, dz, r, mean, rstd);
        float h[8], d[8], w[8], s1 = 0.f, s2 = 0.f;
        widen8(x, h); widen8(dy, d); widen8(weight, w);
        const float m = mean, s = rstd;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[e] = live ? (h[e] - m) * s : 0.f;
            dw[e] = fmaf(d[e], h[e], dw[e]);
            db[e] += d[e];
            d[e] *= w[e] + p.one;
            s1 += d[e];
            s2 = fmaf(d[e], h[e], s2);
        }
        const uint4 dz_now = dz, r_now = r;
        const size_t row = (size_t)(table.begin[g] + v - table.first[g]);
        if (kAhead && v + 1 < v1) fetch(v + 1, x, dy, dz, r, mean, rstd);
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        float2* at = part[v & 1];
        if ((threadIdx.x & 31) == 0) at[threadIdx.x >> 5] = make_float2(s1, s2);
        __syncthreads();
        s1 = s2 = 0.f;
        for (int i = 0; i < warps; ++i) {
            s1 += at[i].x;
            s2 += at[i].y;
        }
        s1 *= inv;
        s2 *= inv;
        if (!live) continue;
        float q[8];
        widen8(dz_now, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = fmaf(d[e] - s1 - h[e] * s2, s, q[e]);
        *reinterpret_cast<uint4*>(p.dx + row * p.dx_stride + c) = round8(d);
        if constexpr (RES) {
            float b[8];
            widen8(r_now, b);
            widen8(gate, q);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dg[e] = fmaf(d[e], b[e], dg[e]);
                d[e] *= q[e];
            }
            *reinterpret_cast<uint4*>(p.dr + row * p.dr_stride + c) = round8(d);
        }
    }
    leave();
}

// The slots of a set, added in the order of the rows: a warp takes every eighth, the eight sums are added in their order.  blockIdx.z:
// which of the three.
__global__ void __launch_bounds__(256) layer_norm_sums_kernel(const __grid_constant__ NormGradArgs p, int blocks) {
    __shared__ RowGroups table;
    __shared__ float4 part[8][32];
    grid_dependency_wait();
    grid_launch_dependents();
    const int total = fill_row_groups(&table, p.row_begin, p.row_end, p.groups, p.rows_cap, false, nullptr);
    const int share = norm_share(total, blocks), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = (blockIdx.x * 32 + lane) * 4, kind = blockIdx.z;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < p.C)
        for (int g = blockIdx.y; g < p.groups; g += p.n_sets) {
            const int begin = table.first[g], end = table.first[g + 1];
            if (begin >= end) continue;
            const int last = (end - 1) / share;
#pragma unroll 4
            for (int b = begin / share + warp; b <= last; b += 8) {
                const float4 s = *reinterpret_cast<const float4*>(p.sums + ((size_t)(b + g) * 3 + kind) * p.C + c);
                sum.x += s.x; sum.y += s.y; sum.z += s.z; sum.w += s.w;
            }
        }
    part[warp][lane] = sum;
    __syncthreads();
    float* to = kind == 0 ? p.dweight : kind == 1 ? p.dbias : p.dgate;
    if (warp == 0 && c < p.C && to != nullptr) {
#pragma unroll
        for (int i = 1; i < 8; ++i) {
            const float4 s = part[i][lane];
            sum.x += s.x; sum.y += s.y; sum.z += s.z; sum.w += s.w;
        }
        *reinterpret_cast<float4*>(to + (size_t)blockIdx.y * p.C + c) = sum;
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------------
template <int W, int P> static cudaError_t norm_launch(const NormArgs& p, int blocks, cudaStream_t st) {
    const dim3 grid(blocks), block(W == 1 ? 256 : W * 32);
    return p.r != nullptr ? launch_overlapped(layer_norm_kernel<W, P, true>, grid, block, 0, st, p)
                          : launch_overlapped(layer_norm_kernel<W, P, false>, grid, block, 0, st, p);
}

static cudaError_t norm_run(const NormArgs& p, cudaStream_t st) {
    const int sms = sm_count();
    // Rows that fill the warps of the GPU a few times over: a warp each.  Fewer: four warps, the latency of a row counts.
    if (p.C > 4096) return norm_launch<8, 4>(p, std::min(p.rows_cap, 8 * sms), st);
    if (p.rows_cap < 16 * sms) {
        const int blocks = std::min(p.rows_cap, 16 * sms);
        if (p.C <= 1024) return norm_launch<4, 1>(p, blocks, st);
        if (p.C <= 2048) return norm_launch<4, 2>(p, blocks, st);
        return norm_launch<4, 4>(p, blocks, st);
    }
    const int blocks = std::min((p.rows_cap + 7) / 8, 8 * sms);
    if (p.C <= 256) return norm_launch<1, 1>(p, blocks, st);
    if (p.C <= 512) return norm_launch<1, 2>(p, blocks, st);
    if (p.C <= 1024) return norm_launch<1, 4>(p, blocks, st);
    if (p.C <= 2048) return norm_launch<1, 8>(p, blocks, st);
    return norm_launch<1, 16>(p, blocks, st);
}

// Blocks of the backward pass: as many as are resident at one time, with two rows each at least.
static int norm_blocks(int rows_cap, int C) {
    const int threads = (C / 8 + 31) & ~31;
    return std::max(1, std::min((rows_cap + 1) / 2, sm_count() * std::max(1, std::min(8, 640 / threads))));
}

template <int T> static cudaError_t norm_grad_launch(const NormGradArgs& p, int blocks, cudaStream_t st) {
    const dim3 grid(blocks), block((p.C / 8 + 31) & ~31);
    return p.r != nullptr ? launch_overlapped(layer_norm_backward_kernel<T, true>, grid, block, 0, st, p)
                          : launch_overlapped(layer_norm_backward_kernel<T, false>, grid, block, 0, st, p);
}

static int check_norm(int rows_cap, int groups, int n_sets, int C, long long set_stride, const void* begin, const void* end) {
    if (rows_cap < 0 || groups < 0 || n_sets < 1 || C < 1 || set_stride < C) return REGIONE_INVALID_ARG;
    if (groups && (!begin || !end)) return REGIONE_INVALID_ARG;
    if (C % 8 || C > kNormMaxC || set_stride % 8 || set_stride > (1LL << 32) || groups > kMaxRowGroups || n_sets > 65535 || rows_cap > (1 << 24))
        return REGIONE_UNSUPPORTED;
    return REGIONE_OK;
}
// A matrix of rows: REGIONE_OK where it may be read or written as such.
static int check_rows(const void* at, long long stride, int C) {
    if (!at || !aligned16(at) || stride < C) return REGIONE_INVALID_ARG;
    return stride % 8 || stride > (1LL << 32) ? REGIONE_UNSUPPORTED : REGIONE_OK;
}

}  // namespace regione

using namespace regione;

extern "C" int regione_layer_norm(const regione_bf16* x, int64_t x_stride, const regione_bf16* r, int64_t r_stride, const regione_bf16* gate,
                                  const regione_bf16* weight, const regione_bf16* bias, int64_t set_stride, int modulated, float eps,
                                  const int32_t* row_begin, const int32_t* row_end, int rows_cap, int groups, int n_sets, int C,
                                  regione_bf16* x_out, int64_t x_out_stride, regione_bf16* out, int64_t out_stride, float* mean,
                                  float* rstd, int32_t* dev_status, void* stream) {
    int rc = check_norm(rows_cap, groups, n_sets, C, set_stride, row_begin, row_end);
    if (rc != REGIONE_OK) return rc;
    if (!(eps >= 0.f) || (gate && !r) || (x_out && !r)) return REGIONE_INVALID_ARG;
    if (!aligned16(gate) || !aligned16(weight) || !aligned16(bias)) return REGIONE_INVALID_ARG;
    if (rows_cap == 0 || groups == 0) return REGIONE_OK;
    if ((rc = check_rows(x, x_stride, C)) != REGIONE_OK || (rc = check_rows(out, out_stride, C)) != REGIONE_OK) return rc;
    if (r && ((rc = check_rows(r, r_stride, C)) != REGIONE_OK || (rc = check_rows(x_out, x_out_stride, C)) != REGIONE_OK)) return rc;
    NormArgs p = {};
    p.x = x; p.r = r; p.gate = gate; p.weight = weight; p.bias = bias;
    p.x_stride = x_stride; p.r_stride = r_stride; p.set_stride = set_stride;
    p.row_begin = row_begin; p.row_end = row_end; p.groups = groups; p.rows_cap = rows_cap; p.n_sets = n_sets; p.C = C;
    p.one = modulated ? 1.0f : 0.0f; p.eps = eps;
    p.x_out = x_out; p.out = out; p.x_out_stride = x_out_stride; p.out_stride = out_stride;
    p.mean = mean; p.rstd = rstd; p.dev_status = dev_status;
    return launch_status(norm_run(p, (cudaStream_t)stream));
}

extern "C" size_t regione_layer_norm_backward_workspace(int rows_cap, int groups, int C) {
    if (rows_cap < 0 || groups < 0 || C < 1 || C % 8 || C > kNormMaxC || groups > kMaxRowGroups || rows_cap > (1 << 24)) return 0;
    return (size_t)(norm_blocks(rows_cap, C) + groups) * 3 * C * sizeof(float);
}

extern "C" int regione_layer_norm_backward(const regione_bf16* x, int64_t x_stride, const float* mean, const float* rstd,
                                           const regione_bf16* dy, int64_t dy_stride, const regione_bf16* dx_out, int64_t dx_out_stride,
                                           const regione_bf16* r, int64_t r_stride, const regione_bf16* gate, const regione_bf16* weight,
                                           int64_t set_stride, int modulated, const int32_t* row_begin, const int32_t* row_end,
                                           int rows_cap, int groups, int n_sets, int C, regione_bf16* dx, int64_t dx_stride,
                                           regione_bf16* dr, int64_t dr_stride, float* dweight, float* dbias, float* dgate,
                                           void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    int rc = check_norm(rows_cap, groups, n_sets, C, set_stride, row_begin, row_end);
    if (rc != REGIONE_OK) return rc;
    if ((gate != nullptr) != (r != nullptr) || (r != nullptr) != (dr != nullptr) || (dgate && !r)) return REGIONE_INVALID_ARG;
    if (!aligned16(gate) || !aligned16(weight) || !aligned16(dweight) || !aligned16(dbias) || !aligned16(dgate) || !aligned16(workspace))
        return REGIONE_INVALID_ARG;
    const bool empty = rows_cap == 0 || groups == 0;  // (the sums are zeros then)
    if (!empty) {
        if (!mean || !rstd) return REGIONE_INVALID_ARG;
        if ((rc = check_rows(x, x_stride, C)) != REGIONE_OK || (rc = check_rows(dy, dy_stride, C)) != REGIONE_OK ||
            (rc = check_rows(dx, dx_stride, C)) != REGIONE_OK) return rc;
        if (dx_out && (rc = check_rows(dx_out, dx_out_stride, C)) != REGIONE_OK) return rc;
        if (r && ((rc = check_rows(r, r_stride, C)) != REGIONE_OK || (rc = check_rows(dr, dr_stride, C)) != REGIONE_OK)) return rc;
        if (!workspace || workspace_bytes < regione_layer_norm_backward_workspace(rows_cap, groups, C)) return REGIONE_WORKSPACE_TOO_SMALL;
    }
    NormGradArgs p = {};
    p.x = x; p.dy = dy; p.dz = dx_out; p.r = r; p.gate = gate; p.weight = weight;
    p.x_stride = x_stride; p.dy_stride = dy_stride; p.dz_stride = dx_out_stride; p.r_stride = r_stride; p.set_stride = set_stride;
    p.mean = mean; p.rstd = rstd; p.row_begin = row_begin; p.row_end = row_end;
    p.groups = empty ? 0 : groups; p.rows_cap = rows_cap; p.n_sets = n_sets; p.C = C; p.one = modulated ? 1.0f : 0.0f;
    p.dx = dx; p.dr = dr; p.dx_stride = dx_stride; p.dr_stride = dr_stride;
    p.sums = (float*)workspace; p.dweight = dweight; p.dbias = dbias; p.dgate = dgate; p.dev_status = dev_status;
    const cudaStream_t st = (cudaStream_t)stream;
    const int blocks = norm_blocks(rows_cap, C);
    if (!empty) {
        const cudaError_t e = C <= 2048 ? norm_grad_launch<256>(p, blocks, st) : C <= 4096 ? norm_grad_launch<512>(p, blocks, st)
                                                                                           : norm_grad_launch<1024>(p, blocks, st);
        if (e != cudaSuccess) return launch_status(e);
    }
    if (!dweight && !dbias && !dgate) return REGIONE_OK;
    const dim3 grid((C + 127) / 128, n_sets, dgate ? 3 : 2);
    return launch_status(launch_overlapped(layer_norm_sums_kernel, grid, dim3(256), 0, st, p, blocks));
}
