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
// Both are bound by device memory.  Forward: one to eight warps have a row, all of its loads in flight before the first is used; the row stays
// in registers, so that the mean of the squared distances is taken from the mean itself and not as a difference of two sums.
// Parameters are read again for every row and come from L1.  34816 x 4096 rows with the residual 184 us, 0.90 of the copy rate; 1075 x
// 2048 5.3, latency.
// Backward: a block has a contiguous share of the rows, gone through by teams, and a thread the same columns of all rows of its team, whose
// sums it keeps in registers; two sums a row cross the team (one barrier).  Where a share passes from one group to the next the
// teams' sums go to a slot of the workspace, and a second kernel adds the slots of a set in the order of the rows: results do
// not depend on timing.  17408 x 2048 rows with the residual 82 us, 0.81 of the copy rate: sixteen warps an SM, which is what the sums leave
// registers for, issue half of the time (a form of 86 us took 58 without its loads).  All arithmetic in fp32.
#include "f32x2.cuh"
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
    long long x_step, dy_step, dz_step, r_step, dx_step, dr_step;      // of a team, from one of its rows to the next: teams * stride
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

// W warps to a row (1: eight rows to a block), P pieces of 8 columns to a thread, of which only the last may lie behind the row.
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
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    const uint64_t one = pair_of(p.one, p.one);
    const bool whole = ((P - 1) * kThreads + t) * 8 < p.C;
    int g = 0;
    for (int v = blockIdx.x * kTeams + team; v < total; v += gridDim.x * kTeams) {
        g = group_of(&table, v, g);
        const size_t row = (size_t)(table.begin[g] + v - table.first[g]);
        const size_t set = (size_t)(g % p.n_sets) * p.set_stride;
        uint4 x[P], r[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            x[i] = r[i] = none;
            if (i < P - 1 || whole) {
                x[i] = ld_once128(p.x + row * p.x_stride + (i * kThreads + t) * 8);
                if (RES) r[i] = ld_once128(p.r + row * p.r_stride + (i * kThreads + t) * 8);
            }
        }
        uint64_t z[P][4], sum = 0;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            widen8(x[i], z[i]);
            if (RES && (i < P - 1 || whole)) {
                uint64_t b[4], q[4];
                widen8(r[i], b);
                if (p.gate != nullptr) {
                    widen8(ldg128(p.gate + set + (i * kThreads + t) * 8), q);
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[i][e] = fma2(q[e], b[e], z[i][e]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[i][e] = add2(b[e], z[i][e]);
                }
                x[i] = round8(z[i]);
                *reinterpret_cast<uint4*>(p.x_out + row * p.x_out_stride + (i * kThreads + t) * 8) = x[i];
                widen8(x[i], z[i]);
            }
            sum = add2(sum, add2(add2(z[i][0], z[i][1]), add2(z[i][2], z[i][3])));
        }
        const float mean = row_sum<W>(sum2(sum), part[0]) * inv;
        const uint64_t minus = pair_of(-mean, -mean);
        uint64_t sq = 0;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (i == P - 1 && !whole) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                z[i][e] = add2(z[i][e], minus);
                sq = fma2(z[i][e], z[i][e], sq);
            }
        }
        const float rstd = rsqrtf(fmaf(row_sum<W>(sum2(sq), part[1]), inv, p.eps));
        if (t == 0) {
            if (p.mean != nullptr) p.mean[row] = mean;
            if (p.rstd != nullptr) p.rstd[row] = rstd;
        }
        const uint64_t scale = pair_of(rstd, rstd);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (i == P - 1 && !whole) break;
            uint64_t w[4], b[4] = {0, 0, 0, 0};
            const size_t at = set + (i * kThreads + t) * 8;
            if (p.bias != nullptr) widen8(ldg128(p.bias + at), b);
            if (p.weight != nullptr) {
                widen8(ldg128(p.weight + at), w);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[i][e] = fma2(mul2(z[i][e], scale), add2(w[e], one), b[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) z[i][e] = fma2(z[i][e], scale, b[e]);
            }
            *reinterpret_cast<uint4*>(p.out + row * p.out_stride + (i * kThreads + t) * 8) = round8(z[i]);
        }
    }
}

// Rows to a block's share: the same in both kernels of the backward pass.
__host__ __device__ __forceinline__ int norm_share(int total, int blocks) { return total > 0 ? (total + blocks - 1) / blocks : 1; }

constexpr int kNormThreads = 512, kNormMaxTeams = 8;

// 16 bytes to shared memory on their own; a thread waits for its own copies only, and reads what it copied itself.
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

// `teams` of `width` threads to a block, a row to a team; AHEAD rows of every team are on their way or at hand, each thread's columns at
// places of its own: no barrier, and the bytes in flight do not depend on registers.
template <bool RES, int EACH, int AHEAD>
__global__ void __launch_bounds__(kNormThreads, 1) layer_norm_backward_kernel(const __grid_constant__ NormGradArgs p, int width, int teams) {
    extern __shared__ __align__(16) uint8_t ring[];   // [AHEAD][x, dy, dx_out, r][piece][threads] of 16 bytes
    __shared__ RowGroups table;
    __shared__ uint64_t part[2][kNormThreads / 32];   // of a warp: the two sums
    __shared__ float4 stage[kNormThreads];
    grid_dependency_wait();
    grid_launch_dependents();
    const int total = fill_row_groups(&table, p.row_begin, p.row_end, p.groups, p.rows_cap, blockIdx.x == 0, p.dev_status);
    const int share = norm_share(total, gridDim.x);
    const long long v0 = (long long)blockIdx.x * share;
    const int v1 = (int)min((long long)total, v0 + share);
    if (v0 >= v1) return;
    const int team = threadIdx.x / width, t = threadIdx.x - team * width;
    const int warps = width >> 5, lane = threadIdx.x & 31;
    const bool from_elsewhere = p.dz != nullptr;
    const float inv = 1.0f / p.C;
    const uint64_t one = pair_of(p.one, p.one);
    const uint32_t piece_bytes = blockDim.x * 16, array_bytes = EACH * piece_bytes, slot_bytes = (RES ? 4 : 3) * array_bytes;
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(ring) + threadIdx.x * 16;
    int col[EACH];
    bool live[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        col[i] = (i * width + t) * 8;
        live[i] = col[i] < p.C;
    }
    int g = group_of(&table, (int)v0, 0), turn = 0;
    // the rows to fetch: where their group ends, and where they lie
    int next = (int)v0 + team, next_g = g, next_end = 0;
    uint32_t next_slot = 0, slot = 0;
    const uint16_t *x_at = nullptr, *dy_at = nullptr, *dz_at = nullptr, *r_at = nullptr;
    auto fetch = [&] {
        if (next < v1) {
            if (next >= next_end) {
                next_g = group_of(&table, next, next_g);
                next_end = table.first[next_g + 1];
                const size_t row = (size_t)(table.begin[next_g] + next - table.first[next_g]);
                x_at = p.x + row * p.x_stride + col[0];
                dy_at = p.dy + row * p.dy_stride + col[0];
                dz_at = p.dz + row * p.dz_stride + col[0];
                r_at = p.r + row * p.r_stride + col[0];
            }
            uint32_t to = base + next_slot;
#pragma unroll
            for (int i = 0; i < EACH; ++i, to += piece_bytes) {
                if (!live[i]) break;
                copy16(to, x_at + i * width * 8);
                copy16(to + array_bytes, dy_at + i * width * 8);
                if (from_elsewhere) copy16(to + 2 * array_bytes, dz_at + i * width * 8);
                if (RES) copy16(to + 3 * array_bytes, r_at + i * width * 8);
            }
            x_at += p.x_step;
            dy_at += p.dy_step;
            if (from_elsewhere) dz_at += p.dz_step;
            if (RES) r_at += p.r_step;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        next += teams;
        next_slot += slot_bytes;
        if (next_slot == AHEAD * slot_bytes) next_slot = 0;
    };
#pragma unroll 1
    for (int i = 0; i < AHEAD - 1; ++i) fetch();
    int u = (int)v0 + team;
    for (int v = (int)v0; v < v1;) {
        // the share's rows of one group
        g = group_of(&table, v, g);
        const int end = min(v1, table.first[g + 1]);
        const size_t set = (size_t)(g % p.n_sets) * p.set_stride;
        const uint32_t unit = p.one != 0.f ? 0u : 0x3f803f80u;
        uint64_t w[EACH][4], gate[EACH][4];
        uint64_t dw[EACH][4], db[EACH][4], dg[EACH][4];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            uint4 weight = make_uint4(unit, unit, unit, unit), of = make_uint4(0u, 0u, 0u, 0u);
            if (p.weight != nullptr && live[i]) weight = ldg128(p.weight + set + col[i]);
            if (RES && live[i]) of = ldg128(p.gate + set + col[i]);
            widen8(weight, w[i]);
            widen8(of, gate[i]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[i][e] = add2(w[i][e], one);
                dw[i][e] = db[i][e] = dg[i][e] = 0;
            }
        }
        size_t row = (size_t)(table.begin[g] + u - table.first[g]);
        float mean = 0.f, rstd = 0.f;
        if (u < end) {
            mean = p.mean[row];
            rstd = p.rstd[row];
        }
        uint16_t *dx_at = p.dx + row * p.dx_stride + col[0], *dr_at = p.dr + row * p.dr_stride + col[0];
        for (; u < end; u += teams) {
            fetch();                                  // (into the place of the row before this one)
            asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory");
            const uint32_t at = base + slot;
            slot += slot_bytes;
            if (slot == AHEAD * slot_bytes) slot = 0;
            const uint64_t minus = pair_of(-mean, -mean), scale = pair_of(rstd, rstd);
            row += teams;
            if (u + teams < end) {                    // (of the next row)
                mean = p.mean[row];
                rstd = p.rstd[row];
            }
            constexpr bool kKeep = !(RES && EACH > 1);           // room for a row's h and a between the two passes
            uint64_t h[EACH][4], a[EACH][4], sum_a = 0, sum_ah = 0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                if (!live[i]) break;
                widen8(lds128(at + i * piece_bytes), h[i]);
                widen8(lds128(at + i * piece_bytes + array_bytes), a[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    h[i][e] = mul2(add2(h[i][e], minus), scale);
                    dw[i][e] = fma2(a[i][e], h[i][e], dw[i][e]);
                    db[i][e] = add2(a[i][e], db[i][e]);
                    a[i][e] = mul2(a[i][e], w[i][e]);
                    sum_a = add2(sum_a, a[i][e]);
                    sum_ah = fma2(a[i][e], h[i][e], sum_ah);
                }
            }
            uint64_t sums = pair_of(sum2(sum_a), sum2(sum_ah));
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                float x, y;
                parts_of(sums, x, y);
                sums = add2(sums, pair_of(__shfl_xor_sync(0xffffffffu, x, d), __shfl_xor_sync(0xffffffffu, y, d)));
            }
            if (warps > 1) {
                const uint64_t* mine = &part[turn][team * warps];
                if (lane == 0) part[turn][threadIdx.x >> 5] = sums;
                asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(width) : "memory");
                // (each half of a warp has the sums of all warps, up to sixteen: four steps, however many there are)
                sums = (lane & 15) < warps ? mine[lane & 15] : 0;
#pragma unroll
                for (int d = 8; d > 0; d >>= 1) {
                    float x, y;
                    parts_of(sums, x, y);
                    sums = add2(sums, pair_of(__shfl_xor_sync(0xffffffffu, x, d), __shfl_xor_sync(0xffffffffu, y, d)));
                }
                turn ^= 1;                            // (a place is written again two rows on, behind the next one's barrier)
            }
            float s1, s2;
            parts_of(mul2(sums, pair_of(-inv, -inv)), s1, s2);
            const uint64_t mean_a = pair_of(s1, s1), mean_ah = pair_of(s2, s2);
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                if (!live[i]) break;
                uint64_t d[4], q[4] = {0, 0, 0, 0};
                if (!kKeep) {
                    widen8(lds128(at + i * piece_bytes), h[i]);
                    widen8(lds128(at + i * piece_bytes + array_bytes), a[i]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        h[i][e] = mul2(add2(h[i][e], minus), scale);
                        a[i][e] = mul2(a[i][e], w[i][e]);
                    }
                }
                if (from_elsewhere) widen8(lds128(at + i * piece_bytes + 2 * array_bytes), q);
#pragma unroll
                for (int e = 0; e < 4; ++e) d[e] = fma2(fma2(h[i][e], mean_ah, add2(a[i][e], mean_a)), scale, q[e]);
                *reinterpret_cast<uint4*>(dx_at + i * width * 8) = round8(d);
                if constexpr (RES) {
                    widen8(lds128(at + i * piece_bytes + 3 * array_bytes), q);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        dg[i][e] = fma2(d[e], q[e], dg[i][e]);
                        d[e] = mul2(d[e], gate[i][e]);
                    }
                    *reinterpret_cast<uint4*>(dr_at + i * width * 8) = round8(d);
                }
            }
            dx_at += p.dx_step;
            if (RES) dr_at += p.dr_step;
        }
        // the teams' sums, in their order, to the slot of this share and group
        float* to = p.sums + (size_t)(blockIdx.x + g) * 3 * p.C;
        auto gather = [&](const uint64_t (&s)[4], float* to, bool live) {
            float4 f[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                parts_of(s[2 * i], f[i].x, f[i].y);
                parts_of(s[2 * i + 1], f[i].z, f[i].w);
            }
            if (teams > 1) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    __syncthreads();
                    if (team > 0) stage[threadIdx.x] = f[i];
                    __syncthreads();
                    if (team == 0)
                        for (int k = 1; k < teams; ++k) {
                            const float4 other = stage[k * width + t];
                            f[i].x += other.x; f[i].y += other.y; f[i].z += other.z; f[i].w += other.w;
                        }
                }
            }
            if (team != 0 || !live) return;
            reinterpret_cast<float4*>(to)[0] = f[0];
            reinterpret_cast<float4*>(to)[1] = f[1];
        };
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            gather(dw[i], to + col[i], live[i]);
            gather(db[i], to + p.C + col[i], live[i]);
            if (RES) gather(dg[i], to + 2 * p.C + col[i], live[i]);
        }
        v = end;
    }
}

// The slots of a set, added in the order of the rows: a warp takes every sixteenth, the sixteen sums are added in their order.  64 columns to
// a block, so that few sets still make some blocks; ten loads of a warp are on their way at one time, which is all it has where there is
// a block to an SM.  blockIdx.z: which of the three.
constexpr int kSumWarps = 16, kSumColumns = 64;
__global__ void __launch_bounds__(kSumWarps * 32) layer_norm_sums_kernel(const __grid_constant__ NormGradArgs p, int blocks) {
    __shared__ RowGroups table;
    __shared__ float2 part[kSumWarps][32];
    // (the ranges were written ahead of the kernel in front of this one, which had waited for them before it let this one in)
    const int total = fill_row_groups(&table, p.row_begin, p.row_end, p.groups, p.rows_cap, false, nullptr);
    grid_dependency_wait();
    grid_launch_dependents();
    const int share = norm_share(total, blocks), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = blockIdx.x * kSumColumns + lane * 2, kind = blockIdx.z;
    float2 sum = make_float2(0.f, 0.f);
    if (c < p.C)
        for (int g = blockIdx.y; g < p.groups; g += p.n_sets) {
            const int begin = table.first[g], end = table.first[g + 1];
            if (begin >= end) continue;
            const int last = (end - 1) / share;
            constexpr int kBatch = 10;
            for (int b = begin / share + warp; b <= last; b += kBatch * kSumWarps) {
                float2 s[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const float* from = p.sums + ((size_t)(b + i * kSumWarps + g) * 3 + kind) * p.C + c;
                    s[i] = make_float2(0.f, 0.f);
                    if (b + i * kSumWarps <= last) asm volatile("ld.global.v2.f32 {%0, %1}, [%2];" : "=f"(s[i].x), "=f"(s[i].y) : "l"(from));
                }
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    sum.x += s[i].x;
                    sum.y += s[i].y;
                }
            }
        }
    part[warp][lane] = sum;
    __syncthreads();
    float* to = kind == 0 ? p.dweight : kind == 1 ? p.dbias : p.dgate;
    if (warp == 0 && c < p.C && to != nullptr) {
#pragma unroll
        for (int i = 1; i < kSumWarps; ++i) {
            sum.x += part[i][lane].x;
            sum.y += part[i][lane].y;
        }
        *reinterpret_cast<float2*>(to + (size_t)blockIdx.y * p.C + c) = sum;
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------------
template <int W, int P, bool RES> static cudaError_t norm_launch(const NormArgs& p, int blocks, cudaStream_t st) {
    return launch_overlapped(layer_norm_kernel<W, P, RES>, dim3(blocks), dim3(W == 1 ? 256 : W * 32), 0, st, p);
}
template <int W, int P> static cudaError_t norm_launch(const NormArgs& p, int blocks, cudaStream_t st) {
    return p.r != nullptr ? norm_launch<W, P, true>(p, blocks, st) : norm_launch<W, P, false>(p, blocks, st);
}
template <int W> static cudaError_t norm_launch(const NormArgs& p, int blocks, cudaStream_t st) {
    switch ((p.C + W * 256 - 1) / (W * 256)) {
        case 1: return norm_launch<W, 1>(p, blocks, st);
        case 2: return norm_launch<W, 2>(p, blocks, st);
        case 3: return norm_launch<W, 3>(p, blocks, st);
        default: return norm_launch<W, 4>(p, blocks, st);
    }
}

// Warps to a row: what measured fastest.  Few rows: eight or four, the latency of a row counts (300 x 2048: 3.2 us with eight, 3.6 with
// four, 4.8 with two; 1075 x 2048: 5.9, 5.2, 5.6).  Many: one for short rows (17000 x 1024: 13.2 us, four 21; 40000 x 512 with a
// residual 31 and 49), two or four up to 2048 (17000 x 2048: two 26, four 31; with a residual, whose loads are twice as many, 59 and
// 51), four up to 4096 (34000 x 4096 with a residual: 191 us, 0.90 of the copy rate; eight 203).
static cudaError_t norm_run(const NormArgs& p, cudaStream_t st) {
    const int rows = p.rows_cap, sms = sm_count();
    if (p.C > 4096) return norm_launch<8>(p, std::min(rows, 4 * sms), st);
    if (rows < 4 * sms) return norm_launch<8>(p, rows, st);
    if (rows < 16 * sms || p.C > 2048) return norm_launch<4>(p, std::min(rows, 8 * sms), st);
    if (p.C <= 1024) return norm_launch<1>(p, std::min((rows + 7) / 8, 8 * sms), st);
    if (p.r != nullptr) return norm_launch<4, 2, true>(p, std::min(rows, 64 * sms), st);
    const int blocks = std::min(rows, 16 * sms);
    return p.C <= 1536 ? norm_launch<2, 3, false>(p, blocks, st) : norm_launch<2, 4, false>(p, blocks, st);
}

// Of the backward pass: threads of a team, teams of a block, blocks.
struct NormShape {
    int each, width, teams, blocks;                   // pieces of 8 columns of a thread, threads of a team, teams of a block
};
// Eight columns to a thread and up to eight teams; sixteen for rows of more than 4096 columns, which need it, and for many rows without a
// gated residual, where the sums of two pieces still fit in registers and a row's reduction costs half as much (17408 x 2048: 62 us
// with eight, 55 with sixteen; 1101 x 1536: 10.7 and 14; with the residual, 17408 x 2048: 85 and 133, as registers are spilled).  Of the
// copy rate with the residual: 17408 x 1024 0.70, 2048 0.81, 4096 0.82; 2560, whose one team leaves 10 warps to an SM, 0.66; 8704 x 8192,
// sixteen columns to a thread and spilled, 0.52.
static NormShape norm_shape(int rows_cap, int C, bool residual) {
    NormShape n;
    n.each = C > 4096 || (!residual && rows_cap > 16 * sm_count()) ? 2 : 1;
    n.width = (C / 8 + 32 * n.each - 1) / (32 * n.each) * 32;
    n.teams = std::min(kNormMaxTeams, kNormThreads / n.width);
    n.blocks = std::max(1, std::min((rows_cap + n.teams - 1) / n.teams, sm_count()));
    return n;
}
template <bool RES, int EACH, int AHEAD> static cudaError_t norm_grad_launch(const NormGradArgs& p, const NormShape& n, cudaStream_t st) {
    constexpr int kEach = AHEAD * (RES ? 4 : 3) * EACH * 16;           // bytes of a thread
    static int ready[kMaxDevices] = {};
    const int dev = current_device();
    if (dev < 0) return cudaErrorInvalidDevice;
    if (!__atomic_load_n(&ready[dev], __ATOMIC_ACQUIRE)) {
        const cudaError_t e = cudaFuncSetAttribute(layer_norm_backward_kernel<RES, EACH, AHEAD>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   kEach * kNormThreads);
        if (e != cudaSuccess) return e;
        __atomic_store_n(&ready[dev], 1, __ATOMIC_RELEASE);
    }
    const int threads = n.width * n.teams;
    return launch_overlapped(layer_norm_backward_kernel<RES, EACH, AHEAD>, dim3(n.blocks), dim3(threads), kEach * threads, st, p, n.width, n.teams);
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
    return (size_t)(norm_shape(rows_cap, C, true).blocks + groups) * 3 * C * sizeof(float);
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
    const NormShape n = norm_shape(rows_cap, C, r != nullptr);
    p.x_step = n.teams * p.x_stride; p.dy_step = n.teams * p.dy_stride; p.dz_step = n.teams * p.dz_stride;
    p.r_step = n.teams * p.r_stride; p.dx_step = n.teams * p.dx_stride; p.dr_step = n.teams * p.dr_stride;
    if (!empty) {
        const cudaError_t e = n.each == 2 ? (r ? norm_grad_launch<true, 2, 3>(p, n, st) : norm_grad_launch<false, 2, 3>(p, n, st))
                                          : (r ? norm_grad_launch<true, 1, 4>(p, n, st) : norm_grad_launch<false, 1, 4>(p, n, st));
        if (e != cudaSuccess) return launch_status(e);
    }
    if (!dweight && !dbias && !dgate) return REGIONE_OK;
    const dim3 grid((C + kSumColumns - 1) / kSumColumns, n_sets, dgate ? 3 : 2);
    return launch_status(launch_overlapped(layer_norm_sums_kernel, grid, dim3(kSumWarps * 32), 0, st, p, n.blocks));
}
