// Rotary positions with several axes for rows of Q and K (regione_rotary_axes), behind their per-head RMS normalisation, and the
// rotation's gradient.
//
// The paper takes the attention layer of the editors as given.  Their tokens have places with several coordinates: which image (the
// edited one, its reference, the text), which frame, which row and column; a request's own when the images of a batch are not alike,
// and between whole numbers when an image was resized.  The method fixes that a recomputed token keeps its place (Sec. 4
// "Region-Aware Generation"), so that the row list of a region step names the places as well as the rows.
//
//   y = x / sqrt(mean(x^2) + eps) * weight              over the D elements of a row and head (where asked for)
//   t_i = position[axis_i] * freq_i                      for the D/2 pairs, (a, b) -> (a cos t - b sin t, a sin t + b cos t)
//
// Angles are formed here and not read from a table: frequency in turns as the sum of two fp32 numbers, the product with the position
// exact in two parts, whole turns taken off before anything is rounded.  Of a product of T turns the second part and what the frequency's 48
// bits leave out are off by 1.6 2^-47 T together, what is left of a turn and its radians by 2^-24: no more than 2^-22 turns up to
// 2^23 turns, and 2^-45 T beyond (one fp32 product at position 10^5 is off by 2^-8 radians, as much as the bf16 output).
//
// Bound by device memory, 4 bytes an element, where rows have many heads: 20 000 rows of 48 heads of 128 86 us, 0.89 of the copy rate.  A warp
// has a row, or a part of its heads where rows are few; its lanes form the angles of the D/2 pairs once and leave them in shared memory,
// then go through the heads, up to eight loads of 16 bytes a lane in flight.  What a row takes before its first head (its place, its angles,
// the factors of Q and of K), which a warp waits for row by row, bounds rows of few heads: 46 352 rows of 20 heads of 64 54 us, 0.68, with
// sixteen warps an SM, which is what the registers leave, that issue 57 % of the time.
#include "f32x2.cuh"

#include <algorithm>
#include <cmath>

namespace regione {

constexpr int kRotaryMaxD = 256, kRotaryWarps = 8, kRotaryAxes = 4;

struct RotaryArgs {
    const uint16_t *q, *k;                            // rows row_stride apart, requests batch_stride apart, heads of a row side by side
    long long q_batch, q_row, k_batch, k_row;
    uint16_t *q_out, *k_out;
    long long q_out_batch, q_out_row, k_out_batch, k_out_row;
    const int32_t *idx, *n;                           // [B, cap], [B], or NULL
    const float* positions;                           // [B or 1, n_pos, axes]
    long long positions_batch;
    int B, n_pos, cap, Hq, Hk, D, axes;
    int compact;                                      // row j is read; else row idx[b, j]
    const uint16_t *q_weight, *k_weight;
    float eps, sign;                                  // sign: -1 turns back
    int parts_log;                                    // 1 << this warps share a row
    int32_t* dev_status;
    float turns_hi[kRotaryMaxD / 2], turns_lo[kRotaryMaxD / 2];
    uint8_t axis[kRotaryMaxD / 2];
};

// A lane's pieces of 8 elements of a head, LANES lanes to a head: in the half layout a piece and the one D/2 elements further on, whose
// elements are the partners of its own; else EACH pieces, LANES apart.  LANES is a power of two; where that is more than a head has
// for them, lanes have nothing to do (heads of 80: 6 of 16), and EACH is 3 where that leaves none (heads of 48, 96 and 192).
template <int LANES, int EACH, bool HALF> struct RotaryShape {
    static constexpr int kLoads = HALF ? 2 : EACH;                     // of a pass
    static constexpr int kAhead = EACH > 1 ? 2 : 4;                    // passes whose loads are on their way
    static constexpr int kPairs = HALF ? LANES * 8 : LANES * EACH * 4; // of a head, at most
    // An SM's blocks: as many as keep that in registers.  (Halves, 20 000 rows of 48 heads of 128: 84 us with two blocks and four passes, 93 with
    // three and two; 3 x 4099 rows of 26 heads of 96 without norms: 23.8 with three pieces a lane, 26 with a quarter of the lanes idle.)
    static constexpr int kBlocks = HALF || EACH > 1 ? 2 : 3;
};

template <int LANES, int EACH, bool HALF, bool NORM>
__global__ void __launch_bounds__(kRotaryWarps * 32, (RotaryShape<LANES, EACH, HALF>::kBlocks))
rotary_axes_kernel(const __grid_constant__ RotaryArgs p) {
    using Shape = RotaryShape<LANES, EACH, HALF>;
    constexpr int kLoads = Shape::kLoads, kAhead = Shape::kAhead;
    __shared__ __align__(16) float cos_of[kRotaryWarps][Shape::kPairs], sin_of[kRotaryWarps][Shape::kPairs];
    __shared__ float2 turns_of[Shape::kPairs];
    __shared__ int axis_of[Shape::kPairs];
    constexpr int kHeads = 32 / LANES;                // of a pass of the warp
    constexpr int kPairs = (Shape::kPairs + 31) / 32; // of a lane
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pairs = p.D / 2;
    // The pairs' frequencies: from the launch's parameters once a block, since 32 addresses of them take a warp 32 turns, then a lane keeps
    // those of the pairs whose angles it forms.
    if (threadIdx.x < Shape::kPairs) {
        turns_of[threadIdx.x] = make_float2(p.turns_hi[threadIdx.x], p.turns_lo[threadIdx.x]);
        axis_of[threadIdx.x] = p.axis[threadIdx.x];
    }
    __syncthreads();
    float2 turns[kPairs];
    int axis[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        const int at = min(lane + 32 * i, Shape::kPairs - 1);
        turns[i] = turns_of[at];
        axis[i] = axis_of[at];
    }
    grid_dependency_wait();
    grid_launch_dependents();
    const int g = lane & (LANES - 1), in_pass = lane / LANES, pieces = p.D / 8, units = HALF ? pieces / 2 : pieces;
    const bool on = EACH > 1 || g < units;
    const int apart = 8 * (HALF ? units : LANES);     // elements from one of the lane's pieces to the next
    const float inv = 1.0f / p.D;
    const int heads = p.Hq + p.Hk, passes = (heads + kHeads - 1) / kHeads;
    const uint32_t total = ((uint32_t)p.B * p.cap) << p.parts_log;
    for (uint32_t item = blockIdx.x * kRotaryWarps + warp; item < total; item += gridDim.x * kRotaryWarps) {
        const int row = (int)(item >> p.parts_log), part = (int)(item & ((1u << p.parts_log) - 1));
        const int b = (int)((uint32_t)row / (uint32_t)p.cap), j = row - b * p.cap;
        int live = p.cap;
        if (p.n != nullptr) {
            live = p.n[b];
            if (live < 0 || live > p.cap) {
                if (j == 0 && part == 0 && lane == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
                live = live < 0 ? 0 : p.cap;
            }
        }
        if (j >= live) continue;
        int place = j;
        if (p.idx != nullptr) {
            place = p.idx[row];
            if (place < 0 || place >= p.n_pos) {
                if (lane == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
                continue;
            }
        }
        const long long from = p.compact ? j : place;
        const uint16_t* q = p.q + b * p.q_batch + from * p.q_row + 8 * g;
        const uint16_t* k = p.k + b * p.k_batch + from * p.k_row + 8 * g - (long long)p.Hq * p.D;
        uint16_t* q_out = p.q_out + b * p.q_out_batch + j * p.q_out_row + 8 * g;
        uint16_t* k_out = p.k_out + b * p.k_out_batch + j * p.k_out_row + 8 * g - (long long)p.Hq * p.D;
        const int first_pass = (passes * part) >> p.parts_log, last_pass = (passes * (part + 1)) >> p.parts_log;
        uint4 w[kAhead][kLoads];
        auto fetch = [&](int i0) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (i0 + u >= last_pass) break;       // (for the whole warp)
                const int h = (i0 + u) * kHeads + in_pass;
                const uint16_t* src = (h < p.Hq ? q : k) + h * p.D;
                const bool in = on && h < heads;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    w[u][i] = make_uint4(0u, 0u, 0u, 0u);
                    // (not through the path of read-only data: the row may be turned in place)
                    if (in) asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                                         : "=r"(w[u][i].x), "=r"(w[u][i].y), "=r"(w[u][i].z), "=r"(w[u][i].w) : "l"(src + i * apart));
                }
            }
        };
        fetch(first_pass);
        // the angles, while the first heads are on their way: lane a has the position on axis a
        const float at = lane < p.axes ? p.positions[b * p.positions_batch + (long long)place * p.axes + lane] : 0.f;
        __syncwarp();                                 // (the row before has read its angles)
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const float x = __shfl_sync(0xffffffffu, at, axis[i]);
            if (lane + 32 * i < pairs) {
                const float whole = x * turns[i].x, rest = fmaf(x, turns[i].y, fmaf(x, turns[i].x, -whole));
                float turn = (whole - rintf(whole)) + rest;
                turn = (turn - rintf(turn)) * 6.283185307179586f;
                // (the fast forms: 2^-21 off within half a turn, a hundredth of the output's rounding)
                cos_of[warp][lane + 32 * i] = __cosf(turn);
                sin_of[warp][lane + 32 * i] = __sinf(turn) * p.sign;
            }
        }
        __syncwarp();
        // What the lane's elements are multiplied with.
        //   halves, a piece x and its partner y: cosines, sines with both signs, and the weights as they are; forming weights times angles
        //   takes longer than the multiplications where a row has few passes, and as long where it has twelve
        //   pairs, (a, b) -> r (a own.x + b other.x, a own.y + b other.y): weights and angles in one, the same for all heads of Q, and of K
        uint64_t own[HALF ? 1 : kLoads][4], other[kLoads][4];
        uint4 weight_of[2];
        auto factors = [&](const uint16_t* weight) {
            if constexpr (HALF && NORM) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    weight_of[i] = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);     // ones
                    if (weight != nullptr && on) weight_of[i] = ldg128(weight + 8 * g + i * apart);
                }
            } else if constexpr (!HALF) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int first = on ? 4 * (g + LANES * i) : 0;
                    const float4 cs = *reinterpret_cast<const float4*>(&cos_of[warp][first]), sn = *reinterpret_cast<const float4*>(&sin_of[warp][first]);
                    const float c[4] = {cs.x, cs.y, cs.z, cs.w}, s[4] = {sn.x, sn.y, sn.z, sn.w};
                    uint4 v = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);          // ones
                    if (NORM && weight != nullptr && on) v = ldg128(weight + 8 * g + i * apart);       // (from L1: registers are short)
                    const uint32_t of[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        own[i][e] = pair_of(c[e], s[e]);
                        other[i][e] = pair_of(-s[e], c[e]);
                        if constexpr (NORM) {
                            own[i][e] = mul2(own[i][e], pair_of(bf16_lo(of[e]), bf16_lo(of[e])));
                            other[i][e] = mul2(other[i][e], pair_of(bf16_hi(of[e]), bf16_hi(of[e])));
                        }
                    }
                }
            }
        };
        if constexpr (HALF) {
            const int first = on ? 8 * g : 0;
            const float *c = &cos_of[warp][first], *s = &sin_of[warp][first];
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const float4 cs = *reinterpret_cast<const float4*>(c + 2 * e), sn = *reinterpret_cast<const float4*>(s + 2 * e);
                own[0][e] = pair_of(cs.x, cs.y);
                own[0][e + 1] = pair_of(cs.z, cs.w);
                other[0][e] = pair_of(-sn.x, -sn.y);
                other[0][e + 1] = pair_of(-sn.z, -sn.w);
                other[1][e] = pair_of(sn.x, sn.y);
                other[1][e + 1] = pair_of(sn.z, sn.w);
            }
        }
        bool of_k = first_pass * kHeads + in_pass >= p.Hq;
        factors(of_k ? p.k_weight : p.q_weight);

        // ---- heads of Q, then of K: this part's share of the passes ------------------------------------------------------------
        for (int i0 = first_pass; i0 < last_pass; i0 += kAhead) {
            if (i0 > first_pass) fetch(i0);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (i0 + u >= last_pass) break;
                const int h = (i0 + u) * kHeads + in_pass;
                if (NORM && !of_k && h >= p.Hq) {                    // (once a row)
                    of_k = true;
                    factors(p.k_weight);
                }
                uint64_t x[kLoads][4], r2 = 0;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) widen8(w[u][i], x[i]);
                if constexpr (NORM) {
                    uint64_t squares = 0;
#pragma unroll
                    for (int i = 0; i < kLoads; ++i)
                        squares = fma2(x[i][0], x[i][0], fma2(x[i][1], x[i][1], fma2(x[i][2], x[i][2], fma2(x[i][3], x[i][3], squares))));
                    float ss = sum2(squares);
#pragma unroll
                    for (int d = LANES / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
                    const float r = rsqrtf(fmaf(ss, inv, p.eps));
                    r2 = pair_of(r, r);
                }
                if constexpr (HALF && NORM)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint64_t m[4];
                        widen8(weight_of[i], m);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[i][e] = mul2(x[i][e], m[e]);
                    }
                const bool in = on && h < heads;
                uint16_t* dst = (h < p.Hq ? q_out : k_out) + h * p.D;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    uint64_t o[4];
                    if constexpr (HALF) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = fma2(x[1 - i][e], other[i][e], mul2(x[i][e], own[0][e]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float a, b;
                            parts_of(x[i][e], a, b);
                            o[e] = fma2(pair_of(b, b), other[i][e], mul2(pair_of(a, a), own[i][e]));
                        }
                    }
                    if constexpr (NORM)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = mul2(o[e], r2);
                    if (in) *reinterpret_cast<uint4*>(dst + i * apart) = round8(o);
                }
            }
        }
    }
}

template <int LANES, int EACH, bool HALF> static cudaError_t rotary_run(RotaryArgs& p, bool norm, cudaStream_t st) {
    // Warps to a row: what takes the fewest rounds of resident warps, an item as many turns as it has passes over heads and four more for
    // its angles (4000 rows of 48 heads of 128: one 23.1 us, two 19.9; 20 000 rows: one).
    constexpr int kBlocks = RotaryShape<LANES, EACH, HALF>::kBlocks;
    const int passes = ((p.Hq + p.Hk) * LANES + 31) / 32;
    const long long rows = (long long)p.B * p.cap, resident = (long long)kBlocks * kRotaryWarps * sm_count();
    long long least = 0x7fffffffffffffffLL;
    for (int log = 0; log <= 4 && (log == 0 || (1 << log) <= passes); ++log) {
        const long long cost = (((rows << log) + resident - 1) / resident) * ((passes + (1 << log) - 1) / (1 << log) + 4);
        if (cost >= least) continue;
        least = cost;
        p.parts_log = log;
    }
    const dim3 grid((unsigned)std::min(((rows << p.parts_log) + kRotaryWarps - 1) / kRotaryWarps, (long long)kBlocks * sm_count()));
    const dim3 block(kRotaryWarps * 32);
    return norm ? launch_overlapped(rotary_axes_kernel<LANES, EACH, HALF, true>, grid, block, 0, st, p)
                : launch_overlapped(rotary_axes_kernel<LANES, EACH, HALF, false>, grid, block, 0, st, p);
}

// Rows of [B, rows, H, D] with requests and rows apart.
static int check_heads(const void* at, int H, int D, long long batch, long long row) {
    if (!at || !aligned16(at) || row < (long long)H * D || batch < 0) return REGIONE_INVALID_ARG;
    return row % 8 || batch % 8 || row > (1LL << 32) || batch > (1LL << 48) ? REGIONE_UNSUPPORTED : REGIONE_OK;
}

}  // namespace regione

using namespace regione;

extern "C" int regione_rotary_axes(const regione_bf16* q, int64_t q_batch, int64_t q_row, const regione_bf16* k, int64_t k_batch,
                                   int64_t k_row, const int32_t* idx, const int32_t* n, const float* positions, int64_t positions_batch,
                                   int B, int n_pos, int cap, int Hq, int Hk, int D, int axes, int src_compact, const double* freq,
                                   const int32_t* axis, int rope_layout, int inverse, int normalise, const regione_bf16* q_weight,
                                   const regione_bf16* k_weight, float eps, regione_bf16* q_out, int64_t q_out_batch,
                                   int64_t q_out_row, regione_bf16* k_out, int64_t k_out_batch, int64_t k_out_row,
                                   int32_t* dev_status, void* stream) {
    if (!freq || !axis || B < 0 || n_pos < 0 || cap < 0 || Hq < 1 || Hk < 0 || D < 1 || axes < 1) return REGIONE_INVALID_ARG;
    if ((k != nullptr) != (Hk > 0) || (k != nullptr) != (k_out != nullptr)) return REGIONE_INVALID_ARG;
    if (rope_layout != REGIONE_ROPE_INTERLEAVED && rope_layout != REGIONE_ROPE_HALF) return REGIONE_INVALID_ARG;
    if (normalise ? !(eps >= 0.f) : q_weight || k_weight) return REGIONE_INVALID_ARG;
    if (inverse && normalise) return REGIONE_UNSUPPORTED;           // (the gradient of the rotation alone)
    if (!aligned16(q_weight) || !aligned16(k_weight) || positions_batch < 0) return REGIONE_INVALID_ARG;
    if (!idx && cap > n_pos) return REGIONE_INVALID_ARG;
    if ((long long)B * cap > 0x7ffffffLL) return REGIONE_UNSUPPORTED;
    if (D % 16 || D > kRotaryMaxD || axes > kRotaryAxes || Hq > 65536 || Hk > 65536 || B > 65535 || cap > (1 << 24) || n_pos > (1 << 28))
        return REGIONE_UNSUPPORTED;
    for (int i = 0; i < D / 2; ++i)
        if (axis[i] < 0 || axis[i] >= axes || !(std::fabs(freq[i]) <= 1e7)) return REGIONE_INVALID_ARG;
    if (B == 0 || cap == 0) return REGIONE_OK;
    if (!positions) return REGIONE_INVALID_ARG;
    int rc;
    if ((rc = check_heads(q, Hq, D, q_batch, q_row)) != REGIONE_OK || (rc = check_heads(q_out, Hq, D, q_out_batch, q_out_row)) != REGIONE_OK) return rc;
    if (k && ((rc = check_heads(k, Hk, D, k_batch, k_row)) != REGIONE_OK || (rc = check_heads(k_out, Hk, D, k_out_batch, k_out_row)) != REGIONE_OK)) return rc;
    if (B > 1 && (q_out_batch == 0 || (k && k_out_batch == 0))) return REGIONE_INVALID_ARG;   // (requests would write the same rows)
    RotaryArgs p = {};
    p.q = q; p.k = k; p.q_batch = q_batch; p.q_row = q_row; p.k_batch = k_batch; p.k_row = k_row;
    p.q_out = q_out; p.k_out = k_out; p.q_out_batch = q_out_batch; p.q_out_row = q_out_row; p.k_out_batch = k_out_batch; p.k_out_row = k_out_row;
    p.idx = idx; p.n = n; p.positions = positions; p.positions_batch = positions_batch;
    p.B = B; p.n_pos = n_pos; p.cap = cap; p.Hq = Hq; p.Hk = Hk; p.D = D; p.axes = axes; p.compact = src_compact || !idx;
    p.q_weight = q_weight; p.k_weight = k_weight; p.eps = eps; p.sign = inverse ? -1.0f : 1.0f; p.dev_status = dev_status;
    for (int i = 0; i < D / 2; ++i) {
        const double turns = freq[i] * 0.15915494309189533576888;   // 1 / (2 pi)
        p.turns_hi[i] = (float)turns;
        p.turns_lo[i] = (float)(turns - (double)p.turns_hi[i]);
        p.axis[i] = (uint8_t)axis[i];
    }
    const int pieces = D / 8, units = rope_layout == REGIONE_ROPE_HALF ? pieces / 2 : pieces;
    const bool norm = normalise != 0;
    cudaStream_t st = (cudaStream_t)stream;
    if (rope_layout == REGIONE_ROPE_HALF) {
        if (units <= 1) return launch_status(rotary_run<1, 1, true>(p, norm, st));
        if (units <= 2) return launch_status(rotary_run<2, 1, true>(p, norm, st));
        if (units <= 4) return launch_status(rotary_run<4, 1, true>(p, norm, st));
        if (units <= 8) return launch_status(rotary_run<8, 1, true>(p, norm, st));
        return launch_status(rotary_run<16, 1, true>(p, norm, st));
    }
    if (units == 6) return launch_status(rotary_run<2, 3, false>(p, norm, st));
    if (units == 12) return launch_status(rotary_run<4, 3, false>(p, norm, st));
    if (units == 24) return launch_status(rotary_run<8, 3, false>(p, norm, st));
    if (units <= 2) return launch_status(rotary_run<2, 1, false>(p, norm, st));
    if (units <= 4) return launch_status(rotary_run<4, 1, false>(p, norm, st));
    if (units <= 8) return launch_status(rotary_run<8, 1, false>(p, norm, st));
    if (units <= 16) return launch_status(rotary_run<16, 1, false>(p, norm, st));
    return launch_status(rotary_run<32, 1, false>(p, norm, st));
}
