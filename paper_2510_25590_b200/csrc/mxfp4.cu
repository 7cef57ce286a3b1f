// The 4-bit microscaled format: rows of bf16 to codes and scales and back, for the operands of the 4-bit product
// (regione_mxfp4_grouped_matmul) and for the Region-Instruction KV cache (Sec. 4 "Stabilization Stage" keeps K and V of every
// attention layer between full steps; the paper keeps them in the model's precision).
//
// 32 consecutive elements share a scale s = 2^k, stored as the byte k + 127 (E8M0); an element is a 4-bit E2M1 code (1 sign,
// 2 exponent, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6), two to a byte, the earlier one in the low half.
//   k = smallest integer with amax / 2^k <= 6; with amax = m * 2^e, m in [0.5, 1): k = e - 3 + (m > 0.75); k = 0 for amax = 0;
//   k is kept >= -127.  x / s is exact in fp32, so the only rounding is the one to E2M1, to nearest with ties to the even code;
//   (code value) * 2^k is exact in bf16.
//
// All of it is bound by device memory: 2 bytes an element on the bf16 side, 17 / 32 on the other.  A warp takes a task of up to
// kTask consecutive elements of one row, all of whose loads are on their way before the first is used, and the task's scales
// leave in one store of up to 32 bytes.  16384 x 8192 elements: there 48.8 us, back 52.2 (340 MB; 52.6 at the copy rate); K and V
// of 7885 rows of 24 x 128 stored in 20.7 us, widened in 20.8 (19.0).  A grid of four blocks an SM that walks over the tasks, with
// the next task's loads ahead of the work, takes half as long again: what hides the latency is the number of warps.
#include "common.cuh"

#include <algorithm>

namespace regione {

constexpr int kFp4Threads = 256;
constexpr int kFp4Unroll = 4;                        // widening: 8 elements to a lane and step
constexpr int kTask = 32 * 8 * kFp4Unroll;           // 1024 elements

struct Fp4Rows {
    const uint16_t* src[2];       // bf16 [B, src_rows, E]; one tensor, or K and V
    uint16_t* dst[2];             // bf16 [B, cap, E] (widening)
    uint8_t* codes[2];            // [B, cap, E / 2]
    uint8_t* scales[2];           // [B, cap, E / 32]
    const int32_t* idx;           // [B, cap] or NULL: row j
    const int32_t* n;             // [B] or NULL: every row
    int tensors;
    int segs;                     // tasks of a row
    long long src_rows, cap, E, tasks;
    int32_t* dev_status;
};

// Eight bf16 times a power of two `inv` (bf16, exact in fp32) -> eight E2M1 codes (round to nearest even, saturating), the first
// element in bits [3:0].
__device__ __forceinline__ uint32_t pack_e2m1x8(const uint32_t* w, uint32_t inv) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm("{.reg .b16 lo, hi, s, z;\n\t"
            "mov.b32 {lo, hi}, %2;\n\t"
            "mov.b32 {s, z}, %3;\n\t"
            "fma.rn.f32.bf16 %0, lo, s, %4;\n\t"
            "fma.rn.f32.bf16 %1, hi, s, %4;}"
            : "=f"(x[2 * i]), "=f"(x[2 * i + 1]) : "r"(w[i]), "r"(inv), "f"(-0.0f));
    uint32_t r;
    asm("{.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};}"
        : "=r"(r) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
    return r;
}
// Eight codes -> four packed pairs of half-precision values (exact).
__device__ __forceinline__ void unpack_e2m1x8(uint32_t codes, uint32_t h[4]) {
    asm("{.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
}
__device__ __forceinline__ float2 widen_f16x2(uint32_t h2) {
    float2 r;
    asm("{.reg .b16 l, h; mov.b32 {l, h}, %2; cvt.f32.f16 %0, l; cvt.f32.f16 %1, h;}" : "=f"(r.x), "=f"(r.y) : "r"(h2));
    return r;
}

// What a scale byte stands for: 2^(code - 127) (0: a subnormal), 255 a NaN.
__device__ __forceinline__ float scale_value(int code) {
    return __uint_as_float(code == 0 ? 0x00400000u : code < 255 ? (uint32_t)code << 23 : 0x7fc00000u);
}

// k + 127 of a block's scale from its largest magnitude as bf16 bits without their sign.  With exponent field E and seven mantissa
// bits M: e = E - 126 and m > 0.75 where M > 64, which adding 63 carries into E.  (Infinity saturates like the largest finite value; a
// subnormal maximum is below 6 * 2^-127 and ends at the floor.)
__device__ __forceinline__ int fp4_scale_code(uint32_t amax) {
    const int code = max((int)((min(amax, 0x7f7fu) + 63) >> 7) - 2, 0);
    return amax == 0 ? 127 : code;
}

// Per half: the larger magnitude, with some sign.  (A NaN element is ignored.)
__device__ __forceinline__ uint32_t max_magnitude_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// 32 bytes that are read once, in one load (WIDE: 32-byte aligned) or two.
template <bool WIDE> __device__ __forceinline__ void ld_stream256(const uint16_t* src, uint32_t* w) {
    if constexpr (WIDE) {
        asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(src));
    } else {
        const uint4 a = ldg128(src), b = ldg128(src + 8);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
}

// What a warp's task is: a tensor, its row of the source and of the destination, and the first element.  False: nothing to do.
struct Fp4Task {
    int tensor;
    long long src_row, dst_row, first;
};
__device__ __forceinline__ bool fp4_task(const Fp4Rows& p, long long at, int lane, Fp4Task& t) {
    if (at >= p.tasks) return false;
    const int per_row = p.tensors * p.segs;
    int in, b, j;
    if (p.tasks <= 0x7fffffffLL) {                      // (a division in 64 bits takes as long as the task's arithmetic)
        const uint32_t row = (uint32_t)at / (uint32_t)per_row;
        in = (int)((uint32_t)at - row * per_row);
        b = (int)(row / (uint32_t)p.cap);
        j = (int)(row - b * (uint32_t)p.cap);
        t.dst_row = row;
    } else {
        t.dst_row = at / per_row;
        in = (int)(at - t.dst_row * per_row);
        b = (int)(t.dst_row / p.cap);
        j = (int)(t.dst_row - b * p.cap);
    }
    t.tensor = in >= p.segs;
    t.first = (long long)(in - t.tensor * p.segs) * kTask;
    const int row = p.idx != nullptr ? p.idx[t.dst_row] : j;
    if (p.n != nullptr) {
        const int live = p.n[b];
        if ((live < 0 || live > p.cap) && j == 0 && in == 0 && lane == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
        if (j >= live) return false;
    }
    if (row < 0 || row >= p.src_rows) {
        if (lane == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
        return false;
    }
    t.src_row = b * p.src_rows + row;
    return true;
}

// 16 elements to a lane: the arithmetic is 4 instructions an element, which at 80 % of the issue slots was what bounded the form with 8
// elements to a lane (7 an element; 16384 x 8192 in 65 us).
template <bool WIDE>
__global__ void __launch_bounds__(kFp4Threads) mxfp4_quantize_kernel(const Fp4Rows p) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    Fp4Task t;
    if (!fp4_task(p, (long long)blockIdx.x * (kFp4Threads / 32) + (threadIdx.x >> 5), lane, t)) return;
    const uint16_t* src = (t.tensor ? p.src[1] : p.src[0]) + t.src_row * p.E + t.first + lane * 16;
    const long long at = t.dst_row * p.E + t.first;
    uint8_t* codes = (t.tensor ? p.codes[1] : p.codes[0]) + at / 2 + lane * 8;
    const int live = (int)min((long long)kTask, p.E - t.first);          // elements, a multiple of 32
    uint32_t w[kTask / 512][8];
#pragma unroll
    for (int u = 0; u < kTask / 512; ++u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[u][i] = 0u;
        if (u * 512 + lane * 16 < live) ld_stream256<WIDE>(src + u * 512, w[u]);
    }
    int scale = 0;                                                      // of block `lane` of the task
#pragma unroll
    for (int u = 0; u < kTask / 512; ++u) {
        uint32_t m = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max_magnitude_bf16x2(m, w[u][i]);
        m = max_magnitude_bf16x2(m, __shfl_xor_sync(0xffffffffu, m, 1));
        const int code = fp4_scale_code(max(m & 0x7fffu, (m >> 16) & 0x7fffu));
        const uint32_t inv = (uint32_t)(254 - code) << 7;               // 2^(127 - code) as bf16; code is at most 253
        const int from = __shfl_sync(0xffffffffu, code, (lane & 15) * 2);
        if ((lane >> 4) == u) scale = from;
        uint2 q;
        q.x = pack_e2m1x8(w[u], inv);
        q.y = pack_e2m1x8(w[u] + 4, inv);
        if (u * 512 + lane * 16 < live) *reinterpret_cast<uint2*>(codes + u * 256) = q;
    }
    if (lane * 32 < live) (t.tensor ? p.scales[1] : p.scales[0])[at / 32 + lane] = (uint8_t)scale;
}

__global__ void __launch_bounds__(kFp4Threads) mxfp4_dequantize_kernel(const Fp4Rows p) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    Fp4Task t;
    if (!fp4_task(p, (long long)blockIdx.x * (kFp4Threads / 32) + (threadIdx.x >> 5), lane, t)) return;
    const int tensor = t.tensor;
    const long long at = t.dst_row * p.E + t.first;
    const uint8_t* codes = (tensor ? p.codes[1] : p.codes[0]) + at / 2;
    const uint8_t* scales = (tensor ? p.scales[1] : p.scales[0]) + at / 32;
    uint16_t* dst = (tensor ? p.dst[1] : p.dst[0]) + at;
    const int live = (int)min((long long)kTask, p.E - t.first);
    uint32_t q[kFp4Unroll];
#pragma unroll
    for (int u = 0; u < kFp4Unroll; ++u) {
        const int e = (u * 32 + lane) * 8;
        q[u] = e < live ? __ldcs(reinterpret_cast<const uint32_t*>(codes + e / 2)) : 0u;
    }
    const int mine = lane * 32 < live ? scales[lane] : 127;
#pragma unroll
    for (int u = 0; u < kFp4Unroll; ++u) {
        const float s = scale_value(__shfl_sync(0xffffffffu, mine, u * 8 + (lane >> 2)));
        uint32_t h[4];
        unpack_e2m1x8(q[u], h);
        const float2 a = widen_f16x2(h[0]), b = widen_f16x2(h[1]), c = widen_f16x2(h[2]), d = widen_f16x2(h[3]);
        uint4 w;
        w.x = pack_bf16x2(a.x * s, a.y * s); w.y = pack_bf16x2(b.x * s, b.y * s);
        w.z = pack_bf16x2(c.x * s, c.y * s); w.w = pack_bf16x2(d.x * s, d.y * s);
        const int e = (u * 32 + lane) * 8;
        if (e < live) *reinterpret_cast<uint4*>(dst + e) = w;
    }
}

// Rows that lie one behind the other and are all live are one long row.
static int launch_fp4_rows(bool quantize, Fp4Rows p, int B, cudaStream_t st) {
    if (B * std::max(p.cap, p.src_rows) > (1LL << 50) / p.E) return REGIONE_UNSUPPORTED;   // elements: nothing below passes 64 bits
    if (p.idx == nullptr && p.n == nullptr && p.src_rows == p.cap) {
        p.E *= p.cap * B;
        p.cap = p.src_rows = 1;
        B = 1;
    }
    const long long segs = (p.E + kTask - 1) / kTask;
    if (segs > 0x7fffffffLL / 2) return REGIONE_UNSUPPORTED;
    p.segs = (int)segs;
    p.tasks = (long long)B * p.cap * p.tensors * segs;
    const long long blocks = (p.tasks + kFp4Threads / 32 - 1) / (kFp4Threads / 32);
    if (blocks > 0x7fffffffLL) return REGIONE_UNSUPPORTED;
    const bool wide = ((reinterpret_cast<uintptr_t>(p.src[0]) | reinterpret_cast<uintptr_t>(p.src[1])) & 31) == 0;
    return launch_status(launch_overlapped(!quantize ? mxfp4_dequantize_kernel : wide ? mxfp4_quantize_kernel<true>
                                                                                      : mxfp4_quantize_kernel<false>,
                                           dim3((unsigned)blocks), dim3(kFp4Threads), 0, st, p));
}

}  // namespace regione

using namespace regione;

static int check_fp4_rows(const void* wide, const void* codes, const void* scales, int B, long long cap, long long K) {
    if (B < 0 || cap < 0 || K < 1) return REGIONE_INVALID_ARG;
    if (B > 0 && cap > 0 && (!wide || !codes || !scales)) return REGIONE_INVALID_ARG;
    if (!aligned16(wide) || !aligned16(codes)) return REGIONE_INVALID_ARG;
    return K % 32 || K > 0x7fffffffLL || cap > 0x7fffffffLL ? REGIONE_UNSUPPORTED : REGIONE_OK;
}

extern "C" int regione_mxfp4_quantize(const regione_bf16* x, const int32_t* idx, const int32_t* n, int B, int64_t src_rows,
                                      int64_t cap, int64_t K, uint8_t* codes, uint8_t* scales, int32_t* dev_status,
                                      void* stream) {
    const int rc = check_fp4_rows(x, codes, scales, B, cap, K);
    if (rc != REGIONE_OK) return rc;
    if (src_rows < 0 || (!idx && cap > src_rows)) return REGIONE_INVALID_ARG;
    if (src_rows > 0x7fffffffLL) return REGIONE_UNSUPPORTED;
    if (B == 0 || cap == 0) return REGIONE_OK;
    Fp4Rows p = {};
    p.src[0] = x; p.codes[0] = codes; p.scales[0] = scales;
    p.idx = idx; p.n = n; p.tensors = 1;
    p.src_rows = src_rows; p.cap = cap; p.E = K; p.dev_status = dev_status;
    return launch_fp4_rows(true, p, B, (cudaStream_t)stream);
}

extern "C" int regione_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, const int32_t* n, int B, int64_t cap,
                                        int64_t K, regione_bf16* x, int32_t* dev_status, void* stream) {
    const int rc = check_fp4_rows(x, codes, scales, B, cap, K);
    if (rc != REGIONE_OK) return rc;
    if (B == 0 || cap == 0) return REGIONE_OK;
    Fp4Rows p = {};
    p.dst[0] = x; p.codes[0] = const_cast<uint8_t*>(codes); p.scales[0] = const_cast<uint8_t*>(scales);
    p.n = n; p.tensors = 1;
    p.src_rows = p.cap = cap; p.E = K; p.dev_status = dev_status;
    return launch_fp4_rows(false, p, B, (cudaStream_t)stream);
}

static int check_fp4_cache(const void* k, const void* v, const void* k_q, const void* v_q, const void* k_scale,
                           const void* v_scale, const void* n, int B, int Nc_cap, int H, int D) {
    if (!k || !v || !k_q || !v_q || !k_scale || !v_scale || !n) return REGIONE_INVALID_ARG;
    if (B < 0 || Nc_cap < 0 || H < 1) return REGIONE_INVALID_ARG;
    if (D != 64 && D != 128) return REGIONE_UNSUPPORTED;
    if (!aligned16(k) || !aligned16(v) || !aligned16(k_q) || !aligned16(v_q)) return REGIONE_INVALID_ARG;
    return REGIONE_OK;
}

extern "C" int regione_rikv_store_mxfp4(const regione_bf16* k_full, const regione_bf16* v_full, const int32_t* keep_rows,
                                        const int32_t* n_keep, int B, int N_full, int Nc_cap, int H, int D, uint8_t* k_q,
                                        uint8_t* v_q, uint8_t* k_scale, uint8_t* v_scale, int32_t* dev_status,
                                        void* stream) {
    const int rc = check_fp4_cache(k_full, v_full, k_q, v_q, k_scale, v_scale, n_keep, B, Nc_cap, H, D);
    if (rc != REGIONE_OK) return rc;
    if (!keep_rows || N_full < 0) return REGIONE_INVALID_ARG;
    if (B == 0 || Nc_cap == 0) return REGIONE_OK;
    Fp4Rows p = {};
    p.src[0] = k_full; p.codes[0] = k_q; p.scales[0] = k_scale;
    p.src[1] = v_full; p.codes[1] = v_q; p.scales[1] = v_scale;
    p.idx = keep_rows; p.n = n_keep; p.tensors = 2;
    p.src_rows = N_full; p.cap = Nc_cap; p.E = (long long)H * D; p.dev_status = dev_status;
    return launch_fp4_rows(true, p, B, (cudaStream_t)stream);
}

extern "C" int regione_rikv_load_mxfp4(const uint8_t* k_q, const uint8_t* v_q, const uint8_t* k_scale,
                                       const uint8_t* v_scale, const int32_t* n_keep, int B, int Nc_cap, int H, int D,
                                       regione_bf16* k_cache, regione_bf16* v_cache, int32_t* dev_status, void* stream) {
    const int rc = check_fp4_cache(k_cache, v_cache, k_q, v_q, k_scale, v_scale, n_keep, B, Nc_cap, H, D);
    if (rc != REGIONE_OK) return rc;
    if (B == 0 || Nc_cap == 0) return REGIONE_OK;
    Fp4Rows p = {};
    p.dst[0] = k_cache; p.codes[0] = const_cast<uint8_t*>(k_q); p.scales[0] = const_cast<uint8_t*>(k_scale);
    p.dst[1] = v_cache; p.codes[1] = const_cast<uint8_t*>(v_q); p.scales[1] = const_cast<uint8_t*>(v_scale);
    p.n = n_keep; p.tensors = 2;
    p.src_rows = p.cap = Nc_cap; p.E = (long long)H * D; p.dev_status = dev_status;
    return launch_fp4_rows(false, p, B, (cudaStream_t)stream);
}
