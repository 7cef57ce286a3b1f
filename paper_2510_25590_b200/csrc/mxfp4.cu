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
// kTask consecutive elements of one row: kUnroll loads a lane are on their way before the first is used, 8 elements to a lane (16
// bytes of bf16, 4 of codes), 4 lanes to a scale, and the task's scales leave in one store of up to 32 bytes.
#include "common.cuh"

#include <algorithm>

namespace regione {

constexpr int kFp4Threads = 256;
constexpr int kFp4Unroll = 4;
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

// Two fp32 -> two E2M1 codes (round to nearest even, saturating); `lo` lands in bits [3:0].
__device__ __forceinline__ uint32_t pack_e2m1x2(float lo, float hi) {
    uint32_t r;
    asm("{.reg .b8 c; cvt.rn.satfinite.e2m1x2.f32 c, %1, %2; cvt.u32.u8 %0, c;}" : "=r"(r) : "f"(hi), "f"(lo));
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

// 2^k, -149 <= k <= 127 (below -126 a subnormal).
__device__ __forceinline__ float pow2(int k) {
    return __uint_as_float(k >= -126 ? (uint32_t)(k + 127) << 23 : 1u << (k + 149));
}

// k + 127 of a block's scale from its largest magnitude as bf16 bits without their sign.  With exponent field E and seven mantissa
// bits M: e = E - 126 and m > 0.75 where M > 64.  (Infinity saturates like the largest finite value; a subnormal maximum is below
// 6 * 2^-127 and ends at the floor.)
__device__ __forceinline__ int fp4_scale_code(uint32_t amax) {
    if (amax == 0) return 127;
    amax = min(amax, 0x7f7fu);
    return max((int)(amax >> 7) - 2 + ((amax & 127) > 64 ? 1 : 0), 0);
}

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));      // (a NaN element is ignored)
    return r;
}

// What a warp's task is: a tensor, its row of the source and of the destination, and the first element.  False: nothing to do.
__device__ __forceinline__ bool fp4_task(const Fp4Rows& p, long long task, int lane, int& tensor, long long& src_row,
                                         long long& dst_row, long long& first) {
    const long long per_row = (long long)p.tensors * p.segs;
    dst_row = task / per_row;
    const int in = (int)(task - dst_row * per_row);
    tensor = in / p.segs;
    first = (long long)(in - tensor * p.segs) * kTask;
    const int b = (int)(dst_row / p.cap);
    const long long j = dst_row - b * p.cap;
    if (p.n != nullptr) {
        const int live = p.n[b];
        if ((live < 0 || live > p.cap) && j == 0 && in == 0 && lane == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
        if (j >= live) return false;
    }
    long long row = j;
    if (p.idx != nullptr) row = p.idx[dst_row];
    if (row < 0 || row >= p.src_rows) {
        if (lane == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
        return false;
    }
    src_row = b * p.src_rows + row;
    return true;
}

__global__ void __launch_bounds__(kFp4Threads) mxfp4_quantize_kernel(const Fp4Rows p) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    const long long task = (long long)blockIdx.x * (kFp4Threads / 32) + (threadIdx.x >> 5);
    if (task >= p.tasks) return;
    int tensor;
    long long src_row, dst_row, first;
    if (!fp4_task(p, task, lane, tensor, src_row, dst_row, first)) return;
    const uint16_t* src = (tensor ? p.src[1] : p.src[0]) + src_row * p.E + first;
    uint8_t* codes = (tensor ? p.codes[1] : p.codes[0]) + (dst_row * p.E + first) / 2;
    const int live = (int)min((long long)kTask, p.E - first);            // elements, a multiple of 32
    uint4 w[kFp4Unroll];
#pragma unroll
    for (int u = 0; u < kFp4Unroll; ++u) {
        const int e = (u * 32 + lane) * 8;
        w[u] = make_uint4(0u, 0u, 0u, 0u);
        if (e < live) w[u] = ld_stream128(src + e);
    }
    int mine = 0;                                                       // scale of block `lane` of the task
#pragma unroll
    for (int u = 0; u < kFp4Unroll; ++u) {
        constexpr uint32_t kAbs = 0x7fff7fffu;
        uint32_t m = max_bf16x2(max_bf16x2(w[u].x & kAbs, w[u].y & kAbs), max_bf16x2(w[u].z & kAbs, w[u].w & kAbs));
        m = max_bf16x2(m, 0u);                                           // (four pairs of NaN)
        m = max_bf16x2(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max_bf16x2(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const int code = fp4_scale_code(max(m & 0xffffu, m >> 16));
        const float inv = pow2(127 - code);
        const int from = __shfl_sync(0xffffffffu, code, (lane & 7) * 4);
        if ((lane >> 3) == u) mine = from;
        const uint32_t q = pack_e2m1x2(bf16_lo(w[u].x) * inv, bf16_hi(w[u].x) * inv) |
                           (pack_e2m1x2(bf16_lo(w[u].y) * inv, bf16_hi(w[u].y) * inv) << 8) |
                           (pack_e2m1x2(bf16_lo(w[u].z) * inv, bf16_hi(w[u].z) * inv) << 16) |
                           (pack_e2m1x2(bf16_lo(w[u].w) * inv, bf16_hi(w[u].w) * inv) << 24);
        const int e = (u * 32 + lane) * 8;
        if (e < live) *reinterpret_cast<uint32_t*>(codes + e / 2) = q;
    }
    if (lane * 32 < live) (tensor ? p.scales[1] : p.scales[0])[(dst_row * p.E + first) / 32 + lane] = (uint8_t)mine;
}

__global__ void __launch_bounds__(kFp4Threads) mxfp4_dequantize_kernel(const Fp4Rows p) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    const long long task = (long long)blockIdx.x * (kFp4Threads / 32) + (threadIdx.x >> 5);
    if (task >= p.tasks) return;
    int tensor;
    long long row, dst_row, first;
    if (!fp4_task(p, task, lane, tensor, row, dst_row, first)) return;
    const long long at = dst_row * p.E + first;
    const uint8_t* codes = (tensor ? p.codes[1] : p.codes[0]) + at / 2;
    const uint8_t* scales = (tensor ? p.scales[1] : p.scales[0]) + at / 32;
    uint16_t* dst = (tensor ? p.dst[1] : p.dst[0]) + at;
    const int live = (int)min((long long)kTask, p.E - first);
    uint32_t q[kFp4Unroll];
#pragma unroll
    for (int u = 0; u < kFp4Unroll; ++u) {
        const int e = (u * 32 + lane) * 8;
        q[u] = e < live ? __ldcs(reinterpret_cast<const uint32_t*>(codes + e / 2)) : 0u;
    }
    const int mine = lane * 32 < live ? scales[lane] : 127;
#pragma unroll
    for (int u = 0; u < kFp4Unroll; ++u) {
        const float s = pow2(__shfl_sync(0xffffffffu, mine, u * 8 + (lane >> 2)) - 127);
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
static int launch_fp4_rows(void (*kernel)(Fp4Rows), Fp4Rows p, int B, cudaStream_t st) {
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
    return launch_status(launch_overlapped(kernel, dim3((unsigned)blocks), dim3(kFp4Threads), 0, st, p));
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
    return launch_fp4_rows(mxfp4_quantize_kernel, p, B, (cudaStream_t)stream);
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
    return launch_fp4_rows(mxfp4_dequantize_kernel, p, B, (cudaStream_t)stream);
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
    return launch_fp4_rows(mxfp4_quantize_kernel, p, B, (cudaStream_t)stream);
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
    return launch_fp4_rows(mxfp4_dequantize_kernel, p, B, (cudaStream_t)stream);
}
