// Two fp32 operations in one instruction, and pairs of bf16 numbers as such.
#pragma once

#include "common.cuh"

namespace regione {

__device__ __forceinline__ uint64_t pair_of(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void parts_of(uint64_t p, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(p)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Two bf16 numbers of a word, the lower one first, and back (round to nearest even).
__device__ __forceinline__ uint64_t widen2(uint32_t w) { return pair_of(bf16_lo(w), bf16_hi(w)); }
__device__ __forceinline__ uint32_t round2(uint64_t p) {
    float x, y;
    parts_of(p, x, y);
    return pack_bf16x2(x, y);
}
__device__ __forceinline__ float sum2(uint64_t p) {
    float x, y;
    parts_of(p, x, y);
    return x + y;
}
// Eight of them.
__device__ __forceinline__ void widen8(const uint4& w, uint64_t (&x)[4]) {
    x[0] = widen2(w.x); x[1] = widen2(w.y); x[2] = widen2(w.z); x[3] = widen2(w.w);
}
__device__ __forceinline__ uint4 round8(const uint64_t (&x)[4]) { return make_uint4(round2(x[0]), round2(x[1]), round2(x[2]), round2(x[3])); }

}  // namespace regione
