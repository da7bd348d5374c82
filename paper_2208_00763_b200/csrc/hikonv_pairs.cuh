// Arithmetic on pairs of floats in one register pair.
#pragma once

#include <cstdint>

namespace hikonv {

__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// v / s, rounded as the division is, by the rounded reciprocal y of s, for an s that divides_quickly and quotients in 2^-32 .. 2^32 (smaller ones come
// out small).
// Two steps after Markstein (Computation of elementary functions on the IBM RISC System/6000 processor, 1990): q' = q + (v - q s) / s, with the
// remainder by a fused multiply-add and 1 / s by its rounded value y.  The product v y is within 1.5 steps of v / s; after the first step
// q is off by at most 1/2 + 2^-22 steps u, its remainder is exact, and the second rounds v / s + e with |e| <= (1/2 + 2^-22) u s |1/s - y|.
// For s in [1, 2) that is below (1/2 + 2^-22) u s 2^-25, while v / s, a quotient of 24-bit numbers, lies at least u 2^-24 / s from any
// point between two floats: the same rounding for s^2 (1/2 + 2^-22) < 2, that is for all but the last few mantissas.  A zero comes out as +0.
__device__ __forceinline__ uint64_t quotient_pair(uint64_t v, uint64_t minus_s, uint64_t y) {
    uint64_t q = mul_pair(v, y);
    q = fma_pair(fma_pair(q, minus_s, v), y, q);
    return fma_pair(fma_pair(q, minus_s, v), y, q);
}
// Remainders far from underflow, and a mantissa at least sixteen steps below 2.
__device__ __forceinline__ bool divides_quickly(float s) {
    return s >= 0x1p-64f && s <= 0x1p64f && (__float_as_uint(s) & 0x7FFFF0u) != 0x7FFFF0u;
}

}  // namespace hikonv
