// What the kernels of the linear layers share: reading codes, groups of rows, and the epilogue.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "hikonv_cuda.cuh"
#include "hikonv_linear.h"

namespace hikonv {

// Row range of a group, whatever the offsets say: within 0 .. M, and empty where it would end before it begins.
__device__ __forceinline__ int2 group_rows(const LinearParams &p, int e) {
    if (!p.offsets) return make_int2(0, p.M);
    const int a = min(max(load_ordered(p.offsets + e), 0), p.M), b = min(max(load_ordered(p.offsets + e + 1), 0), p.M);
    return make_int2(a, max(a, b));
}

// `bytes` (0 .. 4 W) bytes from any address, as W words whose other bytes are zero or stray neighbours.  Only aligned words that hold at
// least one of the wanted bytes are read.
template <int W>
__device__ __forceinline__ void load_bytes(const uint8_t *src, int bytes, uint32_t (&out)[W]) {
    const uint32_t off = (uint32_t)(uintptr_t)src & 3u;
    const uint32_t *base = reinterpret_cast<const uint32_t *>(src - off);
    const int words = bytes > 0 ? (int)(off + bytes + 3) >> 2 : 0;
    uint32_t v[W + 1];
#pragma unroll
    for (int i = 0; i <= W; ++i) v[i] = i < words ? load_ordered(base + i) : 0u;
#pragma unroll
    for (int i = 0; i < W; ++i) out[i] = __funnelshift_r(v[i], v[i + 1], off * 8);
}

// Dense codes to one per byte.  Unsigned codes take their value; signed ones go to the upper bits of their byte, where the sign
// is the byte's (their value times 2^(8 - b): the sums are shifted back once at the end, exactly), which saves the sign extension.
// UP: 0xF0F0F0F0-like masks and left shifts; the codes of a word come in order.
template <bool UP>
__device__ __forceinline__ void unpack4(uint32_t w, uint32_t (&out)[2]) {
    const uint32_t even = UP ? (w << 4) & 0xF0F0F0F0u : w & 0x0F0F0F0Fu, odd = UP ? w & 0xF0F0F0F0u : (w >> 4) & 0x0F0F0F0Fu;
    out[0] = byte_permute(even, odd, 0x5140);
    out[1] = byte_permute(even, odd, 0x7362);
}
template <bool UP>
__device__ __forceinline__ void unpack2(uint32_t w, uint32_t (&out)[4]) {
    uint32_t c[4];                                     // c[i]: codes i, i + 4, i + 8, i + 12
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = UP ? (w << (6 - 2 * i)) & 0xC0C0C0C0u : (w >> (2 * i)) & 0x03030303u;
    const uint32_t a0 = byte_permute(c[0], c[1], 0x5140), a1 = byte_permute(c[0], c[1], 0x7362);
    const uint32_t b0 = byte_permute(c[2], c[3], 0x5140), b1 = byte_permute(c[2], c[3], 0x7362);
    out[0] = byte_permute(a0, b0, 0x5410);
    out[1] = byte_permute(a0, b0, 0x7632);
    out[2] = byte_permute(a1, b1, 0x5410);
    out[3] = byte_permute(a1, b1, 0x7632);
}
// 16 codes in the low half of w.
template <bool UP>
__device__ __forceinline__ void unpack1(uint32_t w, uint32_t (&out)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // four copies of the nibble, one bit kept in each byte, moved to its place by a multiply: bit j of the nibble to bit 8 j
        const uint32_t n = (w >> (4 * i)) & 0xFu;
        const uint32_t spread = (n * 0x00204081u) & 0x01010101u;
        out[i] = UP ? spread << 7 : spread;
    }
}

// ---- epilogue

template <int OUT> struct OutElem { using type = float; };
template <> struct OutElem<HIKONV_OUT_SUMS> { using type = int32_t; };
template <> struct OutElem<HIKONV_OUT_CODES> { using type = uint8_t; };
template <> struct OutElem<HIKONV_OUT_F16> { using type = __half; };
template <> struct OutElem<HIKONV_OUT_BF16> { using type = __nv_bfloat16; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float v, float *o) { *o = v; }
__device__ __forceinline__ void from_float(float v, __half *o) { *o = __float2half_rn(v); }
__device__ __forceinline__ void from_float(float v, __nv_bfloat16 *o) { *o = __float2bfloat16_rn(v); }

// v / (1 + exp(-v)), for v < 0 as v exp(v) / (1 + exp(v)): no exponential overflows, so results down to the smallest normal numbers (v
// near -91.8) keep their bits.  The divisor d lies in [1, 2], so the quotient q of the approximate reciprocal (within 2^-23) needs one step after
// Markstein, q + (a - q d) / d, to be within 2^-20 of a step of the rounded one.  The remainder of infinity is a NaN, which fminf drops.
// 512 x 2048 x 4096 to fp32: 9.5 us, against 8.9 by an approximate division that loses results below v = -87.3 and 9.1 by the uncorrected
// product with the reciprocal; a library division, whose code for other divisors is called, spilled 27 registers of the tiled kernel.
__device__ __forceinline__ float silu(float v) {
    const float t = expf(-fabsf(v)), d = 1.f + t, a = v < 0.f ? v * t : v;
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
    const float q = a * r;
    return fmaf(fminf(fmaf(-q, d, a), 3e38f), r, q);
}
__device__ __forceinline__ float activate(float v, int act) {
    if (act == HIKONV_ACT_RELU) return v < 0.f ? 0.f : v;                      // a NaN stays
    if (act == HIKONV_ACT_SILU) return silu(v);
    if (act == HIKONV_ACT_GELU) return 0.5f * v * (1.f + erff(v * 0.70710678118654752f));
    return v;
}

// What a column of the output needs besides its sum.
struct ColumnTerms {
    float scale, bias;
    int32_t ibias;
};
template <int OUT>
__device__ __forceinline__ ColumnTerms column_terms(const LinearParams &p, int e, int n) {
    ColumnTerms c{1.f, 0.f, 0};
    const size_t at = (size_t)e * p.N + n;
    if (OUT == HIKONV_OUT_CODES) {
        if (p.bias) c.ibias = load_ordered((const int32_t *)p.bias + at);
    } else if (OUT != HIKONV_OUT_SUMS) {
        if (p.w_scale) c.scale = load_ordered(p.w_scale + at);
        if (p.bias) c.bias = load_ordered((const float *)p.bias + at);
    }
    return c;
}

// The value of one output from its sum (already shifted down by p.down).  ACT < 0: the activation is looked up as the kernel runs.
template <int OUT, int ACT = -1>
__device__ __forceinline__ typename OutElem<OUT>::type finish(const LinearParams &p, int32_t sum, float x_scale, const ColumnTerms &c,
                                                              float residual) {
    if constexpr (OUT == HIKONV_OUT_SUMS) {
        return sum;
    } else if constexpr (OUT == HIKONV_OUT_CODES) {
        const long long v = ((long long)sum + c.ibias) >> p.shift;
        return (uint8_t)(int)(v < p.lo ? p.lo : v > p.hi ? p.hi : v);
    } else {
        const float v = activate(fmaf((float)sum * x_scale, c.scale, c.bias), ACT < 0 ? p.act : ACT) + residual;
        typename OutElem<OUT>::type o;
        from_float(v, &o);
        return o;
    }
}
template <typename T>
__device__ __forceinline__ float residual_at(const LinearParams &p, long long m, int n) {
    if constexpr (std::is_same<T, int32_t>::value || std::is_same<T, uint8_t>::value) return 0.f;
    else return p.residual ? to_float(load_ordered((const T *)p.residual + m * p.res_row + n)) : 0.f;
}

// Calls f with the output type as a constant.
template <typename F>
__device__ __forceinline__ void with_out_type(int out_type, F f) {
    switch (out_type) {
        case HIKONV_OUT_SUMS: f(std::integral_constant<int, HIKONV_OUT_SUMS>()); break;
        case HIKONV_OUT_CODES: f(std::integral_constant<int, HIKONV_OUT_CODES>()); break;
        case HIKONV_OUT_F32: f(std::integral_constant<int, HIKONV_OUT_F32>()); break;
        case HIKONV_OUT_F16: f(std::integral_constant<int, HIKONV_OUT_F16>()); break;
        default: f(std::integral_constant<int, HIKONV_OUT_BF16>()); break;
    }
}
// ... and the activation (none for whole numbers).
template <typename F>
__device__ __forceinline__ void with_epilogue(const LinearParams &p, F f) {
    with_out_type(p.out_type, [&](auto kind) {
        if constexpr ((int)HIKONV_OUT_F32 > (int)decltype(kind)::value) {
            f(kind, std::integral_constant<int, HIKONV_ACT_NONE>());
        } else {
            switch (p.act) {
                case HIKONV_ACT_RELU: f(kind, std::integral_constant<int, HIKONV_ACT_RELU>()); break;
                case HIKONV_ACT_SILU: f(kind, std::integral_constant<int, HIKONV_ACT_SILU>()); break;
                case HIKONV_ACT_GELU: f(kind, std::integral_constant<int, HIKONV_ACT_GELU>()); break;
                default: f(kind, std::integral_constant<int, HIKONV_ACT_NONE>()); break;
            }
        }
    });
}

}  // namespace hikonv
