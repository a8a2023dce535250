// Activations in 8 bits: groups of 32 neighbouring channels of a row share a power-of-two scale.  Device pieces shared by the kernels that
// write and read them.
//
//   a = max |x| of the group,  e = least integer with a <= M 2^e (M = 448 for E4M3, 127 for INT8), held to [-117, 119] / [-117, 121]
//   code = x 2^-e rounded to the 8-bit format (to nearest, ties to even; beyond +-M: +-M),  value = code 2^e,  scale byte = e + 127 (E8M0)
//
// A value has 4 (E4M3) or 7 (INT8) significant bits and, by the limits of e, is a finite and normal bf16 number or zero: reading back is exact,
// and so is a product with a bf16 number on the tensor cores.  (At the upper limit elements beyond 448 2^119 and 127 2^121, above 2.9e38,
// are held to it, since the next code times the scale would be infinite.)
// A group with an element that is not finite has scale byte 255 and codes 0; all of it reads back as NaN.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "gaconv.h"

namespace gaconv {

constexpr int kActGroup = GACONV_ACT_GROUP;
static_assert(kActGroup == 32, "lanes of four share a group of 32 channels");

// scale byte of a group from the bits of its largest magnitude (fp32 bits without the sign; NaN counts as large)
template <int FMT>
__device__ __forceinline__ int act_scale_byte(uint32_t a)
{
    constexpr uint32_t top = FMT == GACONV_ACT_E4M3 ? 0x600000u : 0x7e0000u;       // fraction of M: 448 = 1.75 2^8, 127 = 1.984375 2^6
    constexpr int bits = FMT == GACONV_ACT_E4M3 ? 8 : 6, hi = FMT == GACONV_ACT_E4M3 ? 119 : 121;
    if (a >= 0x7f800000u) return 255;
    const int e = (int)(a >> 23) - 127 - bits + ((a & 0x7fffffu) > top ? 1 : 0);      // (subnormal: below the limit whatever the fraction)
    return min(max(e, -117), hi) + 127;
}
// 2^-e of a scale byte as a float (exact: a normal number), 0 for groups that are not finite
__device__ __forceinline__ float act_inverse(int byte) { return byte == 255 ? 0.f : __uint_as_float((uint32_t)(254 - byte) << 23); }

// four scaled values -> four codes.  A NaN (only where the scale is 0: Inf or NaN times 0) must be taken out by the caller.
template <int FMT>
__device__ __forceinline__ uint32_t act_encode4(float a, float b, float c, float d)
{
    if constexpr (FMT == GACONV_ACT_E4M3) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
        return lo | hi << 16;
    } else {
        auto q = [](float v) { return (uint32_t)__float2int_rn(fminf(fmaxf(v, -127.f), 127.f)) & 255u; };
        return q(a) | q(b) << 8 | q(c) << 16 | q(d) << 24;
    }
}

__device__ __forceinline__ uint32_t bf2_mul(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t bf2_sub(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// four codes -> their values times a power of two, bf16 pairs.  E4M3: the code's exponent and fraction moved to their places in a bf16 number stand
// for the value times 2^-120, subnormals included, and `scale2` (from act_scale2) makes up for it; the product is exact.  (Codes 0x7f and 0xff,
// which nothing here writes, give 480.)  INT8: 128 + the low seven bits, less 128 or, with the sign bit, 256: bf16 numbers from 128 to 256 are
// whole and put together by bits.
template <int FMT>
__device__ __forceinline__ uint2 act_decode4(uint32_t w, uint32_t scale2)
{
    uint2 v;
    if constexpr (FMT == GACONV_ACT_E4M3) {
        // (a byte's sign eight times above the byte: shifted by four the sign is in its place, and what is too much is masked)
        asm("prmt.b32 %0, %1, 0, 0x9180;" : "=r"(v.x) : "r"(w));
        asm("prmt.b32 %0, %1, 0, 0xb3a2;" : "=r"(v.y) : "r"(w));
        v.x = v.x << 4 & 0x87f087f0u;
        v.y = v.y << 4 & 0x87f087f0u;
    } else {
        const uint32_t lo = __byte_perm(w, 0, 0x4140), hi = __byte_perm(w, 0, 0x4342), base = 0x43004300u;
        v.x = bf2_sub(lo & 0x007f007fu | base, lo & 0x00800080u | base);
        v.y = bf2_sub(hi & 0x007f007fu | base, hi & 0x00800080u | base);
    }
    v.x = bf2_mul(v.x, scale2);
    v.y = bf2_mul(v.y, scale2);
    return v;
}
// The scale of a byte for act_decode4, twice, as bf16: 2^e for INT8, 2^(120 + e) for E4M3, of which bf16 has room for e up to 7; act_rest2 is
// what is left of larger ones, another factor.  Byte 255: codes are 0, and 0 times infinity, or times the rest NaN, is NaN.
template <int FMT>
__device__ __forceinline__ uint32_t act_scale2(uint32_t byte)
{
    return FMT == GACONV_ACT_E4M3 ? min(byte, 134u) * 0x00800080u + 0x3c003c00u : byte * 0x00800080u;
}
template <int FMT> __device__ __forceinline__ bool act_has_rest(uint32_t byte) { return FMT == GACONV_ACT_E4M3 && byte > 134; }
__device__ __forceinline__ uint32_t act_rest2(uint32_t byte) { return byte == 255 ? 0x7fc07fc0u : byte > 134 ? (byte - 134 + 127) * 0x00800080u : 0x3f803f80u; }
// Quantises N neighbouring elements; the 32 / N lanes of an aligned group of lanes hold the 32 channels of a group and call together, all lanes of
// the warp (elements past the row: 0).  Writes the codes, and from the first of these lanes the scale.  codes: the row's, at the elements;
// `pitch_left`: bytes of the row from there.
template <int FMT, int N>
__device__ __forceinline__ void act_store(const float (&v)[N], uint8_t* codes, int pitch_left, uint8_t* scale, bool first)
{
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) a = max(a, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < 32 / N; o *= 2) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
    if (pitch_left <= 0) return;
    const int byte = act_scale_byte<FMT>(a);
    const float inv = act_inverse(byte);
    uint32_t q[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        q[i] = act_encode4<FMT>(v[4 * i] * inv, v[4 * i + 1] * inv, v[4 * i + 2] * inv, v[4 * i + 3] * inv);
        if (byte == 255) q[i] = 0;
    }
    if constexpr (N == 8) *reinterpret_cast<uint2*>(codes) = make_uint2(q[0], q[1]);
    else *reinterpret_cast<uint32_t*>(codes) = q[0];
    if (first) *scale = (uint8_t)byte;
}

}  // namespace gaconv
