// Rotary positions: the angle and the rotation, shared by the rotation itself
// (rope.cu) and the append into a paged cache (paged.cu), so that both give
// the same bits.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace quartz {

// A frequency in radians per position as a fraction of a turn per position, in
// units of 2^-64 (whole turns dropped): freq = M 2^(E - 1075) with the 53-bit
// M, so M times 2^66 / (2 pi) in integers, shifted by 1077 - E.  Good to 2^-63
// of itself and one unit; and no 64-bit floating point, of which an SM does
// two operations a clock.
__device__ __forceinline__ uint64_t rope_unit(double freq)
{
    const uint64_t bits = static_cast<uint64_t>(__double_as_longlong(freq));
    const int e = static_cast<int>((bits >> 52) & 0x7FF), r = 1077 - (e ? e : 1);
    const uint64_t m = (bits & 0xFFFFFFFFFFFFFull) | (e ? 1ull << 52 : 0ull);
    constexpr uint64_t kTurn = 0xA2F9836E4E441529ull;  // 2^66 / (2 pi)
    const uint64_t lo = m * kTurn, hi = __umul64hi(m, kTurn);
    uint64_t u = 0;
    if (r >= 128) u = 0;
    else if (r >= 64) u = hi >> (r - 64);
    else if (r > 0) u = (lo >> r) | (hi << (64 - r));
    else if (r > -64) u = lo << -r;
    return bits >> 63 ? 0 - u : u;
}

// (scale cos, scale sin) of position times unit.  The product modulo 2^64 loses
// nothing: the angle is off by the unit's own error, |position| times at most
// 2^-63 of the frequency and 2^-64 turns (2^-28, what binary32 holds of an
// eighth of a turn, from position 2^35 on).  Whole quarter turns are
// taken off as integers, so that the binary32 argument of sine and cosine has
// 24 good bits of at most an eighth of a turn.  A product in binary32 would be
// off by 2^-24 of the angle itself: 0.008 radians at position 131072.
__device__ __forceinline__ float2 rope_cos_sin(int64_t position, uint64_t unit, float scale)
{
    const uint64_t angle = static_cast<uint64_t>(position) * unit;
    const uint64_t quarter = (angle + (1ull << 61)) >> 62;
    const int64_t rest = static_cast<int64_t>(angle - (quarter << 62));  // in [-2^61, 2^61)
    float s, c;
    sincospif(static_cast<float>(rest) * 1.0842021724855044e-19f, &s, &c);  // 2^-63: half turns
    const bool swap = quarter & 1, neg_c = (quarter + 1) & 2, neg_s = quarter & 2;
    const float cos_a = swap ? s : c, sin_a = swap ? c : s;
    return make_float2(__fmul_rn(neg_c ? -scale : scale, cos_a), __fmul_rn(neg_s ? -scale : scale, sin_a));
}

// One pair turned; cs = (cos, sin), sine negated for the transpose.  The
// operations are named, so that every kernel rounds alike.
__device__ __forceinline__ float2 rope_turn(float x1, float x2, float2 cs)
{
    return make_float2(__fmaf_rn(cs.x, x1, -__fmul_rn(cs.y, x2)), __fmaf_rn(cs.y, x1, __fmul_rn(cs.x, x2)));
}

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32(float v) { return v; }
template <> __device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }

// Two values side by side, each rounded to T (one conversion for both).
template <typename T> __device__ __forceinline__ uint32_t pack_pair(float a, float b);
template <> __device__ __forceinline__ uint32_t pack_pair<__half>(float a, float b)
{
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <> __device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}

}  // namespace quartz
