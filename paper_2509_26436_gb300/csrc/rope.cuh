// Rotary positions: the angle and the rotation, shared by the rotation itself
// (rope.cu) and the append into a paged cache (paged.cu), so that both give
// the same bits.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace quartz {

// (scale cos, scale sin) of position * freq radians.  freq / 2 pi becomes a
// fraction of a turn in units of 2^-64, and position times that, modulo 2^64,
// is the angle's fraction of a turn without rounding: the only errors are the
// frequency's (2^-53 relative, from its 64-bit type and the division by 2 pi:
// 2^-33 turns at position 2^20 and one radian per position) and the last
// conversion's.  Whole quarter turns are taken off as integers, so that the
// binary32 argument of sine and cosine has 24 good bits of at most an eighth
// of a turn.  A product in binary32 would be off by 2^-24 of the angle itself:
// 0.008 radians at position 131072.
__device__ __forceinline__ float2 rope_cos_sin(int64_t position, double freq, float scale)
{
    double turn = freq * 0.15915494309189533577;  // 1 / (2 pi)
    turn -= floor(turn);
    const uint64_t unit = static_cast<uint64_t>(turn * 18446744073709551616.0);
    const uint64_t angle = static_cast<uint64_t>(position) * unit;
    const uint64_t quarter = (angle + (1ull << 61)) >> 62;
    const int64_t rest = static_cast<int64_t>(angle - (quarter << 62));  // in [-2^61, 2^61)
    float s, c;
    sincospif(static_cast<float>(rest) * 1.0842021724855044e-19f, &s, &c);  // 2^-63: half turns
    float cos_a, sin_a;
    switch (quarter & 3) {
        case 0: cos_a = c, sin_a = s; break;
        case 1: cos_a = -s, sin_a = c; break;
        case 2: cos_a = -c, sin_a = -s; break;
        default: cos_a = s, sin_a = -c; break;
    }
    return make_float2(__fmul_rn(scale, cos_a), __fmul_rn(scale, sin_a));
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

}  // namespace quartz
