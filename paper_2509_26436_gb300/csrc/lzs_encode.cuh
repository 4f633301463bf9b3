// Device side of the symmetric encoder (Section 3, Eq. 1 then Eq. 2): 16
// consecutive elements per lane, four lanes per 64-element group.  Shared by
// the encoder of whole tensors and the append into a paged cache.
#pragma once

#include <cstdint>
#include <cuda_fp16.h>

#include "ptx.cuh"

namespace quartz {

__device__ __forceinline__ uint4 ldg_stream(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

// Adding 1.5 * 2^23 to a float of magnitude below 2^22 rounds it to an
// integer (round-to-nearest-even, the rounding of the addition) and leaves
// that integer in the low mantissa bits: for 0 <= n < 256 the low byte of the
// sum's bit pattern is n.
constexpr float kRoundAddend = 12582912.0f;

// a * b on float pairs, rounded to nearest even (PTX mul.rn.f32x2).
__device__ __forceinline__ float2 mul2_rn(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\t"
        "mov.b64 a, {%2, %3};\n\t"
        "mov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 d, a, b;\n\t"
        "mov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

// Per byte: m (0..7) with the sign s (0x00 or 0xFF) applied in 4-bit two's
// complement: m for s = 0, (16 - m) & 15 for s = 0xFF.
__device__ __forceinline__ uint32_t signed_nibbles(uint32_t m, uint32_t s)
{
    return ((m ^ (s & 0x0F0F0F0Fu)) + (s & 0x01010101u)) & 0x0F0F0F0Fu;
}

// Eq. 2 codes of 8 elements given as four fp16 pairs `w` (the raw words) and
// their sign-cleared copies `a`: q = rne(x r) (capped at +-127 when CAP), c =
// sgn(q) (|q| >> flag), packed as 8 nibbles, element k in bits 4k..4k+3.
template <bool CAP>
__device__ __forceinline__ uint32_t lzs_word8(const uint32_t *w, const uint32_t *a, float r, int flag)
{
    uint32_t u[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&a[i]));
        float2 t = mul2_rn(f, make_float2(r, r));
        if (CAP) {
            t.x = fminf(t.x, 127.0f);
            t.y = fminf(t.y, 127.0f);
        }
        // Two scalar additions: a paired multiply followed by a paired add
        // was observed to be fused into one multiply-add (parity tests
        // failed on exact ties of x r), which rounds the unrounded product.
        const float2 m = make_float2(__fadd_rn(t.x, kRoundAddend), __fadd_rn(t.y, kRoundAddend));
        u[i][0] = __float_as_uint(m.x);
        u[i][1] = __float_as_uint(m.y);
    }
    // byte k of ev / od: |q| of element 2k / 2k + 1
    const uint32_t ev = prmt(prmt(u[0][0], u[1][0], 0x0040u), prmt(u[2][0], u[3][0], 0x0040u), 0x5410u);
    const uint32_t od = prmt(prmt(u[0][1], u[1][1], 0x0040u), prmt(u[2][1], u[3][1], 0x0040u), 0x5410u);
    // byte k of sev / sod: 0xFF when element 2k / 2k + 1 is negative (a
    // selector nibble 8 + b replicates the sign bit of byte b)
    const uint32_t sev = prmt(prmt(w[0], w[1], 0x00D9u), prmt(w[2], w[3], 0x00D9u), 0x5410u);
    const uint32_t sod = prmt(prmt(w[0], w[1], 0x00FBu), prmt(w[2], w[3], 0x00FBu), 0x5410u);
    const uint32_t keep = 0x01010101u * (0xFFu >> flag);
    const uint32_t cev = signed_nibbles((ev >> flag) & keep, sev);
    const uint32_t cod = signed_nibbles((od >> flag) & keep, sod);
    return cev | (cod << 4);
}

__device__ __forceinline__ int lzs_flag_of(float amax_sub, float r)
{
    const int qmax = min(__float2int_rn(__fmul_rn(amax_sub, r)), 127);
    return max(29 - __clz(qmax), 0);
}

// 16-element units per LZS subgroup (G_s >= 16).
template <int GS>
__host__ __device__ constexpr int kUnitsPerSub()
{
    return GS >= 16 ? GS / 16 : 1;
}

// Eq. 1 + Eq. 2 on the 16 elements of one unit (lo, hi: eight fp16 pairs):
// the group scale and, per 8-element half, the FLAG and the eight codes.  All
// 32 lanes must call it together (group and subgroup maxima are shuffles).
struct UnitCodes {
    uint32_t c0, c1;   // codes of elements 0-7 and 8-15 (element k in bits 4k..4k+3)
    int flag0, flag1;  // their FLAGs (equal unless G_s = 8)
    int flag_next;     // G_s >= 16: FLAG of the next subgroup (packed FLAG storage)
    __half s16;        // the group's fp16 scale
};

template <int GS>
__device__ __forceinline__ UnitCodes encode_unit_sym(const uint4 lo, const uint4 hi)
{
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    uint32_t a[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = w[i] & 0x7FFF7FFFu;
    // --- maxima of |x|: each 8-element half, the unit, the group ----------
    __half2 m0 = __hmax2(__hmax2(*reinterpret_cast<const __half2 *>(&a[0]), *reinterpret_cast<const __half2 *>(&a[1])),
                         __hmax2(*reinterpret_cast<const __half2 *>(&a[2]), *reinterpret_cast<const __half2 *>(&a[3])));
    __half2 m1 = __hmax2(__hmax2(*reinterpret_cast<const __half2 *>(&a[4]), *reinterpret_cast<const __half2 *>(&a[5])),
                         __hmax2(*reinterpret_cast<const __half2 *>(&a[6]), *reinterpret_cast<const __half2 *>(&a[7])));
    const float2 f0 = __half22float2(m0), f1 = __half22float2(m1);
    const float sub0 = fmaxf(f0.x, f0.y), sub1 = fmaxf(f1.x, f1.y);
    const float unit_max = fmaxf(sub0, sub1);
    const float pair_max = fmaxf(unit_max, __shfl_xor_sync(0xffffffffu, unit_max, 1));
    const float amax = fmaxf(pair_max, __shfl_xor_sync(0xffffffffu, pair_max, 2));

    // --- Eq. 1: scale and reciprocal (as the per-element path) ------------
    UnitCodes u;
    u.s16 = __float2half_rn(__fdiv_rn(amax, 127.0f));
    const float s = __half2float(u.s16);
    const float r = (s > 0.f) ? __frcp_rn(s) : 0.f;

    // --- Eq. 2: FLAG of each subgroup from its maximum --------------------
    if (GS == 8) {
        u.flag0 = lzs_flag_of(sub0, r);
        u.flag1 = lzs_flag_of(sub1, r);
    } else {
        const float m = GS == 16 ? unit_max : GS == 32 ? pair_max : amax;
        u.flag0 = u.flag1 = lzs_flag_of(m, r);
    }
    if (__float2int_rn(__fmul_rn(amax, r)) > 127) {  // only when the fp16 scale rounded far down
        u.c0 = lzs_word8<true>(w, a, r, u.flag0);
        u.c1 = lzs_word8<true>(w + 4, a + 4, r, u.flag1);
    } else {
        u.c0 = lzs_word8<false>(w, a, r, u.flag0);
        u.c1 = lzs_word8<false>(w + 4, a + 4, r, u.flag1);
    }
    u.flag_next = 0;
    if (GS >= 16) u.flag_next = __shfl_down_sync(0xffffffffu, u.flag0, kUnitsPerSub<GS>());
    return u;
}

// Store one unit's FLAGs: one byte per subgroup, or (packed) two per byte,
// subgroup 2j in the low nibble of byte j; a packed byte is written by the
// lane holding its first subgroup.
template <int GS>
__device__ __forceinline__ void store_unit_flags(const UnitCodes &u, int64_t unit, int lane,
                                                 uint8_t *__restrict__ flags, bool packed)
{
    constexpr int ups = kUnitsPerSub<GS>();
    if (GS == 8) {
        if (packed)
            flags[unit] = static_cast<uint8_t>(u.flag0 | (u.flag1 << 4));
        else
            reinterpret_cast<uint16_t *>(flags)[unit] = static_cast<uint16_t>(u.flag0 | (u.flag1 << 8));
    } else if (packed) {
        if ((lane & (2 * ups - 1)) == 0) flags[unit / (2 * ups)] = static_cast<uint8_t>(u.flag0 | (u.flag_next << 4));
    } else if ((lane & (ups - 1)) == 0) {
        flags[unit / ups] = static_cast<uint8_t>(u.flag0);
    }
}

// Store one unit's encoding: codes, FLAGs, and the scale once per group.
template <int GS>
__device__ __forceinline__ void store_unit_sym(const UnitCodes &u, int64_t unit, int lane,
                                               uint2 *__restrict__ codes, uint8_t *__restrict__ flags,
                                               __half *__restrict__ scales, bool packed)
{
    codes[unit] = make_uint2(u.c0, u.c1);
    store_unit_flags<GS>(u, unit, lane, flags, packed);
    if ((lane & 3) == 0) scales[unit >> 2] = u.s16;
}

}  // namespace quartz
