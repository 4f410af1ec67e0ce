// Device functions of the 8-bit integer operators: rows of 16- or 32-bit numbers, their largest magnitude, their codes.
#pragma once
#include "common.hpp"

namespace dymoe {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

// 16 bytes at an address of any alignment (rows of an odd number of 16-bit values)
typedef uint32_t any16_t __attribute__((ext_vector_type(4), aligned(2)));

__host__ __device__ inline long up_to(long v, long m) { return (v + m - 1) / m * m; }

// Eight consecutive values of a row, as loaded.
template <int DT> struct Raw8 { uint4 a; };
template <> struct Raw8<DYMOE_OUT_F32> { uint4 a, b; };

__host__ __device__ constexpr int dtype_bytes(int dt) { return dt == DYMOE_OUT_F32 ? 4 : 2; }

// values [col, col + 8) of a row of K; those behind its end are zero and are not read
template <int DT>
__device__ __forceinline__ Raw8<DT> load8(const char* row, long col, long K)
{
    Raw8<DT> r;
    const char* const p = row + col * dtype_bytes(DT);
    if (col + 8 <= K) {
        const u32x4_t v = *(const DYMOE_GLOBAL any16_t*)p;
        r.a = __builtin_bit_cast(uint4, v);
        if constexpr (DT == DYMOE_OUT_F32) {
            const u32x4_t w = *(const DYMOE_GLOBAL any16_t*)(p + 16);
            r.b = __builtin_bit_cast(uint4, w);
        }
        return r;
    }
    r.a = make_uint4(0, 0, 0, 0);
    if constexpr (DT == DYMOE_OUT_F32) {
        r.b = make_uint4(0, 0, 0, 0);
        const DYMOE_GLOBAL uint32_t* const e = (const DYMOE_GLOBAL uint32_t*)p;
        if (col + 0 < K) r.a.x = e[0];
        if (col + 1 < K) r.a.y = e[1];
        if (col + 2 < K) r.a.z = e[2];
        if (col + 3 < K) r.a.w = e[3];
        if (col + 4 < K) r.b.x = e[4];
        if (col + 5 < K) r.b.y = e[5];
        if (col + 6 < K) r.b.z = e[6];
    } else {
        const DYMOE_GLOBAL uint16_t* const e = (const DYMOE_GLOBAL uint16_t*)p;
        if (col + 0 < K) r.a.x = e[0];
        if (col + 1 < K) r.a.x |= (uint32_t)e[1] << 16;
        if (col + 2 < K) r.a.y = e[2];
        if (col + 3 < K) r.a.y |= (uint32_t)e[3] << 16;
        if (col + 4 < K) r.a.z = e[4];
        if (col + 5 < K) r.a.z |= (uint32_t)e[5] << 16;
        if (col + 6 < K) r.a.w = e[6];
    }
    return r;
}

// Largest magnitude, as the pattern of the values' own type: without its sign a pattern of an IEEE type orders as the number
// does, infinity behind the finite ones and NaN behind infinity.
template <int DT>
__device__ __forceinline__ uint32_t peak8(const Raw8<DT>& r, uint32_t m)
{
    if constexpr (DT == DYMOE_OUT_F32) {
        m = max(m, r.a.x & 0x7fffffffu); m = max(m, r.a.y & 0x7fffffffu);
        m = max(m, r.a.z & 0x7fffffffu); m = max(m, r.a.w & 0x7fffffffu);
        m = max(m, r.b.x & 0x7fffffffu); m = max(m, r.b.y & 0x7fffffffu);
        m = max(m, r.b.z & 0x7fffffffu); m = max(m, r.b.w & 0x7fffffffu);
        return m;
    } else {
        auto two = [](uint32_t a, uint32_t b) {
            return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a), __builtin_bit_cast(u16x2_t, b)));
        };
        m = two(m, r.a.x & 0x7fff7fffu);
        m = two(m, r.a.y & 0x7fff7fffu);
        m = two(m, r.a.z & 0x7fff7fffu);
        return two(m, r.a.w & 0x7fff7fffu);
    }
}

template <int DT>
__device__ __forceinline__ uint32_t peak_bits(uint32_t m)
{
    return DT == DYMOE_OUT_F32 ? m : max(m & 0xffffu, m >> 16);
}

template <int DT>
__device__ __forceinline__ float peak_value(uint32_t bits)
{
    if constexpr (DT == DYMOE_OUT_F32) return __uint_as_float(bits);
    else if constexpr (DT == DYMOE_OUT_F16) return (float)f16_from_bits(bits);
    else return bf16_bits_to_f32(bits);
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v)
{
    auto step = [](uint32_t a, uint32_t b) { return max(a, b); };
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, true));
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, true));
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// What a row's codes are made with.  code = rint(127 x / a), ties to even, of the real quotient: 127 x is exact in 32 bits for
// 16-bit x; r = 1 / a to an ulp, q0 = 127 x r is off by less than 2^-21 of itself, and a quotient of 16-bit numbers that is not
// halfway between two codes is further than 2^-20 of itself from there (its distance is a whole number of 1 / (2 a) once a and
// x are scaled to integers); one that is halfway is a number of 32 bits, which the correction q0 + (127 x - q0 a) r gives
// exactly.  (32-bit x: the quotient to an ulp, then the same rounding.)
struct RowQ {
    float a, r;
    int shift;        // binary exponent taken off a and x where 127 x could leave the range
};

// scale = a / 127 of the row's largest magnitude a; NaN if that is infinite or NaN (its codes are then 0)
__device__ __forceinline__ RowQ row_q(float a, float& scale)
{
    RowQ q;
    const bool finite = a < __builtin_inff();          // false for NaN
    scale = finite ? a / 127.0f : __builtin_nanf("");
    q.shift = 0;
    if (finite && a > 0.0f && !(a >= 0x1p-100f && a <= 0x1p100f)) q.shift = -(int)__builtin_amdgcn_frexp_expf(a);
    q.a = ldexpf(a, q.shift);
    q.r = finite && a > 0.0f ? __builtin_amdgcn_rcpf(q.a) : 0.0f;
    return q;
}

__device__ __forceinline__ uint32_t code_of(float x, const RowQ& q)
{
    const float t = 127.0f * x;
    const float q0 = t * q.r;
    const float e = fmaf(-q0, q.a, t);
    const float c = fmaf(e, q.r, q0);
    return __float_as_uint(c + 12582912.0f);       // 1.5 * 2^23: the sum's last bit weighs one
}

__device__ __forceinline__ uint32_t pack_codes(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3)
{
    const uint32_t lo = __builtin_amdgcn_perm(c1, c0, 0x0c0c0400u), hi = __builtin_amdgcn_perm(c3, c2, 0x0c0c0400u);
    return lo | (hi << 16);
}

template <int DT>
__device__ __forceinline__ uint2 codes8(const Raw8<DT>& v, const RowQ& q)
{
    float f[8];
    if constexpr (DT == DYMOE_OUT_F32) {
        const uint32_t u[8] = {v.a.x, v.a.y, v.a.z, v.a.w, v.b.x, v.b.y, v.b.z, v.b.w};
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = __uint_as_float(u[i]);
    } else {
        const uint32_t u[4] = {v.a.x, v.a.y, v.a.z, v.a.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if constexpr (DT == DYMOE_OUT_F16) {
                const half2_t h = __builtin_bit_cast(half2_t, u[i]);
                f[2 * i] = (float)h[0];
                f[2 * i + 1] = (float)h[1];
            } else {
                f[2 * i] = bf16_lo(u[i]);
                f[2 * i + 1] = bf16_hi(u[i]);
            }
        }
    }
    if (q.shift != 0) {
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = ldexpf(f[i], q.shift);
    }
    uint2 o;
    o.x = pack_codes(code_of(f[0], q), code_of(f[1], q), code_of(f[2], q), code_of(f[3], q));
    o.y = pack_codes(code_of(f[4], q), code_of(f[5], q), code_of(f[6], q), code_of(f[7], q));
    if (q.r == 0.0f) o = make_uint2(0, 0);
    return o;
}

// One value in a type of the outputs
__device__ __forceinline__ void store_out(void* y, long at, int dt, float v)
{
    if (dt == DYMOE_OUT_F32) ((DYMOE_GLOBAL float*)y)[at] = v;
    else if (dt == DYMOE_OUT_F16) ((DYMOE_GLOBAL _Float16*)y)[at] = (_Float16)v;
    else ((DYMOE_GLOBAL __bf16*)y)[at] = (__bf16)v;
}

}  // namespace dymoe
