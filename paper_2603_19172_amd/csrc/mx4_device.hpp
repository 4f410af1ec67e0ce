// Device functions of the microscaled 4-bit format: numbers of one sign, two exponent and one fraction bit (0, 0.5, 1, 1.5, 2, 3, 4, 6), in
// blocks of 32 with a common power of two in a byte (2^(byte - 127); 255: no number).
#pragma once
#include "int8_device.hpp"

namespace dymoe {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

// The exponent byte of a block whose largest magnitude has the fp32 pattern `a`: floor(log2 a) - 2 = (a >> 23) - 127 - 2, so that the largest
// value lies in [4, 8) times the power of two; at least 2^-127 (subnormal peaks and blocks of zeros), 255 for infinity and NaN.
__device__ __forceinline__ uint32_t mx4_exponent(uint32_t a)
{
    const int e = (int)(a >> 23);
    return e == 255 ? 255u : (uint32_t)max(e - 2, 0);
}

// The power of two as the conversion instructions take it (their scale; 2^-127 is a subnormal fp32)
__device__ __forceinline__ float mx4_unit(uint32_t byte) { return __uint_as_float(byte == 0 ? 0x00400000u : byte << 23); }

// Codes of eight values, the first in the lowest four bits: x / unit to the nearest, ties to even, magnitudes beyond 6 to 6, with x's
// sign.  The conversion instructions round so for every input; of a block that is no number all codes are 0.
template <int DT>
__device__ __forceinline__ uint32_t mx4_codes8(const Raw8<DT>& v, uint32_t byte)
{
    const float unit = mx4_unit(byte);
    uint32_t q = 0;
    if constexpr (DT == DYMOE_OUT_F32) {
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v.a.x), __uint_as_float(v.a.y), unit, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v.a.z), __uint_as_float(v.a.w), unit, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v.b.x), __uint_as_float(v.b.y), unit, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v.b.z), __uint_as_float(v.b.w), unit, 3);
    } else if constexpr (DT == DYMOE_OUT_F16) {
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, __builtin_bit_cast(half2_t, v.a.x), unit, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, __builtin_bit_cast(half2_t, v.a.y), unit, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, __builtin_bit_cast(half2_t, v.a.z), unit, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, __builtin_bit_cast(half2_t, v.a.w), unit, 3);
    } else {
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2_t, v.a.x), unit, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2_t, v.a.y), unit, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2_t, v.a.z), unit, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2_t, v.a.w), unit, 3);
    }
    return byte == 255u ? 0u : q;
}

// The largest of four neighbouring lanes'
__device__ __forceinline__ uint32_t quad_max_u32(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
}

// fp32 pattern of the magnitude that peak8 found
template <int DT>
__device__ __forceinline__ uint32_t peak_f32_bits(uint32_t m) { return __float_as_uint(peak_value<DT>(peak_bits<DT>(m))); }

// 8 and 16 bytes at an address of any alignment (rows of an odd number of 16-bit values), stored at once
typedef uint32_t any8_t __attribute__((ext_vector_type(2), aligned(2)));

// Four neighbouring outputs of a row, `left` of them inside it
__device__ __forceinline__ void store_any4(void* out, long at, int dt, int left, const float (&v)[4])
{
    if (left < 4) {
#pragma unroll
        for (int i = 0; i < 3; i++)
            if (i < left) store_out(out, at + i, dt, v[i]);
    } else if (dt == DYMOE_OUT_F32) {
        *(DYMOE_GLOBAL any16_t*)((float*)out + at) = any16_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    } else if (dt == DYMOE_OUT_F16) {
        *(DYMOE_GLOBAL any8_t*)((uint16_t*)out + at) = any8_t{pack_half2(v[0], v[1]), pack_half2(v[2], v[3])};
    } else {
        const bf16x2_t a = {(__bf16)v[0], (__bf16)v[1]}, b = {(__bf16)v[2], (__bf16)v[3]};
        *(DYMOE_GLOBAL any8_t*)((uint16_t*)out + at) = any8_t{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
    }
}

// byte of a tile-layout matrix that holds code (row, col), col a multiple of 2; and that of the exponent of the block of (row, col)
__device__ __forceinline__ long mx4_tile_byte(long row, long col, long Kp)
{
    const long tile = (row >> 5) * (Kp >> 8) + (col >> 8);
    const int in = (int)(col & 255);
    return tile * 4096 + ((in & 127) >> 5) * 1024 + ((in >> 7) * 32 + (row & 31)) * 16 + (in & 31) / 2;
}
__device__ __forceinline__ long mx4_tile_exponent(long row, long col, long Kp)
{
    const long tile = (row >> 5) * (Kp >> 8) + (col >> 8);
    const int in = (int)(col & 255);
    return tile * 256 + ((in >> 7) * 32 + (row & 31)) * 4 + ((in & 127) >> 5);
}

// 4 bytes a lane, global memory -> LDS[lds_addr_lane0 + 4 * lane]: lds_copy16's smaller brother
__device__ __forceinline__ void lds_copy4(const char* base, uint32_t lane_offset, uint32_t lds_addr_lane0)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                 :
                 : "s"(lds_addr_lane0), "v"(lane_offset), "s"(base)
                 : "memory");
}

// v_mfma_scale_f32_32x32x64_f8f6f4 on 4-bit numbers: lane l holds 32 numbers of row l % 32 of either operand and, in byte A or B of a
// register, their exponent.  A block's products and their sum are exact.  The
// accumulator takes the first half of the lanes' block, then the second half's, rounded to the nearest each time; before that it is cut at 2^-24 of the
// largest power of two of a product, 0.5 counted as 1 (beside 16 and -16, 2^-20 comes through and 2^-21 does not; beside 0.25 and -0.25, 2^-24 and
// 2^-25; a second block beside a first one whose products cancel is not cut).
template <int A, int B>
__device__ __forceinline__ float16_t mfma_mx4(const uint4 a, const uint4 b, const float16_t c, uint32_t sa, uint32_t sb)
{
    const i32x8_t x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, A, (int)sa, B, (int)sb);
}

}  // namespace dymoe
