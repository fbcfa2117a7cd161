// 4-bit matrices: layout, and the conversions and matrix instruction on them.
//
// A matrix [rows][K] is held in fragments of the 32x32x64 matrix instruction,
// so that every reader loads 1 KiB of neighbouring bytes and no product needs
// to rearrange anything:
//   codes  [row tile of 32][k-step of 64][64 lanes][16 bytes]: lane l holds
//          row l%32, elements 32(l/32) .. +31 of the k-step, one block of 32,
//          element e in nibble e%8 of dword e/8;
//   scales [row tile][group of 4 k-steps][64 lanes][4 bytes]: byte s is the
//          scale of lane l's block in k-step s of the group (2^(byte - 127)),
//          so the instruction picks a k-step's scale by its byte select.
// Rows and elements past the matrix are zeros of scale 1.
#pragma once

#include "device.hpp"
#include "internal.hpp"

namespace tpk {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// fp4 x fp4 with a scale per 32, 32x32 += 32x64 * 64x32; S: which byte of the
// scales.  D: lane l holds column l%32, register i row 8(i/4) + 4(l/32) + i%4.
template <int S>
__device__ __forceinline__ floatx16 mfma_fp4(intx4 a, uint32_t sa, intx4 b, uint32_t sb,
                                             floatx16 c)
{
    const intx8 a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    const intx8 b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a8, b8, c, 4, 4, S, (int)sa, S,
                                                           (int)sb);
}

// The scale of a block whose largest magnitude has the fp32 bits `top`:
// 2^(floor(log2) - 2), so that it falls into [4, 8) of the grid that ends at
// 6; not under 2^-127.  NaN or infinity in the block: 255, NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    const uint32_t e = top >> 23;
    return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}

__device__ __forceinline__ float scale_value(uint32_t byte)
{
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7FC00000u : byte << 23);
}

// eight fp32 values / scale to one dword of codes, nearest, ties to even
__device__ __forceinline__ uint32_t codes_of(const float *v, float scale)
{
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    return c;
}

// the same of eight bf16 values in four dwords
__device__ __forceinline__ uint32_t codes_of_bf16(const uint32_t *w, float scale)
{
    bf16x2 p[4];
    __builtin_memcpy(p, w, sizeof p);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, p[0], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, p[1], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, p[2], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, p[3], scale, 3);
    return c;
}

// lanewise largest of the 16-bit halves
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_u16(uint32_t a, uint32_t b)
{
    u16x2 x, y;
    __builtin_memcpy(&x, &a, 4);
    __builtin_memcpy(&y, &b, 4);
    x = __builtin_elementwise_max(x, y);
    __builtin_memcpy(&a, &x, 4);
    return a;
}

}  // namespace tpk
