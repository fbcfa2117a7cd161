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
// Rows and elements past the matrix are zeros of scale 1, up to whole tiles and
// groups, so that no reader has a partial one.
#pragma once

#include "device.hpp"
#include "internal.hpp"

namespace tpk {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
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

// Eight elements k .. k + 7 of a row of K, zeros past it: fp32 in v, bf16
// pairs in w.  vec: rows are 16-byte aligned.
template <bool BF>
__device__ __forceinline__ void load8(const void *row, int64_t k, float *v, uint32_t *w, bool vec,
                                      int64_t K)
{
    if (vec && k + 8 <= K) {
        if constexpr (BF) {
            const uint4 q = *(const uint4 *)((const uint16_t *)row + k);
            w[0] = q.x;
            w[1] = q.y;
            w[2] = q.z;
            w[3] = q.w;
        } else {
            const float4 p = *(const float4 *)((const float *)row + k);
            const float4 q = *(const float4 *)((const float *)row + k + 4);
            v[0] = p.x;
            v[1] = p.y;
            v[2] = p.z;
            v[3] = p.w;
            v[4] = q.x;
            v[5] = q.y;
            v[6] = q.z;
            v[7] = q.w;
        }
    } else if constexpr (BF) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint16_t *p = (const uint16_t *)row + k + 2 * e;
            const uint32_t lo = k + 2 * e < K ? p[0] : 0, hi = k + 2 * e + 1 < K ? p[1] : 0;
            w[e] = lo | hi << 16;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k + e < K ? ((const float *)row)[k + e] : 0.0f;
    }
}

// the largest magnitude of eight values, as fp32 bits
template <bool BF>
__device__ __forceinline__ uint32_t top8(const float *v, const uint32_t *w)
{
    if constexpr (BF) {
        uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
        for (int e = 1; e < 4; ++e) m = max_u16(m, w[e] & 0x7FFF7FFFu);
        const uint32_t hi = m >> 16, lo = m & 0xFFFFu;
        return (hi > lo ? hi : lo) << 16;
    } else {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t b = __float_as_uint(v[e]) & 0x7FFFFFFFu;
            m = b > m ? b : m;
        }
        return m;
    }
}

}  // namespace tpk
