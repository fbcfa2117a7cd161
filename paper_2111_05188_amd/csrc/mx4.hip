// Matrices to 4-bit blocks and back.  Both directions move what they have to
// and compute little; they are bound by the memory.
#include <type_traits>

#include "mx4.hpp"

namespace tpk {
namespace {

// ---------------------------------------------------------------------------
// rows in memory: a wave takes 8 rows x 256 elements (4 k-steps).  Eight lanes
// read a row's 64 elements of a k-step (bf16: 128 bytes), four lanes hold a
// block and take its largest magnitude together, and each stores one dword of
// codes: 8 rows x 16 bytes are neighbours in a fragment.
// VEC: 16-byte loads (base, row pitch and K allow them up to the last block).
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t max_of_four_lanes(uint32_t m)
{
    // quad_perm [1,0,3,2], then [2,3,0,1]
    uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true);
    m = o > m ? o : m;
    o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true);
    return o > m ? o : m;
}

template <bool BF>
__global__ __launch_bounds__(256) void mx4_quantize_rows_kernel(const void *x, int64_t ld,
                                                                Mx4Layout L, uint8_t *dst,
                                                                int vec)
{
    const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t rt = blockIdx.x / (uint32_t)L.groups, g = blockIdx.x - rt * L.groups;
    const int rr = 8 * wv + (lane >> 3), q = lane & 7;      // row of the tile, eighth of the k-step
    const int64_t row = rt * 32 + rr;
    const bool in = row < L.rows;
    const char *src = (const char *)x + (in ? row : 0) * ld * (BF ? 2 : 4);
    float v[4][8];
    uint32_t w[4][4];
#pragma unroll
    for (int s = 0; s < 4; ++s) load8<BF>(src, (g * 4 + s) * 64 + q * 8, v[s], w[s], vec, in ? L.K : 0);
    uint32_t scales = 0;
    // lane of the fragment: row + 32 * half; its dword: eighth % 4
    const int fl = rr + 32 * (q >> 2);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int64_t ks = g * 4 + s;
        const uint32_t top = max_of_four_lanes(top8<BF>(v[s], w[s]));
        const bool empty = !in || ks * 64 + (q >> 2) * 32 >= L.K;   // no element at all
        const uint32_t byte = empty ? 127u : scale_byte(top);
        scales |= byte << (8 * s);
        uint32_t code;
        if constexpr (BF) code = codes_of_bf16(w[s], scale_value(byte));
        else code = codes_of(v[s], scale_value(byte));
        if (byte == 255) code = 0x22222222u;                        // ones of a NaN scale
        *(uint32_t *)(dst + ((rt * L.ksteps + ks) * 64 + fl) * 16 + (q & 3) * 4) = code;
    }
    if ((q & 3) == 0) *(uint32_t *)(dst + L.off_scales + ((rt * L.groups + g) * 64 + fl) * 4) = scales;
}

// ---------------------------------------------------------------------------
// columns in memory (element (row, k) at row + k ld): a lane takes V rows and
// walks down k, so a block needs no other lane; a wave has 64 V rows and the
// blocks of one half (the first or second 32) of a group's 4 k-steps, whose
// scales are one dword.
// ---------------------------------------------------------------------------
template <bool BF, int V>
__global__ __launch_bounds__(256) void mx4_quantize_cols_kernel(const char *x, int64_t ld,
                                                                Mx4Layout L, uint8_t *dst)
{
    constexpr int ES = BF ? 2 : 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const uint32_t strips = (uint32_t)(L.tiles * 32 + 64 * V - 1) / (64 * V);
    const uint32_t unit = blockIdx.x * 4 + wv, gh = unit / strips, g = gh / 2, h = gh % 2;
    if (g >= L.groups) return;
    const uint32_t row0 = (unit - gh * strips) * 64 * V + lane * V;
    if (row0 >= L.tiles * 32) return;
    // A lane's V elements are one aligned word, so that the last one may be read
    // with an element that is not the matrix's.
    const bool in = row0 < L.rows;
    const uint32_t off = (uint32_t)(in ? row0 : (L.rows - 1) / V * V) * ES;
    uint32_t scales[V] = {};
#pragma unroll 1
    for (int s = 0; s < 4; ++s) {
        const int64_t k0 = (int64_t)g * 256 + s * 64 + h * 32;
        float v[V][32];
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const int64_t k = k0 + j < L.K ? k0 + j : L.K - 1;
            const char *p = x + k * ld * ES;
            if constexpr (BF && V == 2) {
                const uint32_t w = load_at<uint32_t>(p, off);
                v[0][j] = __uint_as_float(w << 16);
                v[1][j] = __uint_as_float(w & 0xFFFF0000u);
            } else if constexpr (BF) {
                v[0][j] = __uint_as_float((uint32_t)load_at<uint16_t>(p, off) << 16);
            } else if constexpr (V == 2) {
                const floatx2 w = load_at<floatx2>(p, off);
                v[0][j] = w[0];
                v[1][j] = w[1];
            } else {
                v[0][j] = load_at<float>(p, off);
            }
        }
        const int steps = k0 >= L.K ? 0 : L.K - k0 < 32 ? (int)(L.K - k0) : 32;
        const uint32_t ks = g * 4 + s;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const uint32_t row = row0 + e;
            const int valid = row < L.rows ? steps : 0;
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                v[e][j] = j < valid ? v[e][j] : 0.0f;
                const uint32_t m = __float_as_uint(v[e][j]) & 0x7FFFFFFFu;
                top = m > top ? m : top;
            }
            const uint32_t byte = valid == 0 ? 127u : scale_byte(top);
            const float sc = scale_value(byte);
            uint4 code;
            code.x = codes_of(&v[e][0], sc);
            code.y = codes_of(&v[e][8], sc);
            code.z = codes_of(&v[e][16], sc);
            code.w = codes_of(&v[e][24], sc);
            if (byte == 255) code = make_uint4(0x22222222u, 0x22222222u, 0x22222222u, 0x22222222u);
            scales[e] |= byte << (8 * s);
            const uint32_t fl = (row & 31) + 32 * h;
            *(uint4 *)(dst + (((int64_t)(row >> 5) * L.ksteps + ks) * 64 + fl) * 16) = code;
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const uint32_t row = row0 + e, fl = (row & 31) + 32 * h;
        *(uint32_t *)(dst + L.off_scales + (((int64_t)(row >> 5) * L.groups + g) * 64 + fl) * 4) =
            scales[e];
    }
}

// eight codes to values, before their scale
__device__ __forceinline__ void values_of(uint32_t c, float *v)
{
    floatx2 p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
    v[0] = p[0];
    v[1] = p[1];
    p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
    v[2] = p[0];
    v[3] = p[1];
    p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2);
    v[4] = p[0];
    v[5] = p[1];
    p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
    v[6] = p[0];
    v[7] = p[1];
}

// ---------------------------------------------------------------------------
// back to rows: the places of mx4_quantize_rows_kernel
// ---------------------------------------------------------------------------
template <bool BF>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t *src, Mx4Layout L,
                                                             void *y, int64_t ld)
{
    const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t rt = blockIdx.x / (uint32_t)L.groups, g = blockIdx.x - rt * L.groups;
    const int rr = 8 * wv + (lane >> 3), q = lane & 7, fl = rr + 32 * (q >> 2);
    const int64_t row = rt * 32 + rr;
    if (row >= L.rows) return;
    const uint32_t scales = *(const uint32_t *)(src + L.off_scales + ((rt * L.groups + g) * 64 + fl) * 4);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int64_t ks = g * 4 + s, k = ks * 64 + q * 8;
        if (k >= L.K) continue;
        const uint32_t c = *(const uint32_t *)(src + ((rt * L.ksteps + ks) * 64 + fl) * 16 + (q & 3) * 4);
        const float sc = scale_value(scales >> (8 * s) & 255u);
        float v[8];
        values_of(c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= sc;
        if constexpr (BF) {
            __bf16 *out = (__bf16 *)y + row * ld + k;
            __bf16 w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = to_bf16(v[e]);   // exact: two significant bits
            if (k + 8 <= L.K) {
                __builtin_memcpy(__builtin_assume_aligned(out, 16), w, 16);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (k + e < L.K) out[e] = w[e];
            }
        } else {
            float *out = (float *)y + row * ld + k;
            if (k + 8 <= L.K) {
                *(float4 *)out = make_float4(v[0], v[1], v[2], v[3]);
                *(float4 *)(out + 4) = make_float4(v[4], v[5], v[6], v[7]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (k + e < L.K) out[e] = v[e];
            }
        }
    }
}

// A row tile's codes and scales by row of the tile and dword of eight elements
struct TileReader {
    const uint8_t *codes, *scales;

    __device__ __forceinline__ TileReader(const uint8_t *src, const Mx4Layout &L, int64_t rt)
        : codes(src + rt * L.ksteps * 1024), scales(src + L.off_scales + rt * L.groups * 256)
    {
    }
    __device__ __forceinline__ uint32_t code(uint32_t r, uint32_t d) const
    {
        return load_at<uint32_t>(codes, (d >> 3) * 1024 + (d >> 2 & 1) * 512 + r * 16 + (d & 3) * 4);
    }
    __device__ __forceinline__ float scale(uint32_t r, uint32_t d) const
    {
        return scale_value(load_at<uint8_t>(
            scales, (d >> 5) * 256 + (d >> 2 & 1) * 128 + r * 4 + (d >> 3 & 3)));
    }
};

// ---------------------------------------------------------------------------
// back to rows that follow one another without being 16-byte aligned: eight
// rows begin at a multiple of 16 bytes (if y does), so a workgroup takes eight,
// whose codes share cache lines, and writes them in whole pieces of 16 bytes.
// A piece's elements come from two neighbouring dwords of codes, which may have
// two scales, and where it passes a row's end from the next row's first.
// (65,536 x 1,001 bf16: 115 us with an element a store, 54 with pieces that end
// at the rows' ends, 45 so; 34 where pieces and rows agree.)
// ---------------------------------------------------------------------------
template <bool BF>
__global__ __launch_bounds__(256) void mx4_dequantize_flat_kernel(const uint8_t *src, Mx4Layout L,
                                                                  void *y)
{
    typedef typename std::conditional<BF, __bf16, float>::type T;
    constexpr uint32_t E = 16 / sizeof(T);
    const uint32_t K = (uint32_t)L.K, r0 = (blockIdx.x & 3) * 8;
    const int64_t row0 = (int64_t)blockIdx.x * 8, left = L.rows - row0;
    const uint32_t nrows = left < 8 ? (uint32_t)left : 8;
    const TileReader tile(src, L, blockIdx.x >> 2);
    T *out = (T *)y + row0 * K;
    for (uint32_t p = blockIdx.y * 256 + threadIdx.x; p * E < nrows * K; p += 256 * gridDim.y) {
        const uint32_t q = p * E / K, k = p * E - q * K, r = r0 + q;
        const uint32_t d0 = k / 8, d1 = (d0 + 1) * 8 < K ? d0 + 1 : d0, first = k % 8;
        const uint64_t codes = (uint64_t)tile.code(r, d1) << 32 | tile.code(r, d0);
        const float s0 = tile.scale(r, d0), s1 = tile.scale(r, d1);
        uint32_t w = (uint32_t)(codes >> (4 * first));
        const uint32_t here = K - k;                    // elements up to the row's end
        float s2 = 0.0f;
        if (here < E && q + 1 < nrows) {
            w = (w & ((1u << (4 * here)) - 1)) | tile.code(r + 1, 0) << (4 * here);
            s2 = tile.scale(r + 1, 0);
        }
        float v[8];
        values_of(w, v);
        T z[E];
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) z[e] = (T)(v[e] * (e >= here ? s2 : first + e < 8 ? s0 : s1));
        if (here >= E || q + 1 < nrows) {
            __builtin_memcpy(__builtin_assume_aligned(out + p * E, 16), z, 16);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e)
                if (e < here) out[p * E + e] = z[e];
        }
    }
}

// ---------------------------------------------------------------------------
// back to rows of any pitch and alignment: the same a row at a time, its first
// and last piece by elements; a wave takes eight rows
// ---------------------------------------------------------------------------
template <bool BF>
__global__ __launch_bounds__(256) void mx4_dequantize_odd_kernel(const uint8_t *src, Mx4Layout L,
                                                                 void *y, int64_t ld, int strips)
{
    typedef typename std::conditional<BF, __bf16, float>::type T;
    constexpr int ES = sizeof(T), E = 16 / ES;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x * 4 + wv, row8 = unit / (uint32_t)strips;
    const int piece = (int)(unit - row8 * strips) * 64 + lane, K = (int)L.K;
    const int64_t left = L.rows - (int64_t)row8 * 8;
    if (left <= 0) return;
    const TileReader tile(src, L, row8 / 4);
    const int nrows = left < 8 ? (int)left : 8;
    for (int q = 0; q < nrows; ++q) {
        const uint32_t r = (row8 & 3) * 8 + q;
        char *base = (char *)y + ((int64_t)row8 * 8 + q) * ld * ES;
        const int k0 = piece * E - (int)((uintptr_t)base % 16) / ES;    // the piece's first element
        if (k0 >= K) continue;
        const int d0 = (k0 < 0 ? 0 : k0) / 8, d1 = (d0 + 1) * 8 < K ? d0 + 1 : d0;
        const int first = k0 - d0 * 8;                                  // -7 .. 7
        const uint64_t codes = (uint64_t)tile.code(r, d1) << 32 | tile.code(r, d0);
        const float s0 = tile.scale(r, d0), s1 = tile.scale(r, d1);
        float v[8];
        values_of(first < 0 ? (uint32_t)(codes << (-4 * first)) : (uint32_t)(codes >> (4 * first)), v);
        T z[E];
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = (T)(v[e] * (first + e < 8 ? s0 : s1));
        T *to = (T *)(base + (int64_t)k0 * ES);
        if (k0 >= 0 && k0 + E <= K) {
            __builtin_memcpy(__builtin_assume_aligned(to, 16), z, 16);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (k0 + e >= 0 && k0 + e < K) to[e] = z[e];
        }
    }
}

bool vec16(const void *p, int64_t ld, int es) { return ((uintptr_t)p | (uint64_t)(ld * es)) % 16 == 0; }

}  // namespace

Mx4Layout mx4_layout(int64_t rows, int64_t K)
{
    Mx4Layout L;
    L.rows = rows;
    L.K = K;
    L.tiles = (rows + 31) / 32;
    L.groups = (K + 255) / 256;
    L.ksteps = 4 * L.groups;
    L.off_scales = L.tiles * L.ksteps * 1024;
    L.total = (size_t)(L.off_scales + L.tiles * L.groups * 256);
    return L;
}

hipError_t launch_mx4_quantize(const void *x, bool bf16, int64_t row_stride, int64_t col_stride,
                               const Mx4Layout &L, void *dst, hipStream_t s)
{
    if (col_stride == 1) {
        const dim3 grid((unsigned)(L.tiles * L.groups));
        const int vec = vec16(x, row_stride, bf16 ? 2 : 4);
        if (bf16)
            hipLaunchKernelGGL(mx4_quantize_rows_kernel<true>, grid, dim3(256), 0, s, x, row_stride,
                               L, (uint8_t *)dst, vec);
        else
            hipLaunchKernelGGL(mx4_quantize_rows_kernel<false>, grid, dim3(256), 0, s, x,
                               row_stride, L, (uint8_t *)dst, vec);
        return hipGetLastError();
    }
    // two rows a lane where every pair is aligned and eight waves a CU are left
    // (1,536 x 11,011 fp32, 1,032 or 2,064 waves: 20 or 16 us)
    const int es = bf16 ? 2 : 4;
    const bool two = (L.rows + 127) / 128 * L.groups * 2 >= 2048 &&
                     ((uintptr_t)x | (uint64_t)(col_stride * es)) % (2 * es) == 0;
    const int64_t strips = (L.tiles * 32 + (two ? 127 : 63)) / (two ? 128 : 64);
    const dim3 grid((unsigned)((strips * L.groups * 2 + 3) / 4));
    void (*kernel)(const char *, int64_t, Mx4Layout, uint8_t *) =
        bf16 ? (two ? mx4_quantize_cols_kernel<true, 2> : mx4_quantize_cols_kernel<true, 1>)
             : (two ? mx4_quantize_cols_kernel<false, 2> : mx4_quantize_cols_kernel<false, 1>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const char *)x, col_stride, L,
                       (uint8_t *)dst);
    return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const void *src, const Mx4Layout &L, void *y, bool bf16,
                                 int64_t ld, hipStream_t s)
{
    // (eight rows of under 2^32 elements, a piece in two rows at most, under
    // 2^32 threads)
    if (!vec16(y, ld, bf16 ? 2 : 4) && ld == L.K && L.K >= 8 && (uintptr_t)y % 16 == 0 &&
        L.rows <= 1 << 26) {
        const int64_t pieces = 8 * L.K / (bf16 ? 8 : 4), most = (pieces + 511) / 512;
        const int64_t parts = most < 65535 ? most : 65535;      // two pieces a thread
        hipLaunchKernelGGL((bf16 ? mx4_dequantize_flat_kernel<true> : mx4_dequantize_flat_kernel<false>),
                           dim3((unsigned)((L.rows + 7) / 8), (unsigned)parts), dim3(256), 0, s,
                           (const uint8_t *)src, L, y);
        return hipGetLastError();
    }
    if (!vec16(y, ld, bf16 ? 2 : 4)) {
        // a row's pieces: one more where it begins inside the first
        const int each = bf16 ? 8 : 4;
        const int64_t strips = (L.K + 2 * each - 2) / each / 64 + 1, units = (L.rows + 7) / 8 * strips;
        hipLaunchKernelGGL((bf16 ? mx4_dequantize_odd_kernel<true> : mx4_dequantize_odd_kernel<false>),
                           dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, (const uint8_t *)src, L,
                           y, ld, (int)strips);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((bf16 ? mx4_dequantize_kernel<true> : mx4_dequantize_kernel<false>),
                       dim3((unsigned)(L.tiles * L.groups)), dim3(256), 0, s, (const uint8_t *)src, L,
                       y, ld);
    return hipGetLastError();
}

}  // namespace tpk
