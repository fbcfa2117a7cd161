// Products of 4-bit matrices: y[m][n] = act(sum_k A[m][k] W[n][k] + bias[n]).
//
// The matrix instruction gets W's fragment as its first operand and A's as its
// second, so a lane of the result holds one row m and runs of four
// neighbouring n: stores of 16 (bf16: 8) bytes.  Sums are fp32 and round once.
#include "mx4.hpp"

namespace tpk {
namespace {

// act(z + bias) of four neighbouring columns n .. n + 3 of row m
template <bool BF>
__device__ __forceinline__ void finish4(const Mx4Args &a, int64_t m, int64_t n, float *z,
                                        bool vec)
{
    const int64_t N = a.lw.rows;
    if (n >= N) return;
    if (a.bias) {
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] += n + e < N ? a.bias[n + e] : 0.0f;
    }
    if (a.act == TP_ACT_TANH) {
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = BF ? tanh_for_bf16(z[e]) : tanh_f32(z[e]);
    }
    if constexpr (BF) {
        __bf16 *out = (__bf16 *)a.y + m * a.ldy + n;
        __bf16 w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = to_bf16(z[e]);
        if (vec && n + 4 <= N) {
            __builtin_memcpy(__builtin_assume_aligned(out, 8), w, 8);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < N) out[e] = w[e];
        }
    } else {
        float *out = (float *)a.y + m * a.ldy + n;
        if (vec && n + 4 <= N) {
            *(float4 *)out = make_float4(z[0], z[1], z[2], z[3]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < N) out[e] = z[e];
        }
    }
}

// ---------------------------------------------------------------------------
// Any size.  A workgroup of 2 x 2 waves has 8 x 8 tiles of 32 x 32, a wave 4 x 4
// of them (256 registers of sums: each fragment read from LDS feeds four matrix
// instructions).  Groups of four k-steps go through two LDS buffers: while one
// is multiplied, the next lies in registers and is stored to the other.
// More workgroups than blocks: a part of K each; its sums go to the workspace as the lanes
// hold them, 1 KiB a store, and mx4_join_kernel adds the parts in order.
// 1,536 x 1,001 over K = 65,536: 67 us, 18 of them for launch and sums, then
// 4.1 of the 8.4 PFLOP/s that the instruction reaches; with the copies in a row
// before the matrix instructions 76 us, with fragments straight from L1 and 4 x
// 2 tiles a wave 125 us.
// ---------------------------------------------------------------------------
constexpr int WT = 4, BT = 2 * WT;                  // tiles of a wave, of a workgroup, a side
constexpr int64_t BLOCK_FLOATS = (int64_t)BT * BT * 1024;

__global__ __launch_bounds__(256, 1) void mx4_product_kernel(Mx4Args a, int nblocks, int blocks,
                                                             int groups_per)
{
    constexpr int STAGE = 2 * BT * 4096;            // A's tiles, then W's: four k-steps of each
    __shared__ __attribute__((aligned(16))) char stages[2 * STAGE];
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    // Workgroups go to the eight XCDs in turn; here an XCD's share is neighbours,
    // who read the same part of K of the same tiles, so that its L2 has them.
    const uint32_t total = gridDim.x, xcd = blockIdx.x % 8, each = total / 8, more = total % 8;
    const int at = (int)(xcd * each + (xcd < more ? xcd : more) + blockIdx.x / 8);
    const int part = at / blocks, block = at - part * blocks;
    const int mb = block / nblocks, nb = block - mb * nblocks;
    const int wm = wv >> 1, wn = wv & 1;
    const int64_t ksteps = a.la.ksteps, groups = a.la.groups;
    const int g0 = part * groups_per;
    const int g1 = g0 + groups_per < groups ? g0 + groups_per : (int)groups;
    // tiles past the matrix repeat its last one
    auto a_tile = [&](int i) {
        const int64_t t = (int64_t)mb * BT + i;
        return t < a.la.tiles ? t : a.la.tiles - 1;
    };
    auto w_tile = [&](int j) {
        const int64_t t = (int64_t)nb * BT + j;
        return t < a.lw.tiles ? t : a.lw.tiles - 1;
    };
    // waves 0 and 1 bring A's tiles, 2 and 3 W's, four each
    const uint8_t *from[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
        from[t] = wv < 2 ? a.a + a_tile(wv * 4 + t) * ksteps * 1024
                         : a.w + w_tile(wv * 4 + t - BT) * ksteps * 1024;
    const uint8_t *pa[WT], *pw[WT];
#pragma unroll
    for (int i = 0; i < WT; ++i) {
        pa[i] = a.a + a.la.off_scales + a_tile(wm * WT + i) * groups * 256;
        pw[i] = a.w + a.lw.off_scales + w_tile(wn * WT + i) * groups * 256;
    }
    intx4 share[16];
    uint32_t na[WT], nw[WT];
    auto fetch = [&](int g, int k) {
        share[k] = load_at<intx4>(from[k / 4] + ((int64_t)g * 4 + k % 4) * 1024, lane * 16u);
    };
    auto fetch_scale = [&](int g, int k) {
        if (k < WT) na[k] = load_at<uint32_t>(pa[k] + (int64_t)g * 256, lane * 4u);
        else nw[k - WT] = load_at<uint32_t>(pw[k - WT] + (int64_t)g * 256, lane * 4u);
    };
    auto put = [&](char *to, int k) {
        *(intx4 *)(to + (wv * 16 + k) * 1024 + lane * 16) = share[k];
    };
    floatx16 c[WT][WT] = {};
#pragma unroll
    for (int k = 0; k < 16; ++k) fetch(g0, k);
#pragma unroll
    for (int k = 0; k < 2 * WT; ++k) fetch_scale(g0, k);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        put(stages, k);
        fetch(g0 + 1 < g1 ? g0 + 1 : g0, k);
    }
    for (int g = g0; g < g1; ++g) {
        const char *now = stages + ((g - g0) & 1) * STAGE;
        char *other = stages + ((g - g0 + 1) & 1) * STAGE;
        // (past the last group: the last one again)
        const int next = g + 1 < g1 ? g + 1 : g1 - 1, later = g + 2 < g1 ? g + 2 : g1 - 1;
        // this stage is whole, and nobody reads the one before any more
        workgroup_lds_barrier();
        uint32_t sa[WT], sw[WT];
#pragma unroll
        for (int i = 0; i < WT; ++i) {
            sa[i] = na[i];
            sw[i] = nw[i];
        }
        intx4 fa[2][WT], fw[2][WT];
        auto read = [&](int s, int k) {
            if (k < WT)
                fa[s & 1][k] = *(const intx4 *)(now + ((wm * WT + k) * 4 + s) * 1024 + lane * 16);
            else
                fw[s & 1][k - WT] = *(const intx4 *)(now + ((BT + wn * WT + k - WT) * 4 + s) * 1024 + lane * 16);
        };
#pragma unroll
        for (int k = 0; k < 2 * WT; ++k) read(0, k);
        // Between the matrix instructions, in this order: the next stage from
        // registers to LDS and the one after into the registers just stored;
        // the next k-step's fragments; the next group's scales.
#pragma unroll
        for (int q = 0; q < 4 * WT * WT; ++q) {
            const int s = q / (WT * WT), i = q / WT % WT, j = q % WT, k = q % (WT * WT);
            __builtin_amdgcn_sched_barrier(0);
            if (s == 0) c[i][j] = mfma_fp4<0>(fw[0][j], sw[j], fa[0][i], sa[i], c[i][j]);
            else if (s == 1) c[i][j] = mfma_fp4<1>(fw[1][j], sw[j], fa[1][i], sa[i], c[i][j]);
            else if (s == 2) c[i][j] = mfma_fp4<2>(fw[0][j], sw[j], fa[0][i], sa[i], c[i][j]);
            else c[i][j] = mfma_fp4<3>(fw[1][j], sw[j], fa[1][i], sa[i], c[i][j]);
            if (s < 3 && k % 2 == 0) read(s + 1, k / 2);
            if (s == 0) {
                put(other, k);
                fetch(later, k);
            }
            if (s == 1 && k % 2 == 1) fetch_scale(next, k / 2);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    if ((int)total == blocks) {
        // a row of tiles at a time through the wave's part of the LDS, then in
        // rows of 128 columns (a loop: unrolled, the epilogue of 256 registers
        // is longer than the compiler keeps registers for)
        constexpr int PITCH = (WT * 32 + 4) * 4;
        char *rows = stages + wv * 32 * PITCH;
        const bool vec = ((uintptr_t)a.y | (uint64_t)(a.ldy * (a.y_bf16 ? 2 : 4))) %
                             (a.y_bf16 ? 8 : 16) == 0;
        workgroup_lds_barrier();
#pragma unroll
        for (int i = 0; i < WT; ++i) {
#pragma unroll
            for (int j = 0; j < WT; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    *(floatx4 *)(rows + (lane & 31) * PITCH + (j * 32 + 8 * r + 4 * (lane >> 5)) * 4) =
                        floatx4{c[i][j][4 * r], c[i][j][4 * r + 1], c[i][j][4 * r + 2],
                                c[i][j][4 * r + 3]};
            wave_lds_fence();
            const int64_t m0 = ((int64_t)mb * BT + wm * WT + i) * 32 + (lane >> 5);
            const int64_t n = ((int64_t)nb * BT + wn * WT) * 32 + (lane & 31) * 4;
#pragma unroll 1
            for (int k = 0; k < 32; k += 2) {
                const floatx4 v = *(const floatx4 *)(rows + (k + (lane >> 5)) * PITCH + (lane & 31) * 16);
                float z[4] = {v[0], v[1], v[2], v[3]};
                if (m0 + k >= a.la.rows) continue;
                if (a.y_bf16) finish4<true>(a, m0 + k, n, z, vec);
                else finish4<false>(a, m0 + k, n, z, vec);
            }
            wave_lds_fence();
        }
        return;
    }
    float *sums = (float *)a.work + (int64_t)at * BLOCK_FLOATS;
#pragma unroll
    for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < WT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                store_at(sums + (((wv * WT + i) * WT + j) * 4 + r) * 256, lane * 16u,
                         floatx4{c[i][j][4 * r], c[i][j][4 * r + 1], c[i][j][4 * r + 2],
                                 c[i][j][4 * r + 3]});
}

// the parts of K in order: a thread has four neighbours of a row
__global__ __launch_bounds__(256) void mx4_join_kernel(Mx4Args a, int nblocks, int blocks, int parts)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;     // of a part's fours
    const int block = (int)(at / (BLOCK_FLOATS / 4)), in = (int)(at % (BLOCK_FLOATS / 4));
    const int lane = in & 63, r = in >> 6 & 3, j = in >> 8 & 3, i = in >> 10 & 3, wv = in >> 12;
    const int mb = block / nblocks, nb = block - mb * nblocks;
    const int64_t m = ((int64_t)mb * BT + (wv >> 1) * WT + i) * 32 + (lane & 31);
    const int64_t n = ((int64_t)nb * BT + (wv & 1) * WT + j) * 32 + 8 * r + 4 * (lane >> 5);
    if (m >= a.la.rows || n >= a.lw.rows) return;
    const floatx4 *part = (const floatx4 *)a.work + at;
    const int64_t stride = (int64_t)blocks * (BLOCK_FLOATS / 4);
    floatx4 sum = {};
#pragma unroll 8
    for (int p = 0; p < parts; ++p) sum += part[p * stride];
    float z[4] = {sum[0], sum[1], sum[2], sum[3]};
    if (a.y_bf16) finish4<true>(a, m, n, z, false);
    else finish4<false>(a, m, n, z, false);
}

// ---------------------------------------------------------------------------
// K up to 1,024: a wave keeps its RT x 32 rows of A in registers for all of K
// (a lane's part of a fragment is one block of 32, so rows of x go to 4 bits
// there with no other lane's help), and W goes past it one tile of 32 columns
// at a time, from LDS, where the workgroup's waves share it.  x is read once,
// y written once.  From L1 instead of LDS a tile took 1.7 us against 1.3.
// 65,536 x 1,001 bf16 rows times 1,536: 90 us (2.2 PFLOP/s), 23 of them for x
// at 6 TB/s; then y's 201 MB, LDS reads (13,100 a CU) and 25 us of matrix
// instructions share the rest.
// SRC: x in fp32 (0), bf16 (1), or A in 4 bits (2).  KG groups of 4 k-steps.
// ---------------------------------------------------------------------------
enum { SRC_F32 = 0, SRC_BF16 = 1, SRC_FOUR = 2 };

template <int S, int RT, int KS>
__device__ __forceinline__ void mfma_row(floatx16 (&c)[RT], const intx4 &w, uint32_t scale,
                                         const intx4 (&fa)[RT][KS], int ks,
                                         const uint32_t (&sa)[RT][KS / 4], int g)
{
#pragma unroll
    for (int i = 0; i < RT; ++i) c[i] = mfma_fp4<S>(w, scale, fa[i][ks], sa[i][g], c[i]);
}

// Rows of y from row m0 on as a buffer that ends with the matrix: stores past
// it are dropped.  A wave reaches RT x 32 rows, under 2^31 bytes.
template <bool BF>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t out_buffer(const Mx4Args &a, int64_t m0)
{
    constexpr int ES = BF ? 2 : 4;
    const int64_t bytes = m0 < a.la.rows ? ((a.la.rows - 1 - m0) * a.ldy + a.lw.rows) * ES : 0;
    return __builtin_amdgcn_make_buffer_rsrc((char *)a.y + m0 * a.ldy * ES, 0,
                                             (int)(bytes < 0x7FFFFFFC ? bytes : 0x7FFFFFFC),
                                             0x00027000);
}

// A wave's rows of y go out 256 bytes at a time: results of 64 (bf16: 128)
// columns gather in the wave's part of the LDS, then each store writes four
// whole pieces.  (Stores straight from the result's registers are 8 bytes of
// 32 rows each, or 64 bytes of two rows: 65,536 x 1,536 in bf16 took 158 and
// 124 us against 110.)
// They pass the L2 (the buffer's nt bit), which W's tiles then keep: 65,536
// rows 113 -> 100 us, 4,096 rows 21 -> 19.
constexpr int PIECE = 256, PIECE_PITCH = PIECE + 16, NT = 2;

// results of tile `slot` of the piece: lane l has row l%32 of tile i, columns
// 8 r + 4(l/32) .. +3 in registers 4 r .. 4 r + 3
template <bool BF, int RT>
__device__ __forceinline__ void gather_tile(char *lds, int slot, int lane, int act,
                                            const floatx4 (&bias)[4], floatx16 (&c)[RT])
{
    constexpr int ES = BF ? 2 : 4;
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) c[i][e] += bias[e / 4][e % 4];
    if (act == TP_ACT_TANH) {
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                c[i][e] = BF ? tanh_for_bf16(c[i][e]) : tanh_f32(c[i][e]);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float z[4] = {c[i][4 * r], c[i][4 * r + 1], c[i][4 * r + 2], c[i][4 * r + 3]};
            char *at = lds + (32 * i + (lane & 31)) * PIECE_PITCH +
                       (slot * 32 + 8 * r + 4 * (lane >> 5)) * ES;
            if constexpr (BF) {
                const bf16x4 w = {to_bf16(z[0]), to_bf16(z[1]), to_bf16(z[2]), to_bf16(z[3])};
                *(bf16x4 *)at = w;
            } else {
                *(floatx4 *)at = floatx4{z[0], z[1], z[2], z[3]};
            }
        }
}

// The piece's rows to y from column n0 on, columns under n1.  EVEN: n1 is a
// multiple of 16 bytes and y 4-byte aligned, so that a lane's 16 bytes are all
// in or all out, and no branch stands around the stores: the compiler can count
// them, and what waits for a later load need not wait for them.
template <bool BF, int RT, bool EVEN>
__device__ __forceinline__ void flush_piece(const char *lds, __amdgpu_buffer_rsrc_t out,
                                            uint32_t pitch, int64_t n0, int64_t n1, int lane)
{
    constexpr int ES = BF ? 2 : 4, E = 16 / ES;     // elements of a lane
    const int64_t n = n0 + (lane & 15) * E;
    const char *from = lds + (lane >> 4) * PIECE_PITCH + (lane & 15) * 16;
    const uint32_t to = (uint32_t)(lane >> 4) * pitch + (uint32_t)n * ES;
    if constexpr (EVEN) {
        // (an offset of 2^31 and more is outside every buffer)
        const uint32_t at = n < n1 ? to : 0x80000000u;
#pragma unroll
        for (int k = 0; k < 8 * RT; ++k) {
            const uintx4 v = *(const uintx4 *)(from + 4 * k * PIECE_PITCH);
            __builtin_amdgcn_raw_buffer_store_b128(v, out, (int)(at + 4 * k * pitch), 0, NT);
        }
    } else if (n < n1) {
#pragma unroll 1
        for (int k = 0; k < 8 * RT; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (n + e < n1) {
                    const int at = (int)(to + 4 * k * pitch + e * ES);
                    const char *v = from + 4 * k * PIECE_PITCH + e * ES;
                    if constexpr (BF)
                        __builtin_amdgcn_raw_buffer_store_b16(*(const uint16_t *)v, out, at, 0, 0);
                    else
                        __builtin_amdgcn_raw_buffer_store_b32(*(const uint32_t *)v, out, at, 0, 0);
                }
    }
}

// A block of 32 elements as loaded: bf16 in pairs, fp32
template <bool BF>
struct RawBlock {
    uint32_t w[BF ? 16 : 32];
};

// Rows of x from row m0 on as a buffer that ends with the matrix: the hardware
// returns zeros past it, so a row's last block needs no branch.
template <bool BF>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const Mx4Args &a, int64_t m0)
{
    constexpr int ES = BF ? 2 : 4;
    const int64_t bytes = m0 < a.la.rows ? ((a.la.rows - 1 - m0) * a.ldx + a.la.K) * ES : 0;
    // whole dwords: the last one holds the last element
    const int64_t most = bytes < 0xFFFFFFFC ? (bytes + 3) & ~(int64_t)3 : 0xFFFFFFFC;
    return __builtin_amdgcn_make_buffer_rsrc((void *)((const char *)a.x + m0 * a.ldx * ES), 0,
                                             (int)(uint32_t)most, 0x00027000);
}

// block at byte `off` of the buffer (16-byte aligned)
template <bool BF>
__device__ __forceinline__ void load_block(__amdgpu_buffer_rsrc_t rows, uint32_t off,
                                           RawBlock<BF> &raw)
{
#pragma unroll
    for (int q = 0; q < (BF ? 4 : 8); ++q) {
        const uintx4 v = __builtin_amdgcn_raw_buffer_load_b128(rows, (int)(off + 16 * q), 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) raw.w[4 * q + e] = v[e];
    }
}

// zeros from element n of the block on
template <bool BF>
__device__ __forceinline__ void end_block(RawBlock<BF> &raw, int n)
{
#pragma unroll
    for (int e = 0; e < (BF ? 16 : 32); ++e) {
        if constexpr (BF) raw.w[e] = 2 * e >= n ? 0 : 2 * e + 1 >= n ? raw.w[e] & 0xFFFFu : raw.w[e];
        else raw.w[e] = e >= n ? 0 : raw.w[e];
    }
}

template <bool BF>
__device__ __forceinline__ uint32_t block_to_fp4(const RawBlock<BF> &raw, bool any, intx4 &code)
{
    float v[4][8];
    uint32_t w[4][4], top = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (BF) __builtin_memcpy(w[q], &raw.w[4 * q], 16);
        else __builtin_memcpy(v[q], &raw.w[8 * q], 32);
        const uint32_t t = top8<BF>(v[q], w[q]);
        top = t > top ? t : top;
    }
    const uint32_t byte = any ? scale_byte(top) : 127u;
    const float sc = scale_value(byte);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t c;
        if constexpr (BF) c = codes_of_bf16(w[q], sc);
        else c = codes_of(v[q], sc);
        code[q] = (int)(byte == 255 ? 0x22222222u : c);
    }
    return byte;
}

template <int SRC, int KG, int RT, int NW, bool YBF, bool EVEN>
__global__ __launch_bounds__(64 * NW, 2) void mx4_panel_kernel(Mx4Args a, int tiles_per)
{
    constexpr int KS = 4 * KG, SCALES = KS * 1024, BIAS = SCALES + KG * 256;  // a tile of W
    constexpr int LOADS = KS / NW;                              // of 16 bytes a thread
    __shared__ __attribute__((aligned(16))) char tiles[2][BIAS + 128];
    __shared__ __attribute__((aligned(16))) char pieces[NW][RT * 32 * PIECE_PITCH];
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t mt0 = ((int64_t)blockIdx.x * NW + wv) * RT;   // (past A: reads zeros, stores nothing)
    const int ntiles = (int)a.lw.tiles, nt0 = blockIdx.y * tiles_per;
    const int nt1 = nt0 + tiles_per < ntiles ? nt0 + tiles_per : ntiles;
    const uint8_t *pw = a.w + a.lw.off_scales;
    // the workgroup's share of a tile on its way: registers, then LDS.  The
    // tiles of a whole piece are under way, since a tile takes less time than
    // W's latency; past the last tile they repeat it.
    constexpr int SLOTS = PIECE / (32 * (YBF ? 2 : 4));     // tiles of a piece
    struct Share {
        intx4 code[LOADS];
        uint32_t scale, bias;
    };
    // no bias: a buffer of nothing, which reads as zeros
    const __amdgpu_buffer_rsrc_t biases = __builtin_amdgcn_make_buffer_rsrc(
        (void *)a.bias, 0, a.bias ? (int)(a.lw.rows * 4) : 0, 0x00027000);
    const int wg = wv < KG ? wv : KG - 1;
    auto fetch_tile = [&](int t, Share &to) {
        const int64_t nt = t < nt1 ? t : nt1 - 1;
#pragma unroll
        for (int k = 0; k < LOADS; ++k)
            to.code[k] = load_at<intx4>(a.w + (nt * KS + k * NW + wv) * 1024, lane * 16u);
        to.scale = load_at<uint32_t>(pw + (nt * KG + wg) * 256, lane * 4u);
        to.bias = __builtin_amdgcn_raw_buffer_load_b32(biases, (int)nt * 128 + (lane & 31) * 4, 0, 0);
    };
    auto store_tile = [&](char *to, const Share &from) {
#pragma unroll
        for (int k = 0; k < LOADS; ++k)
            *(intx4 *)(to + (k * NW + wv) * 1024 + lane * 16) = from.code[k];
        *(uint32_t *)(to + SCALES + wg * 256 + lane * 4) = from.scale;
        *(uint32_t *)(to + BIAS + (lane & 31) * 4) = from.bias;     // (the same from every wave)
    };
    // Whole pieces in an order that starts elsewhere for each workgroup, a
    // partial one last: in step, all workgroups would write the same columns at
    // a time, and with a pitch of many 256 bytes that is a few of the memory's
    // channels.
    const int whole = (nt1 - nt0) / SLOTS, turn = whole ? (int)(blockIdx.x % (uint32_t)whole) : 0;
    auto piece_at = [&](int k) {
        const int q = k + turn < whole ? k + turn : k + turn - whole;
        return nt0 + (k < whole ? q : k) * SLOTS;
    };
    Share first, share[SLOTS];
    fetch_tile(piece_at(0), first);

    intx4 fa[RT][KS];
    uint32_t sa[RT][KG];
    if constexpr (SRC == SRC_FOUR) {
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int64_t t = mt0 + i < a.la.tiles ? mt0 + i : a.la.tiles - 1;
#pragma unroll
            for (int s = 0; s < KS; ++s) fa[i][s] = load_at<intx4>(a.a + (t * KS + s) * 1024, lane * 16u);
#pragma unroll
            for (int g = 0; g < KG; ++g)
                sa[i][g] = load_at<uint32_t>(a.a + a.la.off_scales + (t * KG + g) * 256, lane * 4u);
        }
    } else {
        // U k-steps' loads are in flight while the U before go to 4 bits
        constexpr bool BF = SRC == SRC_BF16;
        constexpr int U = BF ? 4 : 2, ES = BF ? 2 : 4;
        const int K = (int)a.la.K, half = (lane >> 5) * 32;
        const __amdgpu_buffer_rsrc_t rows = rows_buffer<BF>(a, mt0 * 32);
        const uint32_t pitch = (uint32_t)a.ldx * ES, off = (lane & 31) * pitch + half * ES;
        RawBlock<BF> raw[2][U];
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int g = 0; g < KG; ++g) sa[i][g] = 0;
        auto fetch = [&](int u, RawBlock<BF> (&to)[U]) {
#pragma unroll
            for (int s = 0; s < U; ++s) {
                const int ks = u * U + s;
                load_block<BF>(rows, off + ks / KS * 32 * pitch + ks % KS * 64 * ES, to[s]);
            }
        };
        fetch(0, raw[0]);
#pragma unroll
        for (int u = 0; u < RT * KS / U; ++u) {
            if (u + 1 < RT * KS / U) fetch(u + 1, raw[(u + 1) & 1]);
#pragma unroll
            for (int s = 0; s < U; ++s) {
                const int ks = (u * U + s) % KS, i = (u * U + s) / KS, left = K - ks * 64 - half;
                // (only the last group of k-steps can end inside)
                if (ks >= KS - 4 && K < ks * 64 + 64) end_block<BF>(raw[u & 1][s], left);
                sa[i][ks / 4] |= block_to_fp4<BF>(raw[u & 1][s], left > 0, fa[i][ks])
                                 << (8 * (ks % 4));
                // keeps the conversion here: the compiler otherwise moves it to
                // the codes' use, and what all units loaded has to wait for it
                asm volatile("" : "+v"(fa[i][ks]));
            }
        }
    }
    store_tile(tiles[0], first);
#pragma unroll
    for (int u = 0; u < SLOTS; ++u)
        fetch_tile(u + 1 < SLOTS ? piece_at(0) + u + 1 : piece_at(1), share[u]);
    const __amdgpu_buffer_rsrc_t out = out_buffer<YBF>(a, mt0 * 32);
    const uint32_t pitch = (uint32_t)a.ldy * (YBF ? 2 : 4);
    char *lds = pieces[wv];
    auto tile_step = [&](int u, int later) {
        char *tile = tiles[u & 1], *other = tiles[(u + 1) & 1];
        // this tile is whole, and nobody reads the one before any more
        workgroup_lds_barrier();
        store_tile(other, share[u]);
        fetch_tile(later, share[u]);
        floatx16 c[RT] = {}, c2[RT] = {};       // even and odd k-steps: twice the chains
        // a group's fragments are read while the group before is multiplied
        intx4 fw[2][4];
        uint32_t sw[2];
        auto read_group = [&](int g) {
#pragma unroll
            for (int s = 0; s < 4; ++s)
                fw[g & 1][s] = *(const intx4 *)(tile + (4 * g + s) * 1024 + lane * 16);
            sw[g & 1] = *(const uint32_t *)(tile + SCALES + g * 256 + lane * 4);
        };
        read_group(0);
#pragma unroll
        for (int g = 0; g < KG; ++g) {
            if (g + 1 < KG) read_group(g + 1);
            __builtin_amdgcn_sched_barrier(0);
            mfma_row<0, RT, KS>(c, fw[g & 1][0], sw[g & 1], fa, 4 * g, sa, g);
            mfma_row<1, RT, KS>(c2, fw[g & 1][1], sw[g & 1], fa, 4 * g + 1, sa, g);
            mfma_row<2, RT, KS>(c, fw[g & 1][2], sw[g & 1], fa, 4 * g + 2, sa, g);
            mfma_row<3, RT, KS>(c2, fw[g & 1][3], sw[g & 1], fa, 4 * g + 3, sa, g);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) c[i] += c2[i];
        floatx4 bias[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
            bias[r] = *(const floatx4 *)(tile + BIAS + (8 * r + 4 * (lane >> 5)) * 4);
        gather_tile<YBF, RT>(lds, u, lane, a.act, bias, c);
    };
    const int64_t N = a.lw.rows;
    auto flush = [&](int t) {
        const int64_t n0 = (int64_t)t * 32, n1 = (int64_t)(t + SLOTS < nt1 ? t + SLOTS : nt1) * 32;
        wave_lds_fence();
        flush_piece<YBF, RT, EVEN>(lds, out, pitch, n0, n1 < N ? n1 : N, lane);
        wave_lds_fence();
    };
    for (int k = 0; k < whole; ++k) {
        // the tile under way after a step is the one SLOTS + 1 further on
        const int next = piece_at(k + 1), after = piece_at(k + 2);
#pragma unroll
        for (int u = 0; u < SLOTS; ++u) tile_step(u, u + 1 < SLOTS ? next + u + 1 : after);
        flush(piece_at(k));
    }
    const int rest = nt1 - nt0 - whole * SLOTS;
    if (rest == 0) return;
#pragma unroll
    for (int u = 0; u < SLOTS - 1; ++u)
        if (u < rest) tile_step(u, nt1);
    flush(nt0 + whole * SLOTS);
}

struct Plan {
    int mblocks, nblocks, parts, groups_per;
};

// Parts of K so that the workgroups fill the GPU once; a part has at least
// four groups of k-steps, and there are at most 64 (each is 256 KiB a workgroup
// to store and to add).
Plan plan_of(int64_t M, int64_t N, int64_t K)
{
    Plan p;
    const int64_t groups = (K + 255) / 256;
    p.mblocks = (int)((M + 32 * BT - 1) / (32 * BT));
    p.nblocks = (int)((N + 32 * BT - 1) / (32 * BT));
    const int64_t blocks = (int64_t)p.mblocks * p.nblocks;
    int64_t parts = blocks < 256 ? 256 / blocks : 1;
    if (parts > 64) parts = 64;
    if (parts > groups / 4) parts = groups / 4;
    if (parts < 1) parts = 1;
    p.groups_per = (int)((groups + parts - 1) / parts);
    p.parts = (int)((groups + p.groups_per - 1) / p.groups_per);
    return p;
}

size_t parts_bytes(const Plan &p)
{
    return p.parts > 1 ? (size_t)p.parts * p.mblocks * p.nblocks * BLOCK_FLOATS * sizeof(float) : 0;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

// x in 4 bits, then the parts of K
size_t mx4_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    const Plan p = plan_of(M, N, K);
    return round256(mx4_layout(M, K).total) + parts_bytes(p) + 256;
}

template <int SRC, int KG, int RT, int NW>
void start_panel(const Mx4Args &a, hipStream_t s)
{
    const int64_t blocks = (a.la.tiles + NW * RT - 1) / (NW * RT), nt = a.lw.tiles;
    int64_t parts = blocks < 256 ? (256 + blocks - 1) / blocks : 1;
    if (parts > nt) parts = nt;
    const int per = (int)((nt + parts - 1) / parts);
    const dim3 grid((unsigned)blocks, (unsigned)((nt + per - 1) / per));
    // 16 bytes of a row of y are all inside it, at addresses of whole dwords
    const int es = a.y_bf16 ? 2 : 4;
    const bool even = a.lw.rows * es % 16 == 0 && ((uintptr_t)a.y | (uint64_t)(a.ldy * es)) % 4 == 0;
    void (*kernel)(Mx4Args, int) =
        a.y_bf16 ? (even ? mx4_panel_kernel<SRC, KG, RT, NW, true, true>
                         : mx4_panel_kernel<SRC, KG, RT, NW, true, false>)
                 : (even ? mx4_panel_kernel<SRC, KG, RT, NW, false, true>
                         : mx4_panel_kernel<SRC, KG, RT, NW, false, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(64 * NW), 0, s, a, per);
}

constexpr int PANEL_RT = 1, PANEL_NW = 4;

template <int SRC>
hipError_t launch_panel(const Mx4Args &a, hipStream_t s)
{
    switch (a.la.groups) {
    case 1: start_panel<SRC, 1, PANEL_RT, PANEL_NW>(a, s); break;
    case 2: start_panel<SRC, 2, PANEL_RT, PANEL_NW>(a, s); break;
    case 3: start_panel<SRC, 3, PANEL_RT, PANEL_NW>(a, s); break;
    default: start_panel<SRC, 4, PANEL_RT, PANEL_NW>(a, s);
    }
    return hipGetLastError();
}

hipError_t launch_mx4_product(const Mx4Args &in, hipStream_t s)
{
    Mx4Args a = in;
    const int es = a.x_bf16 ? 2 : 4;
    // a wave's rows within 2^30 bytes: offsets from 2^31 on are outside its buffers
    constexpr int64_t PITCH_END = ((int64_t)1 << 30) / (32 * PANEL_RT);
    const bool panel = a.la.groups <= 4 && a.ldy * (a.y_bf16 ? 2 : 4) < PITCH_END;
    // rows of x in 16-byte pieces
    if (panel && !a.a && ((uintptr_t)a.x | (uint64_t)(a.ldx * es)) % 16 == 0 &&
        a.ldx * es < PITCH_END)
        return a.x_bf16 ? launch_panel<SRC_BF16>(a, s) : launch_panel<SRC_F32>(a, s);
    const Plan p = plan_of(a.la.rows, a.lw.rows, a.la.K);
    if (!a.a) {
        const hipError_t e = launch_mx4_quantize(a.x, a.x_bf16, a.ldx, 1, a.la, a.work, s);
        if (e != hipSuccess) return e;
        a.a = (const uint8_t *)a.work;
        a.work = (char *)a.work + round256(a.la.total);
    }
    if (panel) return launch_panel<SRC_FOUR>(a, s);
    const int blocks = p.mblocks * p.nblocks;
    hipLaunchKernelGGL(mx4_product_kernel, dim3((unsigned)(blocks * p.parts)), dim3(256), 0, s, a,
                       p.nblocks, blocks, p.groups_per);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    hipLaunchKernelGGL(mx4_join_kernel, dim3((unsigned)(blocks * (BLOCK_FLOATS / 4 / 256))),
                       dim3(256), 0, s, a, p.nblocks, blocks, p.parts);
    return hipGetLastError();
}

}  // namespace tpk
