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

// a 32 x 32 result (register i: n = n0 + 8(i/4) + 4(lane/32) + i%4)
__device__ __forceinline__ void finish_tile(const Mx4Args &a, int64_t m, int64_t n0, int lane,
                                            const floatx16 &c, bool vec)
{
    if (m >= a.la.rows) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float z[4] = {c[4 * r], c[4 * r + 1], c[4 * r + 2], c[4 * r + 3]};
        const int64_t n = n0 + 8 * r + 4 * (lane >> 5);
        if (a.y_bf16) finish4<true>(a, m, n, z, vec);
        else finish4<false>(a, m, n, z, vec);
    }
}

template <int S0>
struct Step {
    template <int TM, int TN>
    static __device__ __forceinline__ void run(floatx16 (&c)[TM][TN], const intx4 (&fa)[TM],
                                               const uint32_t (&sa)[TM], const intx4 (&fw)[TN],
                                               const uint32_t (&sw)[TN])
    {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                c[i][j] = mfma_fp4<S0>(fw[j], sw[j], fa[i], sa[i], c[i][j]);
    }
};

// ---------------------------------------------------------------------------
// Any size: a wave has TM x TN tiles of 32 x 32, a workgroup 2 x 2 waves, and
// each wave streams its fragments from L1 and L2, a group of k-steps ahead.
// gridDim.y > 1: a part of K each, its sums in fp32 to the workspace.
// ---------------------------------------------------------------------------
template <int TM, int TN>
__global__ __launch_bounds__(256) void mx4_product_kernel(Mx4Args a, int nblocks, int groups_per)
{
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int mb = blockIdx.x / nblocks, nb = blockIdx.x - mb * nblocks;
    const int mt0 = (mb * 2 + (wv >> 1)) * TM, nt0 = (nb * 2 + (wv & 1)) * TN;
    const int ksteps = (int)a.la.ksteps, groups = (int)a.la.groups;
    const int g0 = blockIdx.y * groups_per;
    const int g1 = g0 + groups_per < groups ? g0 + groups_per : groups;
    const char *ca[TM], *cw[TN];
    const char *pa[TM], *pw[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t t = mt0 + i < a.la.tiles ? mt0 + i : a.la.tiles - 1;
        ca[i] = (const char *)a.a + t * ksteps * 1024;
        pa[i] = (const char *)a.a + a.la.off_scales + t * groups * 256;
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int64_t t = nt0 + j < a.lw.tiles ? nt0 + j : a.lw.tiles - 1;
        cw[j] = (const char *)a.w + t * ksteps * 1024;
        pw[j] = (const char *)a.w + a.lw.off_scales + t * groups * 256;
    }
    floatx16 c[TM][TN] = {};
    intx4 fa[4][TM], fw[4][TN];
    uint32_t sa[TM], sw[TN];
    auto fetch = [&](int g, intx4 (&ga)[4][TM], intx4 (&gw)[4][TN], uint32_t (&ha)[TM],
                     uint32_t (&hw)[TN]) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int64_t ks = g * 4 + s < ksteps ? g * 4 + s : ksteps - 1;
#pragma unroll
            for (int i = 0; i < TM; ++i)
                ga[s][i] = *(const intx4 *)(scalar(ca[i] + ks * 1024) + (size_t)(lane * 16u));
#pragma unroll
            for (int j = 0; j < TN; ++j)
                gw[s][j] = *(const intx4 *)(scalar(cw[j] + ks * 1024) + (size_t)(lane * 16u));
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
            ha[i] = *(const uint32_t *)(scalar(pa[i] + (int64_t)g * 256) + (size_t)(lane * 4u));
#pragma unroll
        for (int j = 0; j < TN; ++j)
            hw[j] = *(const uint32_t *)(scalar(pw[j] + (int64_t)g * 256) + (size_t)(lane * 4u));
    };
    fetch(g0, fa, fw, sa, sw);
    for (int g = g0; g < g1; ++g) {
        intx4 na[4][TM], nw[4][TN];
        uint32_t ma[TM], mw[TN];
        fetch(g + 1 < g1 ? g + 1 : g, na, nw, ma, mw);
        const int left = ksteps - g * 4;
        Step<0>::run<TM, TN>(c, fa[0], sa, fw[0], sw);
        if (left > 1) Step<1>::run<TM, TN>(c, fa[1], sa, fw[1], sw);
        if (left > 2) Step<2>::run<TM, TN>(c, fa[2], sa, fw[2], sw);
        if (left > 3) Step<3>::run<TM, TN>(c, fa[3], sa, fw[3], sw);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[s][i] = na[s][i];
#pragma unroll
            for (int j = 0; j < TN; ++j) fw[s][j] = nw[s][j];
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) sa[i] = ma[i];
#pragma unroll
        for (int j = 0; j < TN; ++j) sw[j] = mw[j];
    }
    const int64_t M = a.la.rows, N = a.lw.rows;
    const bool vec = ((uintptr_t)a.y | (uint64_t)(a.ldy * (a.y_bf16 ? 2 : 4))) %
                         (a.y_bf16 ? 8 : 16) == 0;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t m = (int64_t)(mt0 + i) * 32 + (lane & 31), n0 = (int64_t)(nt0 + j) * 32;
            if (gridDim.y == 1) {
                finish_tile(a, m, n0, lane, c[i][j], vec);
            } else if (m < M) {
                float *part = (float *)a.work + ((int64_t)blockIdx.y * M + m) * N;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int64_t n = n0 + 8 * (e / 4) + 4 * (lane >> 5) + e % 4;
                    if (n < N) part[n] = c[i][j][e];
                }
            }
        }
}

// the parts of K in order
__global__ __launch_bounds__(256) void mx4_join_kernel(Mx4Args a, int parts)
{
    const int64_t M = a.la.rows, N = a.lw.rows, n4 = (N + 3) / 4;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= M * n4) return;
    const int64_t m = at / n4, n = (at - m * n4) * 4;
    float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = 0; p < parts; ++p) {
        const float *part = (const float *)a.work + ((int64_t)p * M + m) * N + n;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < N) z[e] += part[e];
    }
    if (a.y_bf16) finish4<true>(a, m, n, z, false);
    else finish4<false>(a, m, n, z, false);
}

constexpr int TM = 4, TN = 2;

struct Plan {
    int mblocks, nblocks, parts, groups_per;
};

// Parts of K so that the workgroups fill the GPU once, each with at least
// four groups of k-steps.
Plan plan_of(int64_t M, int64_t N, int64_t K)
{
    Plan p;
    const int64_t mt = (M + 31) / 32, nt = (N + 31) / 32, groups = (K + 255) / 256;
    p.mblocks = (int)((mt + 2 * TM - 1) / (2 * TM));
    p.nblocks = (int)((nt + 2 * TN - 1) / (2 * TN));
    const int64_t blocks = (int64_t)p.mblocks * p.nblocks;
    int64_t parts = blocks < 256 ? 256 / blocks : 1;
    if (parts > groups / 4) parts = groups / 4;
    if (parts < 1) parts = 1;
    p.groups_per = (int)((groups + parts - 1) / parts);
    p.parts = (int)((groups + p.groups_per - 1) / p.groups_per);
    return p;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

// x in 4 bits, then the parts of K
size_t mx4_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    const Plan p = plan_of(M, N, K);
    return round256(mx4_layout(M, K).total) +
           (p.parts > 1 ? (size_t)p.parts * M * N * sizeof(float) : 0) + 256;
}

hipError_t launch_mx4_product(const Mx4Args &in, hipStream_t s)
{
    Mx4Args a = in;
    const Plan p = plan_of(a.la.rows, a.lw.rows, a.la.K);
    if (!a.a) {
        const hipError_t e = launch_mx4_quantize(a.x, a.x_bf16, a.ldx, 1, a.la, a.work, s);
        if (e != hipSuccess) return e;
        a.a = (const uint8_t *)a.work;
        a.work = (char *)a.work + round256(a.la.total);
    }
    hipLaunchKernelGGL((mx4_product_kernel<TM, TN>),
                       dim3((unsigned)(p.mblocks * p.nblocks), (unsigned)p.parts), dim3(256), 0, s,
                       a, p.nblocks, p.groups_per);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    const int64_t threads = a.la.rows * ((a.lw.rows + 3) / 4);
    hipLaunchKernelGGL(mx4_join_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a,
                       p.parts);
    return hipGetLastError();
}

}  // namespace tpk
