// Norms around a block of a residual stream, with the block's gate and the scale
// of what it adds:
//   f = y / rms_group(y) w_post silu(z),  X = x + scale f,  n = X / rms(X) w_pre,
// rms(v) = sqrt(mean v^2 + eps), and the gradients of everything.
//
// LPR lanes have a row (parts of a wave, or a workgroup of 256 for long rows), NV
// vectors of V elements each, and go from row to row with the weights in
// registers.  All arithmetic is fp32; every output is rounded once (n is taken from
// X before its rounding).  One pass: forward three arrays in and two out, backward
// five in and three out, with the weights' gradients summed per lane in fp32 over 32
// rows at most, and in 64 bits and a fixed order over a workgroup's and over all.
//
// Memory bounds it: 1,597,440 rows of 256 in bf16 forward 864 us (4.7 TB/s, the rate of a
// copy); 258,048 odd rows of 301 in fp32 forward 390 us (4.0 TB/s) and back 547
// (4.5), the join of 1,024 workgroups' sums 26; 1,032,192 rows of 256 in bf16 with gradients
// 1,942 us both ways (3.5 TB/s).
#include "device.hpp"
#include "internal.hpp"

namespace tpk {
namespace {

constexpr int NORM_BLOCKS = 1024;           // workgroups, and parts of the weights' gradients
constexpr int NORM_ROWS = 32;               // rows that a lane adds up in fp32

template <bool BF, int V>
struct Vec {
    typedef typename std::conditional<BF, __bf16, float>::type E;
    typedef E type __attribute__((ext_vector_type(V)));
};

template <bool BF, int V>
__device__ __forceinline__ void load_vec(const void *row, int c, int D, float *x)
{
    typedef typename Vec<BF, V>::E E;
    if (!row || c >= D) {
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = 0.0f;
        return;
    }
    if constexpr (V == 1) {
        x[0] = (float)((const E *)row)[c];
    } else {
        const auto v = *(const typename Vec<BF, V>::type *)((const E *)row + c);
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = (float)v[e];
    }
}

template <bool BF, int V>
__device__ __forceinline__ void store_vec(void *row, int c, int D, const float *x)
{
    typedef typename Vec<BF, V>::E E;
    if (!row || c >= D) return;
    if constexpr (V == 1) {
        ((E *)row)[c] = (E)x[0];
    } else {
        typename Vec<BF, V>::type v;
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = (E)x[e];
        *(typename Vec<BF, V>::type *)((E *)row + c) = v;
    }
}

// Sum over `width` neighbouring lanes (a power of two up to 64), in all of them.
__device__ __forceinline__ float some_lanes_sum(float x, int width)
{
    if (width > 1) x = lane_add<1>(x);
    if (width > 2) x = lane_add<2>(x);
    if (width > 4) x = lane_add<4>(x);
    if (width > 8) x = lane_add<8>(x);
    if (width > 16) x = lane_add<16>(x);
    if (width > 32) x = lane_add<32>(x);
    return x;
}

// Sum over a row's lanes, in all of them.
template <int LPR>
__device__ __forceinline__ float row_total(float x, float *lds)
{
    x = lanes_sum<(LPR < 64 ? LPR : 64)>(x);
    if constexpr (LPR > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        x = (lds[0] + lds[1]) + (lds[2] + lds[3]);
    }
    return x;
}

// Sums of a row's s[j][e] over each group of neighbouring channels, in place.
// mode 0: one group; 1: a group is a power of two of vectors, 2^k lanes; 2: any.
template <int V, int LPR, int NV>
__device__ __forceinline__ void group_sums(const NormArgs &a, int lane, float (*s)[V], float *lds)
{
    if (a.mode == 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float t = 0.0f;
#pragma unroll
            for (int e = 0; e < V; ++e) t += s[j][e];
            t = some_lanes_sum(t, a.group / V);
#pragma unroll
            for (int e = 0; e < V; ++e) s[j][e] = t;
        }
        return;
    }
    if (a.mode == 0) {
        float t = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) t += s[j][e];
        t = row_total<LPR>(t, lds);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) s[j][e] = t;
        return;
    }
    float out[NV][V] = {};              // (channels past the last are in no group)
    for (int g = 0; g < a.groups; ++g) {
        const int lo = g * a.group, hi = lo + a.group;
        float t = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int c = (j * LPR + lane) * V + e;
                t += c >= lo && c < hi ? s[j][e] : 0.0f;
            }
        t = row_total<LPR>(t, lds);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int c = (j * LPR + lane) * V + e;
                if (c >= lo && c < hi) out[j][e] = t;
            }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) s[j][e] = out[j][e];
}

// The hardware's exponential of -z log2(e), rounded once, would be off by |z| 2^-24; what
// the product and log2(e) lost goes back in as a factor, and a step of Newton's to the
// reciprocal.  (expf and a division: 1,597,440 rows of 256 in bf16 905 us against 864.)
__device__ __forceinline__ float norm_sigmoid(float z)
{
    constexpr float L = 1.44269504088896341f, L_LOW = 1.44269504088896341 - (double)L, LN2 = 0.693147180559945309f;
    const float near = __builtin_amdgcn_fmed3f(z, -128.0f, 128.0f);     // (past it e is infinite or 0)
    const float lost = fmaf(near, -L_LOW, fmaf(near, -L, near * L));
    const float d = 1.0f + __builtin_amdgcn_exp2f(z * -L) * fmaf(lost, LN2, 1.0f);
    const float s = __builtin_amdgcn_rcpf(d);
    return d < 1e38f ? fmaf(fmaf(-d, s, 1.0f), s, s) : s;
}

// weights of this lane's channels (1 where there are none)
template <int V, int LPR, int NV>
__device__ __forceinline__ void load_weights(const float *w, int lane, int D, float (*out)[V])
{
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = (j * LPR + lane) * V + e;
            out[j][e] = c < D ? (w ? w[c] : 1.0f) : 0.0f;
        }
}

__device__ __forceinline__ const char *row_of(const NormRows &m, int64_t r)
{
    return m.p ? (const char *)m.p + r * m.ld : nullptr;
}

template <bool BF, int V, int LPR, int NV>
__global__ __launch_bounds__(256) void norm_fwd_kernel(NormArgs a)
{
    __shared__ float lds[4];
    constexpr int RPB = 256 / LPR;
    const int lane = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    float wp[NV][V], sc[NV][V], wq[NV][V];
    load_weights<V, LPR, NV>(a.w_post, lane, a.D, wp);
    load_weights<V, LPR, NV>(a.scale, lane, a.D, sc);
    load_weights<V, LPR, NV>(a.w_pre, lane, a.D, wq);
    const float inv_group = 1.0f / (float)a.group, inv_D = 1.0f / (float)a.D;
    // (all lanes of a workgroup go round together: rows past the last are empty)
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB) {
        const int64_t r = r0 + slot;
        const bool live = r < a.rows;
        float X[NV][V];
#pragma unroll
        for (int j = 0; j < NV; ++j)
            load_vec<BF, V>(live ? row_of(a.x, r) : nullptr, (j * LPR + lane) * V, a.D, X[j]);
        if (a.y.p) {
            float y[NV][V], z[NV][V], s[NV][V];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                load_vec<BF, V>(live ? row_of(a.y, r) : nullptr, (j * LPR + lane) * V, a.D, y[j]);
                load_vec<BF, V>(live ? row_of(a.z, r) : nullptr, (j * LPR + lane) * V, a.D, z[j]);
            }
            if (a.w_post) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) s[j][e] = y[j][e] * y[j][e];
                group_sums<V, LPR, NV>(a, lane, s, lds);
            }
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float f = y[j][e];
                    if (a.w_post) f = f * rsqrtf(s[j][e] * inv_group + a.eps) * wp[j][e];
                    if (a.z.p) f = f * (z[j][e] * norm_sigmoid(z[j][e]));
                    X[j][e] = X[j][e] + sc[j][e] * f;
                }
        }
        float t = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) t += X[j][e] * X[j][e];
        if (live && a.x_out.p)
#pragma unroll
            for (int j = 0; j < NV; ++j)
                store_vec<BF, V>((void *)row_of(a.x_out, r), (j * LPR + lane) * V, a.D, X[j]);
        if (a.n.p) {
            const float rx = rsqrtf(row_total<LPR>(t, lds) * inv_D + a.eps);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float o[V];
#pragma unroll
                for (int e = 0; e < V; ++e) o[e] = X[j][e] * rx * wq[j][e];
                if (live) store_vec<BF, V>((void *)row_of(a.n, r), (j * LPR + lane) * V, a.D, o);
            }
        }
    }
}

// With xn = X rx, t = dn w_pre:   dX = dx_out + rx (t - xn mean(t xn)),
// dw_pre = dn xn, dscale = dX f, df = dX scale, yn = y ry, g = silu(z):
// dw_post = df yn g, dz = df yn w_post silu'(z), d = df w_post g,
// dy = ry (d - yn mean_group(d yn)), dx = dX.
template <bool BF, int V, int LPR, int NV>
__global__ __launch_bounds__(256) void norm_bwd_kernel(NormArgs a)
{
    __shared__ float lds[4];
    constexpr int RPB = 256 / LPR, C = LPR * NV * V;
    const int lane = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    float wp[NV][V], sc[NV][V], wq[NV][V];
    load_weights<V, LPR, NV>(a.w_post, lane, a.D, wp);
    load_weights<V, LPR, NV>(a.scale, lane, a.D, sc);
    load_weights<V, LPR, NV>(a.w_pre, lane, a.D, wq);
    const float inv_group = 1.0f / (float)a.group, inv_D = 1.0f / (float)a.D;
    // this workgroup's part of the weights' gradients, [3][D]: the lanes' sums go there
    __shared__ float join[RPB > 1 ? RPB * C : 1];
    double *part = a.parts + (int64_t)blockIdx.x * 3 * a.D;
    int64_t r0 = (int64_t)blockIdx.x * RPB;
    for (bool more = false; r0 < a.rows; more = true) {
        float gp[NV][V] = {}, gs[NV][V] = {}, gq[NV][V] = {};
        for (int turn = 0; turn < NORM_ROWS && r0 < a.rows; ++turn, r0 += (int64_t)gridDim.x * RPB) {
            const int64_t r = r0 + slot;
            const bool live = r < a.rows;
            float X[NV][V], y[NV][V], z[NV][V], ry[NV][V], dX[NV][V], dn[NV][V];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * LPR + lane) * V;
                load_vec<BF, V>(live ? row_of(a.x, r) : nullptr, c, a.D, X[j]);
                load_vec<BF, V>(live ? row_of(a.y, r) : nullptr, c, a.D, y[j]);
                load_vec<BF, V>(live ? row_of(a.z, r) : nullptr, c, a.D, z[j]);
                load_vec<BF, V>(live ? row_of(a.dx_out, r) : nullptr, c, a.D, dX[j]);
                load_vec<BF, V>(live ? row_of(a.dn, r) : nullptr, c, a.D, dn[j]);
            }
            if (a.y.p && a.w_post) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) ry[j][e] = y[j][e] * y[j][e];
                group_sums<V, LPR, NV>(a, lane, ry, lds);
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        ry[j][e] = rsqrtf(ry[j][e] * inv_group + a.eps);
                        y[j][e] = y[j][e] * ry[j][e];                       // yn
                    }
            }
            if (a.y.p) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float f = y[j][e] * (a.w_post ? wp[j][e] : 1.0f);
                        if (a.z.p) f = f * (z[j][e] * norm_sigmoid(z[j][e]));
                        X[j][e] = X[j][e] + sc[j][e] * f;
                    }
            }
            if (a.dn.p) {
                float t = 0.0f, u = 0.0f;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        t += X[j][e] * X[j][e];
                        u += X[j][e] * (dn[j][e] * wq[j][e]);
                    }
                t = row_total<LPR>(t, lds);
                u = row_total<LPR>(u, lds);
                const float rx = rsqrtf(t * inv_D + a.eps), m = u * rx * inv_D;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float xn = X[j][e] * rx;
                        dX[j][e] += rx * (dn[j][e] * wq[j][e] - xn * m);
                        gq[j][e] += dn[j][e] * xn;
                    }
            }
            if (live)
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    store_vec<BF, V>((void *)row_of(a.dx, r), (j * LPR + lane) * V, a.D, dX[j]);
            if (!a.y.p) continue;
            float s[NV][V];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float dz[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float w = a.w_post ? wp[j][e] : 1.0f, yn = y[j][e];
                    float g = 1.0f, slope = 0.0f;
                    if (a.z.p) {
                        const float sg = norm_sigmoid(z[j][e]);
                        g = z[j][e] * sg;
                        slope = sg * (1.0f + z[j][e] * (1.0f - sg));
                    }
                    gs[j][e] += dX[j][e] * (yn * w * g);
                    const float df = dX[j][e] * sc[j][e];
                    gp[j][e] += df * (yn * g);
                    dz[e] = df * (yn * w) * slope;
                    dX[j][e] = df * w * g;                                  // d
                    s[j][e] = dX[j][e] * yn;
                }
                if (live && a.dz.p) store_vec<BF, V>((void *)row_of(a.dz, r), (j * LPR + lane) * V, a.D, dz);
            }
            if (a.w_post) {
                group_sums<V, LPR, NV>(a, lane, s, lds);
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        dX[j][e] = ry[j][e] * (dX[j][e] - y[j][e] * (s[j][e] * inv_group));
            }
            if (live)
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    store_vec<BF, V>((void *)row_of(a.dy, r), (j * LPR + lane) * V, a.D, dX[j]);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            float (*g)[V] = k == 0 ? gp : k == 1 ? gs : gq;
            if constexpr (RPB > 1) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) join[slot * C + (j * LPR + lane) * V + e] = g[j][e];
                __syncthreads();
                for (int c = threadIdx.x; c < a.D; c += 256) {
                    double t = more ? part[k * a.D + c] : 0.0;
#pragma unroll
                    for (int q = 0; q < RPB; ++q) t += (double)join[q * C + c];
                    part[k * a.D + c] = t;
                }
            } else {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int c = (j * LPR + lane) * V + e;
                        if (c < a.D) part[k * a.D + c] = (more ? part[k * a.D + c] : 0.0) + (double)g[j][e];
                    }
            }
        }
    }
}

// sums of the workgroups' parts, 16 channels a workgroup, 16 rows at a time
__global__ __launch_bounds__(256) void norm_join_kernel(const double *parts, int blocks, int D, float *w0, float *w1,
                                                        float *w2)
{
    __shared__ double red[16][17];
    const int c = threadIdx.x & 15, q = threadIdx.x >> 4, d = blockIdx.x * 16 + c;
    double s = 0.0;
    if (d < 3 * D)
        for (int k = q; k < blocks; k += 16) s += parts[(int64_t)k * 3 * D + d];
    red[q][c] = s;
    __syncthreads();
    if (q != 0 || d >= 3 * D) return;
    s = 0.0;
    for (int k = 0; k < 16; ++k) s += red[k][c];
    float *to = d < D ? w0 : d < 2 * D ? w1 : w2;
    if (to) to[d % D] = (float)s;
}

template <bool BF, int V, int LPR, int NV>
void start_norm(NormArgs &a, bool backward, hipStream_t s)
{
    constexpr int RPB = 256 / LPR;
    const int64_t want = (a.rows + RPB - 1) / RPB;
    const int blocks = (int)(want < NORM_BLOCKS * (backward ? 1 : 2) ? want : NORM_BLOCKS * (backward ? 1 : 2));
    // group sums without LDS where a group is 2^k neighbouring lanes of one row
    const int lanes = a.group / V;
    a.mode = a.groups == 1 ? 0
             : a.group % V == 0 && (lanes & (lanes - 1)) == 0 && lanes <= (LPR < 64 ? LPR : 64) ? 1 : 2;
    if (!backward) {
        hipLaunchKernelGGL((norm_fwd_kernel<BF, V, LPR, NV>), dim3(blocks), dim3(256), 0, s, a);
        return;
    }
    hipLaunchKernelGGL((norm_bwd_kernel<BF, V, LPR, NV>), dim3(blocks), dim3(256), 0, s, a);
    if (a.dw_post || a.dscale || a.dw_pre)
        hipLaunchKernelGGL(norm_join_kernel, dim3((3 * a.D + 15) / 16), dim3(256), 0, s, a.parts, blocks, a.D,
                           a.dw_post, a.dscale, a.dw_pre);
}

template <bool BF>
void start_norm(NormArgs &a, bool backward, hipStream_t s)
{
    constexpr int V = BF ? 8 : 4;
    bool vec = a.D % V == 0;
    for (const NormRows *m : {&a.x, &a.y, &a.z, &a.x_out, &a.n, &a.dx_out, &a.dn, &a.dx, &a.dy, &a.dz})
        vec = vec && (!m->p || ((uintptr_t)m->p | m->ld) % 16 == 0);
    if (vec) {
        const int v = a.D / V;
        if (v <= 8) start_norm<BF, V, 8, 1>(a, backward, s);
        else if (v <= 16) start_norm<BF, V, 16, 1>(a, backward, s);
        else if (v <= 32) start_norm<BF, V, 32, 1>(a, backward, s);
        else if (v <= 64) start_norm<BF, V, 64, 1>(a, backward, s);
        else if (v <= 128) start_norm<BF, V, 64, 2>(a, backward, s);
        else if (v <= 256) start_norm<BF, V, 256, 1>(a, backward, s);
        else if (v <= 512) start_norm<BF, V, 256, 2>(a, backward, s);
        else start_norm<BF, V, 256, 4>(a, backward, s);
        return;
    }
    // Element by element: 16-byte loads of rows that start anywhere, with the row's last
    // vector ending with it, took 1.46 ms where this takes 0.93 (258,048 rows of 301 in fp32,
    // with gradients; with registers for 512 channels in place of 320, 0.98).
    const int D = a.D;
    if (D <= 64) start_norm<BF, 1, 64, 1>(a, backward, s);
    else if (D <= 128) start_norm<BF, 1, 64, 2>(a, backward, s);
    else if (D <= 192) start_norm<BF, 1, 64, 3>(a, backward, s);
    else if (D <= 256) start_norm<BF, 1, 64, 4>(a, backward, s);
    else if (D <= 320) start_norm<BF, 1, 64, 5>(a, backward, s);
    else if (D <= 384) start_norm<BF, 1, 64, 6>(a, backward, s);
    else if (D <= 512) start_norm<BF, 1, 64, 8>(a, backward, s);
    else if (D <= 1024) start_norm<BF, 1, 256, 4>(a, backward, s);
    else if (D <= 2048) start_norm<BF, 1, 256, 8>(a, backward, s);
    else start_norm<BF, 1, 256, 16>(a, backward, s);
}

}  // namespace

size_t norm_workspace_bytes(int D)
{
    return ((size_t)NORM_BLOCKS * 3 * D * sizeof(double) + 255) / 256 * 256;
}

hipError_t launch_norm(NormArgs &a, bool backward, hipStream_t s)
{
    a.group = a.D / a.groups;
    if (a.bf16) start_norm<true>(a, backward, s);
    else start_norm<false>(a, backward, s);
    return hipGetLastError();
}

}  // namespace tpk
