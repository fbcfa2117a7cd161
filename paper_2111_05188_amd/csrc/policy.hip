// Clipped policy loss of a diagonal Gaussian policy, with entropy and KL, and its
// gradient, in one pass over the stored rows.  A row with mean mu, action a,
// advantage A, the log-probability it was drawn with and, where there is a
// reference policy, its mean m:
//   z = (a - mu)/sigma, logp = sum(-z^2/2 - log sigma) - n/2 ln 2pi,
//   rho = exp(logp - logp_old), s = min(rho A, clip(rho, 1 - lo, 1 + hi) A),
//   KL(ref || pi) = sum log sigma/sigma_r - 1/2 + sigma_r^2/(2 sigma^2) + o^2/2,
//   o = (mu - m)/sigma,
//   L = -mean s + kl mean KL - ent H,
// means over the N rows that the sequences have.  With w = -rho A / N where the
// minimum is rho A, else 0, and k = kl / N:
//   dmu = (w z + k o) / sigma,
//   dlog_sigma = sum over rows of w (z^2 - 1) + k (1 - sigma_r^2/sigma^2 - o^2), - ent.
//
// Everything up to the ratio is in 64 bits: a rounding of 2^-24 in sums of some
// hundred would put a few of a million rows on the other side of the clip, with a
// gradient of theirs there or not.  The arithmetic hides behind the rows' loads.
// LPR lanes have a row.
#include "device.hpp"
#include "internal.hpp"

namespace tpk {
namespace {

constexpr int POLICY_BLOCKS = 1024;
constexpr double LN_2PI = 1.83787706640934533908;

// N, the rows that the sequences have
__global__ __launch_bounds__(1024) void policy_count_kernel(const int32_t *len, int T, int B, double *out)
{
    __shared__ double red[16];
    double s = 0.0;
    for (int b = threadIdx.x; b < B; b += 1024) {
        const int l = len[b];
        s += (double)(l < 0 ? 0 : l > T ? T : l);
    }
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x != 0) return;
    s = 0.0;
    for (int i = 0; i < 16; ++i) s += red[i];
    out[0] = s;
}

template <class E, int V>
__device__ __forceinline__ void load_some(const E *p, int c, int n, double *x)
{
    typedef E vec __attribute__((ext_vector_type(V)));
    if (c >= n) {
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = 0.0;
        return;
    }
    if constexpr (V == 1) {
        x[0] = (double)(float)p[c];
    } else {
        const vec v = *(const vec *)(p + c);
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = (double)(float)v[e];
    }
}

template <int LPR>
__device__ __forceinline__ double lanes_sum(double x)
{
#pragma unroll
    for (int m = 1; m < LPR; m <<= 1) x += __shfl_xor(x, m);
    return x;
}

template <bool BF, int V, int LPR, int NV>
__global__ __launch_bounds__(256) void policy_kernel(PolicyArgs a)
{
    typedef typename std::conditional<BF, __bf16, float>::type E;
    constexpr int RPB = 256 / LPR, C = LPR * NV * V;
    const int lane = threadIdx.x % LPR, slot = threadIdx.x / LPR, n = a.n;
    double inv[NV][V], spread[NV][V], dls[NV][V] = {};
    double ls_sum = 0.0, kl0 = 0.0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = (j * LPR + lane) * V + e;
            const double ls = c < n ? (double)a.log_std[c] : 0.0;
            const double lr = c < n && a.log_std_ref ? (double)a.log_std_ref[c] : ls;
            inv[j][e] = c < n ? exp(-ls) : 0.0;
            spread[j][e] = exp(2.0 * (lr - ls));
            ls_sum += ls;
            kl0 += c < n ? ls - lr - 0.5 + 0.5 * spread[j][e] : 0.0;
        }
    ls_sum = lanes_sum<LPR>(ls_sum) + 0.5 * LN_2PI * n;
    kl0 = lanes_sum<LPR>(kl0);
    const int64_t rows = (int64_t)a.T * a.B;
    const double N = a.len ? a.count[0] : (double)rows;
    const double share = N > 0.0 ? 1.0 / N : 0.0, k = a.kl_coef * share;
    const double lo = 1.0 - a.clip_low, hi = 1.0 + a.clip_high;
    double sum_s = 0.0, sum_kl = 0.0, sum_out = 0.0;
    for (int64_t r = (int64_t)blockIdx.x * RPB + slot; r < rows; r += (int64_t)gridDim.x * RPB) {
        E *dmu = (E *)a.dmu + r * a.ld_dmu;
        bool live = true;
        if (a.len) {
            const int64_t t = r / a.B;
            live = t < a.len[r - t * a.B];
        }
        double z[NV][V], o[NV][V], d[NV][V];
        double w = 0.0;
        if (live) {
            double q = 0.0, kl = 0.0;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * LPR + lane) * V;
                double mu[V], x[V], m[V];
                load_some<E, V>((const E *)a.mu + r * a.ld_mu, c, n, mu);
                load_some<float, V>(a.action + r * n, c, n, x);
                if (a.mu_ref) load_some<float, V>(a.mu_ref + r * n, c, n, m);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    z[j][e] = (x[e] - mu[e]) * inv[j][e];
                    o[j][e] = a.mu_ref ? (mu[e] - m[e]) * inv[j][e] : 0.0;
                    q = fma(z[j][e], z[j][e], q);
                    kl = fma(o[j][e], o[j][e], kl);
                }
            }
            q = lanes_sum<LPR>(q);
            kl = lanes_sum<LPR>(kl);
            const double ratio = exp(-0.5 * q - ls_sum - (double)a.logp[r]);
            const double A = (double)a.adv[r];
            const double clipped = ratio < lo ? lo : ratio > hi ? hi : ratio;
            const double s1 = ratio * A, s2 = clipped * A;
            const bool open = s1 <= s2;
            w = open ? -s1 * share : 0.0;
            if (lane == 0) {
                sum_s += open ? s1 : s2;
                if (a.mu_ref) sum_kl += kl0 + 0.5 * kl;
                sum_out += ratio < lo || ratio > hi ? 1.0 : 0.0;
            }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * LPR + lane) * V;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                d[j][e] = 0.0;
                if (!live) continue;
                d[j][e] = w * z[j][e] * inv[j][e];
                double g = w * (z[j][e] * z[j][e] - 1.0);
                if (a.mu_ref) {
                    d[j][e] += k * o[j][e] * inv[j][e];
                    g += k * (1.0 - spread[j][e] - o[j][e] * o[j][e]);
                }
                dls[j][e] += g;
            }
            if (c < n) {
                if constexpr (V == 1) {
                    dmu[c] = (E)(float)d[j][0];
                } else {
                    typedef E vec __attribute__((ext_vector_type(V)));
                    vec v;
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] = (E)(float)d[j][e];
                    *(vec *)(dmu + c) = v;
                }
            }
        }
    }
    // this workgroup's sums
    __shared__ double join[RPB * C];
    __shared__ double red[3][RPB];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) join[slot * C + (j * LPR + lane) * V + e] = dls[j][e];
    if (lane == 0) {
        red[0][slot] = sum_s;
        red[1][slot] = sum_kl;
        red[2][slot] = sum_out;
    }
    __syncthreads();
    double *part = a.parts + (int64_t)blockIdx.x * (n + 3);
    for (int c = threadIdx.x; c < n + 3; c += 256) {
        double t = 0.0;
        for (int q = 0; q < RPB; ++q) t += c < 3 ? red[c][q] : join[q * C + c - 3];
        part[c] = t;
    }
}

// the workgroups' sums in a fixed order: one workgroup for each column of them
__global__ __launch_bounds__(256) void policy_join_kernel(PolicyArgs a, int blocks)
{
    __shared__ double red[4];
    const int c = blockIdx.x, n = a.n;
    auto total = [&](int col) {
        double s = 0.0;
        for (int q = threadIdx.x; q < blocks; q += 256) s += a.parts[(int64_t)q * (n + 3) + col];
        s = wave_sum(s);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
        __syncthreads();
        return (red[0] + red[1]) + (red[2] + red[3]);
    };
    if (c > 0) {
        const double s = total(c + 2);
        if (threadIdx.x == 0) a.dlog_std[c - 1] = (float)(s - a.ent_coef);
        return;
    }
    const double rows = (double)((int64_t)a.T * a.B), N = a.len ? a.count[0] : rows;
    const double share = N > 0.0 ? 1.0 / N : 0.0;
    const double s = total(0), kl = total(1), out = total(2);
    if (threadIdx.x != 0) return;
    double H = 0.0;
    for (int i = 0; i < n; ++i) H += (double)a.log_std[i] + 0.5 * (1.0 + LN_2PI);
    const double policy = N > 0.0 ? -s * share : 0.0, mean_kl = kl * share;
    a.stats[0] = policy + a.kl_coef * mean_kl - a.ent_coef * H;
    a.stats[1] = policy;
    a.stats[2] = mean_kl;
    a.stats[3] = H;
    a.stats[4] = out * share;
    a.stats[5] = N;
}

template <bool BF, int V, int LPR, int NV>
void start_policy(PolicyArgs &a, hipStream_t s)
{
    constexpr int RPB = 256 / LPR;
    const int64_t want = ((int64_t)a.T * a.B + RPB - 1) / RPB;
    const int blocks = (int)(want < POLICY_BLOCKS ? want : POLICY_BLOCKS);
    hipLaunchKernelGGL((policy_kernel<BF, V, LPR, NV>), dim3(blocks), dim3(256), 0, s, a);
    hipLaunchKernelGGL(policy_join_kernel, dim3(a.n + 1), dim3(256), 0, s, a, blocks);
}

template <bool BF>
void start_policy(PolicyArgs &a, hipStream_t s)
{
    const size_t es = BF ? 2 : 4;
    const auto allows = [&](int V) {
        return a.n % V == 0 && ((uintptr_t)a.mu | (uintptr_t)a.dmu | a.ld_mu * es | a.ld_dmu * es) % (V * es) == 0 &&
               ((uintptr_t)a.action | (uintptr_t)a.mu_ref) % (4 * V) == 0;
    };
    const int n = a.n;
    if (allows(4)) {
        if (n <= 32) start_policy<BF, 4, 8, 1>(a, s);
        else if (n <= 64) start_policy<BF, 4, 16, 1>(a, s);
        else start_policy<BF, 4, 32, 1>(a, s);
    } else if (allows(2)) {
        if (n <= 16) start_policy<BF, 2, 8, 1>(a, s);
        else if (n <= 32) start_policy<BF, 2, 16, 1>(a, s);
        else if (n <= 64) start_policy<BF, 2, 32, 1>(a, s);
        else start_policy<BF, 2, 64, 1>(a, s);
    } else {
        if (n <= 8) start_policy<BF, 1, 8, 1>(a, s);
        else if (n <= 16) start_policy<BF, 1, 16, 1>(a, s);
        else if (n <= 32) start_policy<BF, 1, 32, 1>(a, s);
        else if (n <= 64) start_policy<BF, 1, 64, 1>(a, s);
        else start_policy<BF, 1, 64, 2>(a, s);
    }
}

}  // namespace

size_t policy_workspace_bytes(int n)
{
    return (256 + (size_t)POLICY_BLOCKS * (n + 3) * sizeof(double) + 255) / 256 * 256;
}

hipError_t launch_policy_loss(PolicyArgs &a, hipStream_t s)
{
    a.count = (double *)a.work;
    a.parts = (double *)((char *)a.work + 256);
    if (a.len) {
        hipLaunchKernelGGL(policy_count_kernel, dim3(1), dim3(1024), 0, s, a.len, a.T, a.B, a.count);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.bf16) start_policy<true>(a, s);
    else start_policy<false>(a, s);
    return hipGetLastError();
}

}  // namespace tpk
