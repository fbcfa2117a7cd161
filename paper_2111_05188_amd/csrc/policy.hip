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
// gradient of theirs there or not.  The arithmetic hides behind the rows' loads:
// 1,597,440 rows of 100, bf16, 453 us (4.3 TB/s); 258,048 of 30, fp32, half of them past their
// sequences' ends, 41 us (1.9 TB/s of what is read and written), of which the join of the
// workgroups' sums takes 6.
// LPR lanes have a row.
#include "device.hpp"
#include "internal.hpp"

namespace tpk {
namespace {

// Workgroups, and parts of the sums.  1,597,440 rows of 100: 533 us with 1,024, 453
// with 2,048; 258,048 rows of 30, which each have few of: 41 and 48.
constexpr int POLICY_BLOCKS = 2048, POLICY_FEW = 1024;
// up to so many sequences every workgroup adds up the lengths by itself
constexpr int POLICY_LENS = 8192;
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
struct Some {
    typedef E vec __attribute__((ext_vector_type(V)));
    vec v;
    __device__ __forceinline__ void load(const E *p, int c, int n)
    {
        v = vec{};
        if (c < n) v = *(const vec *)(p + c);
    }
    __device__ __forceinline__ double at(int e) const { return (double)(float)v[e]; }
};

template <bool BF, int V, int LPR, int NV>
__global__ __launch_bounds__(256) void policy_kernel(PolicyArgs a)
{
    typedef typename std::conditional<BF, __bf16, float>::type E;
    // (a gradient that is rounded to bf16 is worked out in 32 bits)
    typedef typename std::conditional<BF, float, double>::type F;
    constexpr int RPB = 256 / LPR, C = LPR * NV * V;
    const int lane = threadIdx.x % LPR, slot = threadIdx.x / LPR, n = a.n;
    double inv[NV][V], tilt[NV][V], dls[NV][V] = {};
    double ls_sum = 0.0, kl0 = 0.0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = (j * LPR + lane) * V + e;
            const double ls = c < n ? (double)a.log_std[c] : 0.0;
            const double lr = c < n && a.log_std_ref ? (double)a.log_std_ref[c] : ls;
            inv[j][e] = c < n ? exp(-ls) : 0.0;
            const double spread = exp(2.0 * (lr - ls));
            tilt[j][e] = 1.0 - spread;
            ls_sum += ls;
            kl0 += c < n ? ls - lr - 0.5 + 0.5 * spread : 0.0;
        }
    ls_sum = lanes_sum<LPR>(ls_sum) + 0.5 * LN_2PI * n;
    kl0 = lanes_sum<LPR>(kl0);
    const int64_t rows = (int64_t)a.T * a.B;
    __shared__ double red[3][RPB > 4 ? RPB : 4];
    double N = (double)rows;
    if (a.len && a.B > POLICY_LENS) {
        N = a.count[0];
    } else if (a.len) {                     // (whole numbers: any order gives the same)
        int64_t s = 0;
        for (int b = threadIdx.x; b < a.B; b += 256) {
            const int l = a.len[b];
            s += l < 0 ? 0 : l > a.T ? a.T : l;
        }
        const double d = lanes_sum<64>((double)s);
        if ((threadIdx.x & 63) == 0) red[0][threadIdx.x >> 6] = d;
        __syncthreads();
        N = red[0][0] + red[0][1] + red[0][2] + red[0][3];
        __syncthreads();
        if (blockIdx.x == 0 && threadIdx.x == 0) a.count[0] = N;
    }
    const double share = N > 0.0 ? 1.0 / N : 0.0, k = a.kl_coef * share;
    const double lo = 1.0 - a.clip_low, hi = 1.0 + a.clip_high;
    double sum_s = 0.0, sum_kl = 0.0, sum_out = 0.0;
    // the next row's loads are under way while one is worked on; (t, b) goes along
    Some<E, V> mu[NV];
    Some<float, V> x[NV], m[NV];
    float logp_old = 0.0f, adv = 0.0f;
    bool live = false;
    const int64_t hop = (int64_t)gridDim.x * RPB, hop_t = hop / a.B;
    const int hop_b = (int)(hop - hop_t * a.B);
    int64_t r = (int64_t)blockIdx.x * RPB + slot, t = r / a.B;
    int b = (int)(r - t * a.B);
    auto fetch = [&] {
        live = r < rows && (!a.len || t < a.len[b]);
        if (!live) return;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * LPR + lane) * V;
            mu[j].load((const E *)a.mu + r * a.ld_mu, c, n);
            x[j].load(a.action + r * n, c, n);
            if (a.mu_ref) m[j].load(a.mu_ref + r * n, c, n);
        }
        logp_old = a.logp[r];
        adv = a.adv[r];
    };
    fetch();
    while (r < rows) {
        E *dmu = (E *)a.dmu + r * a.ld_dmu;
        const bool on = live;
        const double old = (double)logp_old, A = (double)adv;
        double z[NV][V], o[NV][V];
        double w = 0.0, q = 0.0, kl = 0.0;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                z[j][e] = (x[j].at(e) - mu[j].at(e)) * inv[j][e];
                o[j][e] = a.mu_ref ? (mu[j].at(e) - m[j].at(e)) * inv[j][e] : 0.0;
                q = fma(z[j][e], z[j][e], q);
                kl = fma(o[j][e], o[j][e], kl);
            }
        r += hop;
        t += hop_t;
        b += hop_b;
        if (b >= a.B) {
            b -= a.B;
            ++t;
        }
        fetch();
        if (on) {
            q = lanes_sum<LPR>(q);
            kl = lanes_sum<LPR>(kl);
            const double ratio = exp(-0.5 * q - ls_sum - old);
            const double clipped = ratio < lo ? lo : ratio > hi ? hi : ratio;
            const double s1 = ratio * A, s2 = clipped * A;
            // (a NaN that the row brought goes on to the gradient, infinity times no advantage does not)
            const bool open = s1 <= s2 || ratio != ratio || A != A;
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
            F d[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                d[e] = 0;
                if (!on) continue;
                const double Z = z[j][e], O = o[j][e];
                d[e] = (F)w * (F)Z;
                double g = w * fma(Z, Z, -1.0);
                if (a.mu_ref) {
                    d[e] += (F)k * (F)O;
                    g = fma(k, fma(-O, O, tilt[j][e]), g);
                }
                d[e] *= (F)inv[j][e];
                dls[j][e] += g;
            }
            if (c < n) {
                if constexpr (V == 1) {
                    dmu[c] = (E)(float)d[0];
                } else {
                    typedef E vec __attribute__((ext_vector_type(V)));
                    vec v;
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] = (E)(float)d[e];
                    *(vec *)(dmu + c) = v;
                }
            }
        }
    }
    // this workgroup's sums
    __shared__ double join[RPB * C];
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
    const int most = want < 32 * POLICY_BLOCKS ? POLICY_FEW : POLICY_BLOCKS;
    const int blocks = (int)(want < most ? want : most);
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
    if (a.len && a.B > POLICY_LENS) {
        hipLaunchKernelGGL(policy_count_kernel, dim3(1), dim3(1024), 0, s, a.len, a.T, a.B, a.count);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.bf16) start_policy<true>(a, s);
    else start_policy<false>(a, s);
    return hipGetLastError();
}

}  // namespace tpk
