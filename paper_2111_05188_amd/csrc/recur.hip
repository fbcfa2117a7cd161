// Gated linear recurrence over bars: whole sequences, their gradients, and one
// step.  Channel d of sequence b, pre-activations x, r, i:
//   rho = 1/(1+exp(-r)), iota = 1/(1+exp(-i)), L = -8 softplus(lambda_d) rho,
//   a = exp(L), beta = sqrt(1 - a^2), u = beta iota x, h <- a h + u.
//
// A wave holds 64 lanes x V neighbouring channels of one sequence, so episode
// ends and lengths are scalars of the wave.  Steps come in chunks of C; a
// chunk's loads are issued one chunk (of this wave) ahead.  W waves of a
// workgroup take neighbouring chunks: each reduces its own to the map
// h -> P h + H, the maps go through LDS, and every wave starts from its own
// carry.  S segments split a long sequence over workgroups the same way, with
// the maps of all segments from a first launch.
//
// With many sequences the memory bounds it: 390 steps x 4,096 sequences x 512
// channels in bf16 take 1.32 ms, 6.6 GB at 5.0 TB/s, and 3.8 ms with the
// gradients (18.9 GB at 4.9: the gates are read again, and the states before
// every chunk are kept instead of all of them).
//
// 1 - a^2 comes from a - 1 by a polynomial rather than from a: long memories
// have a within 1e-4 of 1, and what fp32 leaves of 1 - a is what their states
// are made of.
#include "device.hpp"
#include "internal.hpp"

namespace tpk {
namespace {

constexpr int C = RECUR_CHUNK;
constexpr float LOG2E = 1.44269504088896341f;
constexpr float RATE = 8.0f;

// ---------------------------------------------------------------------------
// V neighbouring elements of a row
// ---------------------------------------------------------------------------
template <int BYTES> struct RawOf;
template <> struct RawOf<2> { typedef uint16_t type; };
template <> struct RawOf<4> { typedef uint32_t type; };
template <> struct RawOf<8> {
    typedef uint32_t type __attribute__((ext_vector_type(2)));
};
template <> struct RawOf<16> {
    typedef uint32_t type __attribute__((ext_vector_type(4)));
};

template <bool BF, int V>
using Raw = typename RawOf<(BF ? 2 : 4) * V>::type;

template <bool BF, int V, bool ONCE = false>
__device__ __forceinline__ Raw<BF, V> load_row(const void *row, uint32_t d)
{
    return load_at<Raw<BF, V>, ONCE>(row, d * (BF ? 2u : 4u));
}

template <bool BF, int V>
__device__ __forceinline__ void unpack(const Raw<BF, V> &raw, float *v)
{
    if constexpr (BF && V == 1) {
        v[0] = __uint_as_float((uint32_t)raw << 16);
    } else {
        uint32_t w[BF ? V / 2 : V];
        __builtin_memcpy(w, &raw, sizeof w);
#pragma unroll
        for (int e = 0; e < V; ++e)
            v[e] = __uint_as_float(!BF ? w[e] : e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    }
}

// bf16: round to nearest even, the only rounding of an output
template <bool BF, int V, bool ONCE = false>
__device__ __forceinline__ void store_row(void *row, uint32_t d, const float *v)
{
    Raw<BF, V> raw;
    if constexpr (BF) {
        __bf16 w[V];
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = to_bf16(v[e]);
        __builtin_memcpy(&raw, w, sizeof raw);
    } else {
        __builtin_memcpy(&raw, v, sizeof raw);
    }
    store_at<ONCE>(row, d * (BF ? 2u : 4u), raw);
}

// V neighbouring fp32 states of a row of D (aligned to a dword each)
template <int V, bool ONCE>
__device__ __forceinline__ void load_states(const float *row, uint32_t d, float *v)
{
    typedef float F __attribute__((ext_vector_type(V), aligned(4)));
    const F f = load_at<F, ONCE>(row, d * 4u);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = f[e];
}

template <int V, bool ONCE>
__device__ __forceinline__ void store_states(float *row, uint32_t d, const float *v)
{
    typedef float F __attribute__((ext_vector_type(V), aligned(4)));
    F f;
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = v[e];
    store_at<ONCE>(row, d * 4u, f);
}

template <int V>
__device__ __forceinline__ void store_f32(float *p, const float *v)
{
#pragma unroll
    for (int e = 0; e < V; ++e) p[e] = v[e];
}

// ---------------------------------------------------------------------------
// gates
// ---------------------------------------------------------------------------
__device__ __forceinline__ float softplus(float x)
{
    // (NaN stays NaN)
    return (x > 0.0f ? x : 0.0f) + log1pf(expf(-fabsf(x))) + (x != x ? x : 0.0f);
}

__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(x * -LOG2E); }

// a = exp(L) and a - 1 of L = -s rho <= 0 (L2 = L log2 e): near 0 from L + L^2
// q(L), q fitted for the least relative error of a - 1 (fp32 7e-8 with
// rounding; for results that go to bf16 3e-7), else from the hardware exp2.
// a is never 0, so that an infinite state stays one (adding the smallest normal
// number changes nothing above 2^-101, and leaves a NaN one).
template <bool BF>
__device__ __forceinline__ bool decay(float L, float L2, float &a, float &am1)
{
    const float far = __builtin_amdgcn_exp2f(L2) + 0x1p-126f;
    float q;
    if constexpr (BF) {
        q = 0x1.362a9cp-5f;
        q = fmaf(q, L, 0x1.543758p-3f);
        q = fmaf(q, L, 0x1.fffa18p-2f);
    } else {
        q = 0x1.27275ep-10f;
        q = fmaf(q, L, 0x1.0c7a58p-7f);
        q = fmaf(q, L, 0x1.550cbcp-5f);
        q = fmaf(q, L, 0x1.55535ap-3f);
        q = fmaf(q, L, 0x1.fffff6p-2f);
    }
    const float near = fmaf(L * L, q, L);
    const bool is_near = L > (BF ? -0.25f : -0.5f);
    a = is_near ? 1.0f + near : far;
    am1 = is_near ? near : far - 1.0f;
    return is_near;
}

// What a chunk keeps of a.  bf16: a itself.  fp32: a - 1 (<= 0) where that is
// the exact one of the two, else a (> 0), so that neither a long memory's 1 - a
// nor a short one's a loses digits.
template <bool BF>
__device__ __forceinline__ float keep(bool is_near, float a, float am1)
{
    if constexpr (BF) return a;
    return is_near ? am1 : a;
}

template <bool BF> constexpr float KEEP_ONE = BF ? 1.0f : 0.0f;   // a = 1

// (a - 1) h of an infinite h must not meet h: there the largest finite number
// stands for it (and for a NaN, which the sum has all the same)
__device__ __forceinline__ float finite(float h)
{
    return __builtin_amdgcn_fmed3f(h, -__FLT_MAX__, __FLT_MAX__);
}

// a h + u
template <bool BF>
__device__ __forceinline__ float advance(float c, float h, float u)
{
    if constexpr (BF) return fmaf(c, h, u);
    return fmaf(c, c > 0.0f ? h : finite(h), c > 0.0f ? u : h + u);
}

// a g
template <bool BF>
__device__ __forceinline__ float fade(float c, float g)
{
    if constexpr (BF) return c * g;
    return fmaf(c, c > 0.0f ? g : finite(g), c > 0.0f ? 0.0f : g);
}

// a P of a product of decays P, which is never infinite
template <bool BF>
__device__ __forceinline__ float fade_p(float c, float P)
{
    if constexpr (BF) return c * P;
    return fmaf(c, P, c > 0.0f ? 0.0f : P);
}

// h -> a h + u
template <bool BF>
__device__ __forceinline__ void gate(float x, float r, float i, float s, float s2, float &c,
                                     float &u)
{
    const float rho = __builtin_amdgcn_rcpf(1.0f + exp_neg(r));
    const float iota = __builtin_amdgcn_rcpf(1.0f + exp_neg(i));
    float a, am1;
    const bool is_near = decay<BF>(-(s * rho), -(s2 * rho), a, am1);
    c = keep<BF>(is_near, a, am1);
    u = __builtin_amdgcn_sqrtf(-am1 * (2.0f + am1)) * (iota * x);
}

// what the gradients need besides: dx = g cx, di = g ci, w = g cw, dr = w cr
template <bool BF>
__device__ __forceinline__ void gate_grad(float x, float r, float i, float s, float s2,
                                          float hprev, float &c, float &u, float &cx, float &ci,
                                          float &cw, float &cr)
{
    const float er = exp_neg(r), ei = exp_neg(i);
    const float rho = __builtin_amdgcn_rcpf(1.0f + er), iota = __builtin_amdgcn_rcpf(1.0f + ei);
    const float L = -(s * rho);
    float a, am1;
    const bool is_near = decay<BF>(L, -(s2 * rho), a, am1);
    c = keep<BF>(is_near, a, am1);
    float v = -am1 * (2.0f + am1);
    v = v < 1e-37f ? 1e-37f : v;            // L = 0: beta = L / beta = 0
    const float rb = __builtin_amdgcn_rsqf(v), beta = v * rb, q = iota * x;
    // 1 - sigmoid: from exp(-z) where 1 - sigmoid(z) would cancel
    const float ni = ei < 1.0f ? ei * iota : 1.0f - iota;
    cr = er < 1.0f ? er * rho : 1.0f - rho;
    u = beta * q;
    cx = beta * iota;
    ci = u * ni;
    cw = a * (L * hprev - (q * a) * (L * rb));
}

// ---------------------------------------------------------------------------
// a wave's place
// ---------------------------------------------------------------------------
template <int V, int W>
struct Place {
    int lane, w, b, d;
    bool live;            // this lane's channels exist
    uint32_t dc;          // its channels, or the last ones
    int len, t0, t1;
};

template <int W> constexpr int GROUP = W == 1 ? 4 : 1;

template <int V, int W>
__device__ __forceinline__ bool place(const RecurArgs &a, int segment, Place<V, W> &p)
{
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = blockIdx.x * GROUP<W> + (W == 1 ? wv : 0);
    if (unit >= a.units) return false;
    p.lane = threadIdx.x & 63;
    p.w = W == 1 ? 0 : wv;
    p.b = unit / a.blocks_d;
    p.d = (unit - p.b * a.blocks_d) * 64 * V + p.lane * V;
    p.live = p.d < a.D;
    p.dc = (uint32_t)(p.live ? p.d : a.D - V);
    int len = a.len ? a.len[p.b] : a.T;
    len = __builtin_amdgcn_readfirstlane(len);
    p.len = len < 0 ? 0 : len > a.T ? a.T : len;
    p.t0 = segment * a.seg_len;
    p.t1 = a.T - p.t0 < a.seg_len ? a.T : p.t0 + a.seg_len;
    return true;
}

// steps of the chunk at t that belong to the sequence
__device__ __forceinline__ int valid_steps(int len, int t)
{
    const int n = len - t;
    return n < 0 ? 0 : n > C ? C : n;
}

__device__ __forceinline__ uint8_t load_done(const RecurArgs &a, int b, int t, int lane)
{
    if (!a.done || lane >= C) return 0;
    const int tt = t + lane < a.T ? t + lane : a.T - 1;
    return a.done[(int64_t)tt * a.B + b];
}

__device__ __forceinline__ uint32_t done_bits(uint8_t flag, int nv)
{
    return (uint32_t)__ballot(flag != 0) & ((1u << nv) - 1u);
}

__device__ __forceinline__ char *row_at(const RecurRows &m, int b, int t)
{
    return (char *)m.p + (m.st * t + m.sb * b);
}

// rows t .. t + C - 1 of sequence b, the last one of all again past T
template <bool BF, int V, bool ONCE = false>
__device__ __forceinline__ void load_chunk(const RecurRows &m, int b, int t, int T, uint32_t d,
                                           Raw<BF, V> *raw)
{
    const char *row = row_at(m, b, t < T ? t : T - 1);
#pragma unroll
    for (int k = 0; k < C; ++k) {
        raw[k] = load_row<BF, V, ONCE>(row, d);
        row += t + k + 1 < T ? m.st : 0;
    }
}

// A map h -> P h + H with an episode's end in it forgets whatever h is, NaN and
// infinity too.  That has a mark of its own, a negative P: a product of decays
// reaches 0 without one, and then a NaN has to stay, as it does step by step.
// So that an infinity stays as well, P does not fall to 0.
constexpr float FORGETS = -1.0f, LEAST = 0x1p-149f;

// P of a chunk's map; ends: one of its steps ends an episode
__device__ __forceinline__ float map_p(float P, bool ends) { return ends ? FORGETS : fmaxf(P, LEAST); }

// the map m after the state c
__device__ __forceinline__ float join(float2 m, float c)
{
    return m.x < 0.0f ? m.y : fmaf(m.x, c, m.y);
}

// and after the map P.  (A NaN among the decays is in H too, and stays there.)
__device__ __forceinline__ float join_p(float2 m, float P)
{
    return map_p(m.x * P, m.x < 0.0f || P < 0.0f);
}

// the shapes that split a sequence over workgroups: calls of few waves
template <int V, int W> constexpr bool SEGMENTS = V == 1 && W == 4;

// The maps of `n` segments after the states c, from segment `first` on, forward
// or (BACK) backward.  Each wave reduces a share of them, sixteen loads in
// flight; the shares go through LDS.
template <int V, int W, bool BACK>
__device__ __forceinline__ void join_segments(const float2 *maps, int64_t BD, int first, int n,
                                              float2 (*lds)[64 * V], int w, int lane,
                                              float (&c)[V])
{
    if (n <= 0) return;
    const int per = (n + W - 1) / W, a0 = w * per, a1 = a0 + per < n ? a0 + per : n;
    float P[V], H[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        P[e] = 1.0f;
        H[e] = 0.0f;
    }
#pragma unroll 1
    for (int k = a0; k < a1; k += 16) {
        float2 m[16][V];
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int at = k + q < a1 ? k + q : a1 - 1;
            const float2 *from = maps + (int64_t)(BACK ? first - at : first + at) * BD;
#pragma unroll
            for (int e = 0; e < V; ++e) m[q][e] = from[e];
        }
#pragma unroll
        for (int q = 0; q < 16; ++q)
            if (k + q < a1) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    H[e] = join(m[q][e], H[e]);
                    P[e] = join_p(m[q][e], P[e]);
                }
            }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) lds[w][lane * V + e] = make_float2(P[e], H[e]);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) c[e] = join(lds[j][lane * V + e], c[e]);
}

// ---------------------------------------------------------------------------
// forward: states (SUMMARY = false), or a segment's map alone
// ---------------------------------------------------------------------------
template <bool BF, int V, int W, bool SUMMARY, bool ONCE>
__global__ __launch_bounds__(64 * W * GROUP<W>) void recur_fwd_kernel(RecurArgs a)
{
    __shared__ float2 maps[W == 1 ? 1 : 2][W][W == 1 ? 1 : 64 * V];
    Place<V, W> p;
    if (!place<V, W>(a, blockIdx.y, p)) return;
    float s[V], s2[V], carry[V], carryP[V];
    const int64_t bd = (int64_t)p.b * a.D + p.dc, BD = (int64_t)a.B * a.D;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        s[e] = RATE * softplus(a.lam[p.dc + e]);
        s2[e] = s[e] * LOG2E;
        const bool copied = SEGMENTS<V, W> && gridDim.y > 1;
        carry[e] = SUMMARY ? 0.0f
                   : copied ? a.maps[(gridDim.y - 1) * BD + bd + e].y
                   : a.h0   ? a.h0[bd + e]
                            : 0.0f;
        carryP[e] = 1.0f;
    }
    if constexpr (!SUMMARY && SEGMENTS<V, W>)
        join_segments<V, W, false>(a.maps + bd, BD, 0, (int)blockIdx.y, maps[1], p.w, p.lane, carry);

    Raw<BF, V> x[C], r[C], i[C];
    auto fetch = [&](int t) {
        load_chunk<BF, V, ONCE>(a.x, p.b, t, a.T, p.dc, x);
        load_chunk<BF, V, ONCE>(a.r, p.b, t, a.T, p.dc, r);
        load_chunk<BF, V, ONCE>(a.i, p.b, t, a.T, p.dc, i);
    };
    int t = p.t0 + p.w * C, par = 0;
    fetch(t);
    uint8_t flag = load_done(a, p.b, t, p.lane);
    for (int tile = p.t0; tile < p.t1; tile += W * C, t += W * C) {
        const int nv = valid_steps(p.len, t);
        const uint32_t clear = done_bits(flag, nv);
        const bool plain = nv == C && clear == 0;
        float c[C][V], u[C][V];
#pragma unroll
        for (int k = 0; k < C; ++k) {
            float xs[V], rs[V], is[V];
            unpack<BF, V>(x[k], xs);
            unpack<BF, V>(r[k], rs);
            unpack<BF, V>(i[k], is);
#pragma unroll
            for (int e = 0; e < V; ++e)
                gate<BF>(xs[e], rs[e], is[e], s[e], s2[e], c[k][e], u[k][e]);
        }
        if (tile + W * C < p.t1) {
            fetch(t + W * C);
            flag = load_done(a, p.b, t + W * C, p.lane);
        }
        if (!plain) {
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    c[k][e] = k < nv ? c[k][e] : KEEP_ONE<BF>;
                    u[k][e] = k < nv ? u[k][e] : 0.0f;
                }
        }
        float h[V];
        if constexpr (W > 1) {
            float P[V], H[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                P[e] = 1.0f;
                H[e] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    H[e] = advance<BF>(c[k][e], H[e], u[k][e]);
                    P[e] = fade_p<BF>(c[k][e], P[e]);
                    if (!plain && (clear >> k & 1)) H[e] = 0.0f;
                }
#pragma unroll
            for (int e = 0; e < V; ++e)
                maps[par][p.w][p.lane * V + e] = make_float2(map_p(P[e], clear != 0), H[e]);
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e) h[e] = carry[e];
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (j == p.w) h[e] = carry[e];
                    const float2 m = maps[par][j][p.lane * V + e];
                    carry[e] = join(m, carry[e]);
                    if (SUMMARY) carryP[e] = join_p(m, carryP[e]);
                }
            par ^= 1;
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) h[e] = carry[e];
        }
        if constexpr (!SUMMARY) {
            if (a.saved && p.live && t < a.T)
                store_states<V, ONCE>(a.saved + (int64_t)(t / C) * BD + (int64_t)p.b * a.D, p.dc, h);
            char *out = row_at(a.y, p.b, t);
            const bool stored = p.live && a.y.p;
#pragma unroll
            for (int k = 0; k < C; ++k) {
                float y[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    h[e] = advance<BF>(c[k][e], h[e], u[k][e]);
                    y[e] = plain || k < nv ? h[e] : 0.0f;
                    if (!plain && (clear >> k & 1)) h[e] = 0.0f;
                }
                if (stored && t + k < a.T) store_row<BF, V, ONCE>(out + k * a.y.st, p.dc, y);
            }
            if constexpr (W == 1) {
#pragma unroll
                for (int e = 0; e < V; ++e) carry[e] = h[e];
            }
        }
    }
    if (!p.live || p.w != 0) return;
    if constexpr (SUMMARY) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            a.maps[blockIdx.y * BD + bd + e] = make_float2(carryP[e], carry[e]);
            // Segments read the first states while the last one stores the last
            // states, which may be the same buffer: they read a copy, kept where
            // the last segment would have its map, which nobody needs.
            if (blockIdx.y == 0)
                a.maps[gridDim.y * BD + bd + e] = make_float2(0.0f, a.h0 ? a.h0[bd + e] : 0.0f);
        }
    } else if (p.t1 == a.T && a.h_last) {
        store_f32<V>(a.h_last + bd, carry);
    }
}

// ---------------------------------------------------------------------------
// backward: g_t = dy_t + G_t, G_{t-1} = a_t g_t (0 across an episode's end),
// from the last step to the first.  The forward pass left the state before
// every chunk, so a chunk's coefficients need no other chunk.
// ---------------------------------------------------------------------------
template <bool BF, int V, int W, bool ONCE>
__global__ __launch_bounds__(64 * W * GROUP<W>) void recur_bwd_kernel(RecurArgs a)
{
    __shared__ float2 maps[W == 1 ? 1 : 2][W][W == 1 ? 1 : 64 * V];
    Place<V, W> p;
    if (!place<V, W>(a, blockIdx.y, p)) return;
    float s[V], s2[V], carry[V], sum[V];
    const int64_t bd = (int64_t)p.b * a.D + p.dc, BD = (int64_t)a.B * a.D;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        s[e] = RATE * softplus(a.lam[p.dc + e]);
        s2[e] = s[e] * LOG2E;
        const bool copied = SEGMENTS<V, W> && gridDim.y > 1;
        carry[e] = copied ? a.maps[bd + e].y : a.dh_last ? a.dh_last[bd + e] : 0.0f;
        sum[e] = 0.0f;
    }
    if constexpr (SEGMENTS<V, W>)
        join_segments<V, W, true>(a.maps + bd, BD, (int)gridDim.y - 1,
                                  (int)(gridDim.y - 1 - blockIdx.y), maps[1], p.w, p.lane, carry);
    const int tiles = (p.t1 - p.t0 + W * C - 1) / (W * C);
    int t = p.t0 + (tiles - 1) * W * C + p.w * C, par = 0;

    Raw<BF, V> x[C], r[C], i[C], dy[C];
    float hs[V];
    auto fetch = [&](int tc) {
        load_chunk<BF, V, ONCE>(a.x, p.b, tc, a.T, p.dc, x);
        load_chunk<BF, V, ONCE>(a.r, p.b, tc, a.T, p.dc, r);
        load_chunk<BF, V, ONCE>(a.i, p.b, tc, a.T, p.dc, i);
        load_chunk<BF, V, ONCE>(a.dy, p.b, tc, a.T, p.dc, dy);
        const int tt = tc < a.T ? tc : a.T - 1;
        load_states<V, ONCE>(a.saved + (int64_t)(tt / C) * BD + (int64_t)p.b * a.D, p.dc, hs);
    };
    fetch(t);
    uint8_t flag = load_done(a, p.b, t, p.lane);
    for (int n = 0; n < tiles; ++n, t -= W * C) {
        const int nv = valid_steps(p.len, t);
        const uint32_t clear = done_bits(flag, nv);
        const bool plain = nv == C && clear == 0;
        float c[C][V], cx[C][V], ci[C][V], cw[C][V], cr[C][V], g[C][V], h[V];
#pragma unroll
        for (int e = 0; e < V; ++e) h[e] = hs[e];
#pragma unroll
        for (int k = 0; k < C; ++k) {
            float xs[V], rs[V], is[V];
            unpack<BF, V>(x[k], xs);
            unpack<BF, V>(r[k], rs);
            unpack<BF, V>(i[k], is);
            unpack<BF, V>(dy[k], g[k]);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float u;
                gate_grad<BF>(xs[e], rs[e], is[e], s[e], s2[e], h[e], c[k][e], u, cx[k][e],
                              ci[k][e], cw[k][e], cr[k][e]);
                h[e] = advance<BF>(c[k][e], h[e], u);
                if (!plain && (clear >> k & 1)) h[e] = 0.0f;
            }
        }
        if (n + 1 < tiles) {
            fetch(t - W * C);
            flag = load_done(a, p.b, t - W * C, p.lane);
        }
        if (!plain) {
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const bool in = k < nv;
                    c[k][e] = in ? c[k][e] : KEEP_ONE<BF>;
                    cx[k][e] = in ? cx[k][e] : 0.0f;
                    ci[k][e] = in ? ci[k][e] : 0.0f;
                    cw[k][e] = in ? cw[k][e] : 0.0f;
                    cr[k][e] = in ? cr[k][e] : 0.0f;
                    g[k][e] = in ? g[k][e] : 0.0f;
                }
        }
        float G[V];
        if constexpr (W > 1) {
            float P[V], H[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                P[e] = 1.0f;
                H[e] = 0.0f;
            }
#pragma unroll
            for (int k = C - 1; k >= 0; --k)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (!plain && (clear >> k & 1)) H[e] = 0.0f;
                    const float gg = g[k][e] + H[e];
                    H[e] = fade<BF>(c[k][e], gg);
                    P[e] = fade_p<BF>(c[k][e], P[e]);
                }
#pragma unroll
            for (int e = 0; e < V; ++e)
                maps[par][p.w][p.lane * V + e] = make_float2(map_p(P[e], clear != 0), H[e]);
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e) G[e] = carry[e];
#pragma unroll
            for (int j = W - 1; j >= 0; --j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (j == p.w) G[e] = carry[e];
                    const float2 m = maps[par][j][p.lane * V + e];
                    carry[e] = join(m, carry[e]);
                }
            par ^= 1;
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) G[e] = carry[e];
        }
        char *outx = row_at(a.dx, p.b, t), *outr = row_at(a.dr, p.b, t),
             *outi = row_at(a.di, p.b, t);
#pragma unroll
        for (int k = C - 1; k >= 0; --k) {
            float dx[V], dr[V], di[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (!plain && (clear >> k & 1)) G[e] = 0.0f;
                const float gg = g[k][e] + G[e], ww = gg * cw[k][e];
                // past a sequence's end every coefficient is 0, but G may be infinite
                const bool in = plain || k < nv;
                dx[e] = in ? gg * cx[k][e] : 0.0f;
                di[e] = in ? gg * ci[k][e] : 0.0f;
                dr[e] = in ? ww * cr[k][e] : 0.0f;
                sum[e] += in ? ww : 0.0f;
                G[e] = fade<BF>(c[k][e], gg);
            }
            if (p.live && t + k < a.T) {
                store_row<BF, V, ONCE>(outx + k * a.dx.st, p.dc, dx);
                store_row<BF, V, ONCE>(outr + k * a.dr.st, p.dc, dr);
                store_row<BF, V, ONCE>(outi + k * a.di.st, p.dc, di);
            }
        }
        if constexpr (W == 1) {
#pragma unroll
            for (int e = 0; e < V; ++e) carry[e] = G[e];
        }
    }
    // lambda's part of this sequence and segment
    if constexpr (W > 1) {
        float *part = (float *)&maps[0][0][0];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) part[(p.w * 64 + p.lane) * V + e] = sum[e];
        __syncthreads();
        if (p.w != 0) return;
#pragma unroll
        for (int e = 0; e < V; ++e)
            for (int j = 1; j < W; ++j) sum[e] += part[(j * 64 + p.lane) * V + e];
    }
    if (!p.live) return;
    store_f32<V>(a.parts + ((int64_t)blockIdx.y * a.B + p.b) * a.D + p.dc, sum);
    if (p.t0 == 0 && a.dh0) store_f32<V>(a.dh0 + bd, carry);
}

// a segment's map of G alone (a, dy)
template <bool BF, int V, int W>
__global__ __launch_bounds__(64 * W * GROUP<W>) void recur_bwd_map_kernel(RecurArgs a)
{
    __shared__ float2 maps[2][W][64 * V];
    Place<V, W> p;
    const int segment = blockIdx.y + 1;
    if (!place<V, W>(a, segment, p)) return;
    float s[V], s2[V], carry[V], carryP[V];
    const int64_t bd = (int64_t)p.b * a.D + p.dc, BD = (int64_t)a.B * a.D;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        s[e] = RATE * softplus(a.lam[p.dc + e]);
        s2[e] = s[e] * LOG2E;
        carry[e] = 0.0f;
        carryP[e] = 1.0f;
    }
    const int tiles = (p.t1 - p.t0 + W * C - 1) / (W * C);
    int t = p.t0 + (tiles - 1) * W * C + p.w * C, par = 0;
    Raw<BF, V> r[C], dy[C];
    auto fetch = [&](int tc) {
        load_chunk<BF, V>(a.r, p.b, tc, a.T, p.dc, r);
        load_chunk<BF, V>(a.dy, p.b, tc, a.T, p.dc, dy);
    };
    fetch(t);
    uint8_t flag = load_done(a, p.b, t, p.lane);
    for (int n = 0; n < tiles; ++n, t -= W * C) {
        const int nv = valid_steps(p.len, t);
        const uint32_t clear = done_bits(flag, nv);
        float c[C][V], g[C][V], P[V], H[V];
#pragma unroll
        for (int k = 0; k < C; ++k) {
            float rs[V];
            unpack<BF, V>(r[k], rs);
            unpack<BF, V>(dy[k], g[k]);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float rho = __builtin_amdgcn_rcpf(1.0f + exp_neg(rs[e]));
                float am, am1;
                const bool is_near = decay<BF>(-(s[e] * rho), -(s2[e] * rho), am, am1);
                c[k][e] = k < nv ? keep<BF>(is_near, am, am1) : KEEP_ONE<BF>;
                g[k][e] = k < nv ? g[k][e] : 0.0f;
            }
        }
        if (n + 1 < tiles) {
            fetch(t - W * C);
            flag = load_done(a, p.b, t - W * C, p.lane);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            P[e] = 1.0f;
            H[e] = 0.0f;
        }
#pragma unroll
        for (int k = C - 1; k >= 0; --k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (clear >> k & 1) H[e] = 0.0f;
                const float gg = g[k][e] + H[e];
                H[e] = fade<BF>(c[k][e], gg);
                P[e] = fade_p<BF>(c[k][e], P[e]);
            }
#pragma unroll
        for (int e = 0; e < V; ++e)
            maps[par][p.w][p.lane * V + e] = make_float2(map_p(P[e], clear != 0), H[e]);
        __syncthreads();
#pragma unroll
        for (int j = W - 1; j >= 0; --j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float2 m = maps[par][j][p.lane * V + e];
                carry[e] = join(m, carry[e]);
                carryP[e] = join_p(m, carryP[e]);
            }
        par ^= 1;
    }
    if (!p.live || p.w != 0) return;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        a.maps[segment * BD + bd + e] = make_float2(carryP[e], carry[e]);
        // (a copy, as of the first states forward: dh0 may be its buffer)
        if (segment == 1) a.maps[bd + e] = make_float2(0.0f, a.dh_last ? a.dh_last[bd + e] : 0.0f);
    }
}

// dlambda_d = sigmoid(lambda) / softplus(lambda) * sum over rows of parts,
// in 64 bits, 64 row groups of 16 channels, joined in a fixed order.
__global__ __launch_bounds__(1024) void recur_lambda_kernel(const float *parts, int64_t rows, int D,
                                                            const float *lam, float *dlam)
{
    __shared__ double red[64][17];
    const int c = threadIdx.x & 15, rg = threadIdx.x >> 4, d = blockIdx.x * 16 + c;
    double s = 0.0;
    if (d < D) {
        // (sixteen loads in flight: 4,096 rows of 512 33 us one at a time, 11 so)
        int64_t k = rg;
        for (; k + 15 * 64 < rows; k += 16 * 64) {
            float v[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) v[q] = parts[(k + q * 64) * D + d];
#pragma unroll
            for (int q = 0; q < 16; ++q) s += (double)v[q];
        }
        for (; k < rows; k += 64) s += (double)parts[k * D + d];
    }
    red[rg][c] = s;
    __syncthreads();
    if (rg != 0 || d >= D) return;
    s = 0.0;
    for (int k = 0; k < 64; ++k) s += red[k][c];
    const double l = (double)lam[d];
    // sigmoid / softplus -> 1 as lambda falls: exp(l) (1 - exp(l)/2) of both
    const double e = exp(-fabs(l)), sp = (l > 0.0 ? l : 0.0) + log1p(e);
    const double sg = l > 0.0 ? 1.0 / (1.0 + e) : e / (1.0 + e);
    dlam[d] = (float)(s * (l < -700.0 ? 1.0 : sg / sp));
}

// ---------------------------------------------------------------------------
// one step: a wave has 64 V channels of `rows` sequences, so that lambda's
// softplus, some hundred instructions, is taken once for all of them
// ---------------------------------------------------------------------------
template <bool BF, int V, bool ONCE>
__global__ __launch_bounds__(256) void recur_step_kernel(RecurArgs a, int rows)
{
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = blockIdx.x * 4 + wv;
    if (unit >= a.units) return;
    const int set = unit / a.blocks_d, b0 = set * rows;
    const int d = (unit - set * a.blocks_d) * 64 * V + (threadIdx.x & 63) * V;
    if (d >= a.D) return;
    const int b1 = a.B - b0 < rows ? a.B : b0 + rows;
    float s[V], s2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        s[e] = RATE * softplus(a.lam[d + e]);
        s2[e] = s[e] * LOG2E;
    }
    typedef float state __attribute__((ext_vector_type(V)));
    for (int b = b0; b < b1; ++b) {
        float x[V], r[V], i[V], h[V];
        unpack<BF, V>(load_row<BF, V, ONCE>(row_at(a.x, b, 0), d), x);
        unpack<BF, V>(load_row<BF, V, ONCE>(row_at(a.r, b, 0), d), r);
        unpack<BF, V>(load_row<BF, V, ONCE>(row_at(a.i, b, 0), d), i);
        const state was = load_at<state, ONCE>(a.h0 + (int64_t)b * a.D, d * 4u);
        const bool clear = a.done && a.done[b] != 0;
        state now;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float c, u;
            gate<BF>(x[e], r[e], i[e], s[e], s2[e], c, u);
            h[e] = advance<BF>(c, was[e], u);
            now[e] = clear ? 0.0f : h[e];
        }
        if (a.y.p) store_row<BF, V, ONCE>(row_at(a.y, b, 0), d, h);
        store_at<ONCE>(a.h_last + (int64_t)b * a.D, d * 4u, now);
    }
}

bool rows_allow(const RecurRows &m, int V, int es)
{
    return !m.p || (((uintptr_t)m.p | m.st | m.sb) % (V * es) == 0);
}

bool allows(const RecurArgs &a, int V)
{
    const int es = a.bf16 ? 2 : 4;
    if (a.D % V) return false;
    for (const RecurRows *m : {&a.x, &a.r, &a.i, &a.y, &a.dy, &a.dx, &a.dr, &a.di})
        if (!rows_allow(*m, V, es)) return false;
    return true;
}

struct Shape {
    int V, W, S, seg_len, blocks_d;
    int64_t units;
};

// Two channels a lane, waves of a workgroup along time (W), segments (S), by
// how many waves a call has.  Measured (bf16, us, T x B x D; forward):
//   390 x 4,096 x 512 (32,768 units of one wave)   W = 1       1,320
//   390 x 64 x 512    (512)     W = 1, 4, 16: 73, 34, 43;  W = 4, S = 2: 46
//   2,520 x 16 x 256  (64)      W = 4, S = 1, 4, 16, 64: 135, 69, 44, 43; W = 16: 99
//   24,570 x 1 x 512  (8)       W = 4, S = 16, 64, 128, 256: 151, 61, 53, 54
//   256 x 64 x 64     (64)      W = 16: 14;  W = 4, S = 8: 14 in two launches
// A wave's step takes about 60 instructions of four cycles, so few waves on few
// CUs are slower than reading everything twice on all of them.
Shape shape_of(int T, int B, int D, bool wide)
{
    Shape s;
    auto units = [&](int V) { return (int64_t)B * ((D + 64 * V - 1) / (64 * V)); };
    s.V = wide && D > 64 && units(2) >= 1024 ? 2 : 1;
    s.units = units(s.V);
    s.blocks_d = (D + 64 * s.V - 1) / (64 * s.V);
    if (s.units >= 2048 || T <= C) s.W = 1;
    else if (s.units >= 512 || T <= 4 * C || T > 2 * 16 * C) s.W = 4;
    else s.W = 16;
    s.S = 1;
    const int tile = s.W * C;
    const int64_t tiles = ((int64_t)T + tile - 1) / tile, waves = s.units * s.W;
    if (s.W == 4 && waves < 1024 && tiles > 1) {
        int64_t want = 4096 / waves;
        if (want > 256) want = 256;
        if (want > tiles) want = tiles;
        const int64_t per = (tiles + want - 1) / want;
        s.S = (int)((tiles + per - 1) / per);
    }
    s.seg_len = (int)((tiles + s.S - 1) / s.S) * tile;
    return s;
}

template <bool BF, int V, int W, bool ONCE = false>
void start(RecurArgs &a, const Shape &sh, bool backward, hipStream_t s)
{
    const dim3 grid((unsigned)((sh.units + GROUP<W> - 1) / GROUP<W>), (unsigned)sh.S);
    const int threads = 64 * W * GROUP<W>;
    if constexpr (SEGMENTS<V, W>) {
        if (sh.S > 1 && !backward)          // (nobody needs the last segment's map,
            hipLaunchKernelGGL((recur_fwd_kernel<BF, V, W, true, false>), dim3(grid.x, grid.y - 1),
                               dim3(threads), 0, s, a);
        if (sh.S > 1 && backward)           // or, backward, the first one's)
            hipLaunchKernelGGL((recur_bwd_map_kernel<BF, V, W>), dim3(grid.x, grid.y - 1),
                               dim3(threads), 0, s, a);
    }
    if (backward)
        hipLaunchKernelGGL((recur_bwd_kernel<BF, V, W, ONCE>), grid, dim3(threads), 0, s, a);
    else
        hipLaunchKernelGGL((recur_fwd_kernel<BF, V, W, false, ONCE>), grid, dim3(threads), 0, s, a);
}

// Arrays of which the last-level cache (256 MB) holds only a part are read and
// written past the caches: 252 x 1,024 x 256 fp32 forward 209 -> 187 us, backward
// 378 -> 350; a step of 65,536 x 512 156 -> 141, but one of 65,536 x 64, which
// the cache holds, 18 -> 23.
bool once(double bytes) { return bytes > 256e6; }

template <bool BF>
void start_shape(RecurArgs &a, const Shape &sh, bool backward, hipStream_t s)
{
    // (two channels a lane are for many units: never 16 waves of them)
    const bool cold = once((double)a.T * a.B * a.D * (BF ? 2 : 4) * (backward ? 7 : 4));
    if (sh.V == 2 && sh.W == 1) cold ? start<BF, 2, 1, true>(a, sh, backward, s) : start<BF, 2, 1>(a, sh, backward, s);
    else if (sh.V == 2) start<BF, 2, 4>(a, sh, backward, s);
    else if (sh.W == 1) start<BF, 1, 1>(a, sh, backward, s);
    else if (sh.W == 4) start<BF, 1, 4>(a, sh, backward, s);
    else start<BF, 1, 16>(a, sh, backward, s);
}

}  // namespace

// maps of the segments, then (backward) the parts of lambda's gradient; for
// either width of the lanes
size_t recur_workspace_bytes(int T, int B, int D)
{
    size_t most = 256;
    for (bool wide : {false, true}) {
        const Shape s = shape_of(T, B, D, wide);
        const size_t bd = (size_t)B * D;
        const size_t n = (s.S > 1 ? s.S * bd * sizeof(float2) : 0) + s.S * bd * sizeof(float);
        most = n > most ? n : most;
    }
    return (most + 255) / 256 * 256;
}

bool recur_fits(int T, int B, int D)
{
    // step numbers past the last chunk and a row's bytes in 32 bits; workgroups
    // of 256 threads in a 32-bit grid
    return T <= 1 << 30 && D <= 1 << 24 && (int64_t)B * ((D + 63) / 64) <= (int64_t)1 << 25;
}

hipError_t launch_recur(RecurArgs &a, bool backward, hipStream_t s)
{
    const Shape sh = shape_of(a.T, a.B, a.D, allows(a, 2));
    a.units = (int)sh.units;
    a.blocks_d = sh.blocks_d;
    a.seg_len = sh.seg_len;
    const size_t bd = (size_t)a.B * a.D;
    a.maps = (float2 *)a.work;
    a.parts = (float *)((char *)a.work + (sh.S > 1 ? sh.S * bd * sizeof(float2) : 0));
    if (a.bf16) start_shape<true>(a, sh, backward, s);
    else start_shape<false>(a, sh, backward, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !backward) return e;
    hipLaunchKernelGGL(recur_lambda_kernel, dim3((a.D + 15) / 16), dim3(1024), 0, s, a.parts,
                       (int64_t)sh.S * a.B, a.D, a.lam, a.dlam);
    return hipGetLastError();
}

hipError_t launch_recur_step(RecurArgs &a, hipStream_t s)
{
    // four channels a lane where that leaves a wave's lanes full; the states too
    // have to be aligned to a lane's
    const auto fits = [&](int V) {
        return allows(a, V) && ((uintptr_t)a.h0 | (uintptr_t)a.h_last) % (4 * V) == 0;
    };
    const int V = a.D >= 256 && fits(4) ? 4 : a.D >= 128 && fits(2) ? 2 : 1;
    a.blocks_d = (a.D + 64 * V - 1) / (64 * V);
    // sequences a wave: as many as leave 16 waves a CU, at most 16
    const int64_t all = (int64_t)a.B * a.blocks_d;
    const int rows = (int)(all < 8192 ? 1 : all > 16 * 4096 ? 16 : all / 4096);
    a.units = (a.B + rows - 1) / rows * a.blocks_d;
    const bool cold = once((double)a.B * a.D * (4 * (a.bf16 ? 2 : 4) + 8));
    void (*kernel)(RecurArgs, int) =
        a.bf16 ? (V == 4 ? (cold ? recur_step_kernel<true, 4, true> : recur_step_kernel<true, 4, false>)
                  : V == 2 ? recur_step_kernel<true, 2, false> : recur_step_kernel<true, 1, false>)
               : (V == 4 ? (cold ? recur_step_kernel<false, 4, true> : recur_step_kernel<false, 4, false>)
                  : V == 2 ? recur_step_kernel<false, 2, false> : recur_step_kernel<false, 1, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((a.units + 3) / 4)), dim3(256), 0, s, a, rows);
    return hipGetLastError();
}

}  // namespace tpk
