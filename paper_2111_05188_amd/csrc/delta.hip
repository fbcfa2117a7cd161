// Gated delta rule: whole sequences forward, and one step (delta.hpp has the
// formulas).
//
// Forward, a workgroup has one head of one sequence; wave w has columns 16w.. of
// its state, all rows of them, in registers.  Groups of steps go through LDS:
// the next group's loads are under way while one is worked on.  Each wave first
// prepares one piece of the group (its triangles, which do not need the state),
// then all waves run the pieces on their columns.
#include "delta.hpp"

namespace tpk {
namespace {

// a sequence's gates of a group of steps
__device__ __forceinline__ float delta_gate(const DeltaRows &m, const char *base, int64_t t, bool bf)
{
    const char *p = base + t * m.st;
    return bf ? (float)*(const __bf16 *)p : *(const float *)p;
}

// one piece on the state's columns of this wave
template <bool BF, int D, int LD, bool MASK, class E>
__device__ __forceinline__ void run_piece(const E *q, const E *k, E *v, int s, int count, bool ends,
                                          const PieceRows &rows, const typename Tile<BF>::val &Tt,
                                          const typename Tile<BF>::val &Pt, int w, int lane, floatx4 *S)
{
    constexpr int KT = D / 16;
    const int r = 4 * (lane >> 4);
    floatx4 ks = {}, qs = {};
#pragma unroll
    for (int kt = 0; kt < KT; kt += 2) {
        const auto x0 = Tile<BF>::split(S[kt]), x1 = Tile<BF>::split(S[kt + 1]);
        ks = Tile<BF>::mm2(along_row<BF, LD>(k, s, kt, lane), along_row<BF, LD>(k, s, kt + 1, lane), x0, x1, ks);
        qs = Tile<BF>::mm2(along_row<BF, LD>(q, s, kt, lane), along_row<BF, LD>(q, s, kt + 1, lane), x0, x1, qs);
    }
    const floatx4 vv = Tile<BF>::wide(along_col<BF, LD, MASK>(v, s, count, w, lane));
    const floatx4 be = *(const floatx4 *)(rows.beta + r), ak = *(const floatx4 *)(rows.ak + r);
    const floatx4 aq = *(const floatx4 *)(rows.aq + r), au = *(const floatx4 *)(rows.au + r);
    floatx4 R, U = {}, o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        R[i] = !MASK || r + i < count ? be[i] * vv[i] - ak[i] * ks[i] : 0.0f;
        o[i] = aq[i] * qs[i];
    }
    U = Tile<BF>::mm(Tt, Tile<BF>::split(R), U);
    o = Tile<BF>::mm(Pt, Tile<BF>::split(U), o);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!MASK || r + i < count) v[(s + r + i) * LD + 16 * w + (lane & 15)] = (E)o[i];
    if (ends) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) S[kt] = floatx4{};
        return;
    }
    floatx4 W;
#pragma unroll
    for (int i = 0; i < 4; ++i) W[i] = !MASK || r + i < count ? U[i] * au[i] : 0.0f;
    const auto x = Tile<BF>::split(W);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
        S[kt] = Tile<BF>::mm(along_col<BF, LD, MASK>(k, s, count, kt, lane), x, S[kt] * rows.total);
}

template <bool BF, int D>
__global__ __launch_bounds__(4 * D, D == 128 ? 2 : 3) void delta_fwd_kernel(DeltaArgs a)
{
    constexpr int G = DELTA_GROUP, NP = G / 16, KT = D / 16;
    typedef Rows<BF, D, G> RW;
    typedef typename RW::E E;
    typedef typename Tile<BF>::val val;
    constexpr int LD = RW::LD;
    __shared__ __attribute__((aligned(16))) E buf[(3 * G + 16) * LD];
    __shared__ val sT[NP][64], sP[NP][64];
    __shared__ __attribute__((aligned(16))) PieceRows rows[NP];
    __shared__ double cum[NP][16];
    __shared__ float sg[G], sbeta[G];
    __shared__ int sodd[2];
    E *q = buf, *k = q + G * LD, *v = k + G * LD;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / a.H, h = blockIdx.x - b * a.H;
    const int n = lane & 15, r4 = 4 * (lane >> 4);
    int len = a.len ? a.len[b] : a.T;
    len = len < 0 ? 0 : len > a.T ? a.T : len;
    const float rate = -8.0f * delta_softplus(a.lam[h]);
    auto base = [&](const DeltaRows &m) { return (char *)m.p + b * m.sb + h * m.sh; };
    const char *pq = base(a.q), *pk = base(a.k), *pv = base(a.v), *pr = base(a.r), *pb = base(a.b);

    const int64_t st = ((int64_t)b * a.H + h) * a.dk * a.dv;
    const int col = 16 * w + n;
    floatx4 S[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 16 * kt + r4 + i;
            S[kt][i] = a.h0 && row < a.dk && col < a.dv ? a.h0[st + (int64_t)row * a.dv + col] : 0.0f;
        }

    Part fq[RW::N], fk[RW::N], fv[RW::N];
    float fr = 0.0f, fb = 0.0f;
    uint8_t fd = 0;
    auto fetch = [&](int t0) {
        const int count = len - t0 < G ? len - t0 : G;
        RW::fetch(a.q, pq, t0, count, a.dk, fq);
        RW::fetch(a.k, pk, t0, count, a.dk, fk);
        RW::fetch(a.v, pv, t0, count, a.dv, fv);
        if ((int)threadIdx.x < count) {
            fr = delta_gate(a.r, pr, t0 + threadIdx.x, BF);
            fb = delta_gate(a.b, pb, t0 + threadIdx.x, BF);
        }
        fd = a.done && lane < count ? a.done[(int64_t)(t0 + lane) * a.B + b] : 0;
    };
    fetch(0);
    if (threadIdx.x < 2) sodd[threadIdx.x] = 0;
    workgroup_lds_barrier();
    for (int t0 = 0, turn = 0; t0 < a.T; t0 += G, turn ^= 1) {
        const int count = len - t0 < G ? len - t0 : G, all = a.T - t0 < G ? a.T - t0 : G;
        if (count > 0) {
            RW::put(q, fq);
            RW::put(k, fk);
            RW::put(v, fv);
            bool odd = RW::odd(fq) || RW::odd(fk) || RW::odd(fv);
            if ((int)threadIdx.x < count) {
                const float g = rate * delta_sigmoid(fr), be = delta_sigmoid(fb);
                sg[threadIdx.x] = g < -3e38f ? -3e38f : g;
                sbeta[threadIdx.x] = be;
                odd = odd || !(fabsf(fr) < 3e38f) || !(fabsf(fb) < 3e38f);
            }
            const uint64_t ends = __ballot(lane < count && fd != 0);
            if (odd) sodd[turn] = 1;
            if (a.saved) {
                float *to = a.saved + (((int64_t)(t0 / G) * a.B + b) * a.H + h) * D * D + col;
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) to[(16 * kt + r4 + i) * D] = S[kt][i];
            }
            workgroup_lds_barrier();
            if (t0 + G < len) fetch(t0 + G);
            const bool single = __builtin_amdgcn_readfirstlane(sodd[turn]) != 0;
            if (threadIdx.x == 0) sodd[turn ^ 1] = 0;
            for (int s = 0; s < count;) {
                int from = s, to = s;
                for (int p = 0; p <= w && from < count; ++p) {
                    to = piece_end(from, count, ends, single);
                    if (p < w) from = to;
                }
                if (w < NP && from < count) {
                    floatx4 Tt, Tn, Pt, Pn;
                    piece_triangles<BF, D, LD, false>(q, k, sg, sbeta, from, to - from, lane, cum[w], &rows[w], Tt,
                                                      Tn, Pt, Pn);
                    sT[w][lane] = Tile<BF>::split(Tt);
                    sP[w][lane] = Tile<BF>::split(Pt);
                }
                workgroup_lds_barrier();
#pragma unroll 1
                for (int p = 0; p < NP && s < count; ++p) {
                    const int e = piece_end(s, count, ends, single);
                    const bool done = ends >> (e - 1) & 1;
                    if (e - s == 16)
                        run_piece<BF, D, LD, false>(q, k, v, s, 16, done, rows[p], sT[p][lane], sP[p][lane], w,
                                                    lane, S);
                    else
                        run_piece<BF, D, LD, true>(q, k, v, s, e - s, done, rows[p], sT[p][lane], sP[p][lane], w,
                                                   lane, S);
                    s = e;
                }
                workgroup_lds_barrier();
            }
        }
        if (a.y.p) RW::store(a.y, base(a.y), t0, count > 0 ? count : 0, all, a.dv, v);
    }
    if (a.h_last) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * kt + r4 + i;
                if (row < a.dk && col < a.dv) a.h_last[st + (int64_t)row * a.dv + col] = S[kt][i];
            }
    }
}

// One step: a workgroup has one head of one sequence, its state in registers
// between the one read and the one write.  y = e^g S^T q^ + (k^.q^) u, so both
// products are of the state as it came.
template <bool BF, int D, bool VEC>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaArgs a)
{
    typedef typename Tile<BF>::elem E;
    constexpr int CX = D / 4, RY = 256 / CX, NR = D / RY;   // lanes of a row, rows at a time
    __shared__ float sq[D], sk[D], red[2][4][D];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int b = blockIdx.x / a.H, h = blockIdx.x - b * a.H;
    const int c0 = tid % CX * 4, r0 = tid / CX;
    const int64_t st = ((int64_t)b * a.H + h) * a.dk * a.dv;
    floatx4 S[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j) {
        const int row = r0 + j * RY;
        S[j] = floatx4{};
        if (row < a.dk && c0 < a.dv) {
            const float *p = a.h0 + st + (int64_t)row * a.dv + c0;
            if constexpr (VEC) {
                S[j] = *(const floatx4 *)p;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (c0 + i < a.dv) S[j][i] = p[i];
            }
        }
    }
    auto base = [&](const DeltaRows &m) { return (char *)m.p + b * m.sb + h * m.sh; };
    // every wave takes the rows' lengths by itself; wave 0 leaves them for all
    const E *pq = (const E *)base(a.q), *pk = (const E *)base(a.k), *pv = (const E *)base(a.v);
    float x[(D + 63) / 64], y[(D + 63) / 64];
    float qq = 0.0f, kk = 0.0f, qk = 0.0f;
#pragma unroll
    for (int j = 0; j < (D + 63) / 64; ++j) {
        const int c = lane + 64 * j;
        x[j] = c < a.dk ? (float)pq[c] : 0.0f;
        y[j] = c < a.dk ? (float)pk[c] : 0.0f;
        qq += x[j] * x[j];
        kk += y[j] * y[j];
        qk += x[j] * y[j];
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) {
        qq += __shfl_xor(qq, m);
        kk += __shfl_xor(kk, m);
        qk += __shfl_xor(qk, m);
    }
    const float rq = rsqrtf(qq + 1e-6f), rk = rsqrtf(kk + 1e-6f);
    if (w == 0) {
#pragma unroll
        for (int j = 0; j < (D + 63) / 64; ++j) {
            const int c = lane + 64 * j;
            if (c < D) {
                sq[c] = x[j] * rq;
                sk[c] = y[j] * rk;
            }
        }
    }
    const float alpha = delta_exp(-8.0f * delta_softplus(a.lam[h]) *
                                  delta_sigmoid(delta_gate(a.r, base(a.r), 0, BF)));
    const float beta = delta_sigmoid(delta_gate(a.b, base(a.b), 0, BF));
    __syncthreads();
    floatx4 ks = {}, qs = {};
#pragma unroll
    for (int j = 0; j < NR; ++j) {
        const int row = r0 + j * RY;
        ks += S[j] * sk[row];
        qs += S[j] * sq[row];
    }
#pragma unroll
    for (int m = 32; m >= CX; m >>= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ks[i] += __shfl_xor(ks[i], m);
            qs[i] += __shfl_xor(qs[i], m);
        }
    if (lane < CX) {
        *(floatx4 *)&red[0][w][c0] = ks;
        *(floatx4 *)&red[1][w][c0] = qs;
    }
    __syncthreads();
    floatx4 u, o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float ksum = 0.0f, qsum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            ksum += red[0][j][c0 + i];
            qsum += red[1][j][c0 + i];
        }
        const float v = c0 + i < a.dv ? (float)pv[c0 + i] : 0.0f;
        u[i] = beta * (v - alpha * ksum);
        o[i] = alpha * qsum + u[i] * (qk * rq * rk);
    }
    if (a.y.p && r0 == 0) {
        E *py = (E *)base(a.y);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c0 + i < a.dv) py[c0 + i] = (E)o[i];
    }
    const bool clear = a.done && a.done[b] != 0;
#pragma unroll
    for (int j = 0; j < NR; ++j) {
        const int row = r0 + j * RY;
        const floatx4 s = clear ? floatx4{} : S[j] * alpha + u * sk[row];
        if (row < a.dk && c0 < a.dv) {
            float *p = a.h_last + st + (int64_t)row * a.dv + c0;
            if constexpr (VEC) {
                *(floatx4 *)p = s;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (c0 + i < a.dv) p[i] = s[i];
            }
        }
    }
}

template <bool BF>
void start_forward(DeltaArgs &a, hipStream_t s)
{
    const int D = delta_width(a.dk, a.dv);
    void (*kernel)(DeltaArgs) = D == 32 ? delta_fwd_kernel<BF, 32> : D == 64 ? delta_fwd_kernel<BF, 64>
                                                                             : delta_fwd_kernel<BF, 128>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.B * a.H)), dim3(4 * D), 0, s, a);
}

template <bool BF, bool VEC>
void start_step(DeltaArgs &a, hipStream_t s)
{
    const int D = delta_width(a.dk, a.dv);
    void (*kernel)(DeltaArgs) = D == 32 ? delta_step_kernel<BF, 32, VEC>
                                : D == 64 ? delta_step_kernel<BF, 64, VEC> : delta_step_kernel<BF, 128, VEC>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.B * a.H)), dim3(256), 0, s, a);
}

}  // namespace

bool delta_fits(int T, int B, int H)
{
    // steps past the last group and the heads of all sequences in 32 bits
    return T <= 1 << 30 && (int64_t)B * H <= (int64_t)1 << 23;
}

size_t delta_saved_bytes(int T, int B, int H, int dk, int dv)
{
    const size_t D = delta_width(dk, dv);
    return (size_t)((T + DELTA_GROUP - 1) / DELTA_GROUP) * B * H * D * D * sizeof(float);
}

size_t delta_workspace_bytes(int, int B, int H, int, int)
{
    return ((size_t)B * H * sizeof(double) + 255) / 256 * 256;
}

hipError_t launch_delta_forward(DeltaArgs &a, hipStream_t s)
{
    if (a.bf16) start_forward<true>(a, s);
    else start_forward<false>(a, s);
    return hipGetLastError();
}

hipError_t launch_delta_step(DeltaArgs &a, hipStream_t s)
{
    const bool vec = a.dv % 4 == 0 && ((uintptr_t)a.h0 | (uintptr_t)a.h_last) % 16 == 0;
    if (a.bf16) vec ? start_step<true, true>(a, s) : start_step<true, false>(a, s);
    else vec ? start_step<false, true>(a, s) : start_step<false, false>(a, s);
    return hipGetLastError();
}

}  // namespace tpk
