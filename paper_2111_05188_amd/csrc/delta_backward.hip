// Gradients of the gated delta rule (delta.hpp has the forward formulas).  For a
// piece with state S0 before it, G1 the gradient of the state after it, and dY:
//   dU = P^T dY + (gamma_C/gamma) K^ G1,   dR = T^T dU,   dV = beta dR,
//   G0 = gamma_C G1 + (gamma Q^)^T dY - (beta gamma K^)^T dR,
//   M = (dY U^T) o G (lower),  E = -(dR U^T) o beta G (below the diagonal),
//   dQ^ = gamma dY S0^T + M K^,
//   dK^ = -beta gamma dR S0^T + (gamma_C/gamma) U G1^T + M^T Q^ + (E + E^T) K^.
// The pre-activation of beta gets (dR.u)(1 - beta).  The log-decay of a step
// multiplies what every later step of its episode reads, so its gradient is the
// sum of x_c = q^_c.dq^_c + k^_c.dk^_c - 2 dR_c.u_c over the steps from it to the
// episode's end, and <G, S> at the end of the group if the episode goes on: the
// terms of P, L and the states that a decay does not touch cancel in x.
//
// A workgroup has one head of one sequence and goes through its groups from the
// last to the first, each from the state kept before it.  Products over the
// values' columns sum over what different waves hold, so every wave carries two
// strips of the state and of its gradient: columns 16w.. of S and G, and columns
// 16w.. of their transposes, for which the same rows of K, Q, U and dR change
// places in the products.  Nothing is transposed and no state goes through LDS.
#include "delta.hpp"

namespace tpk {
namespace {

__device__ __forceinline__ float gate_at(const DeltaRows &m, const char *base, int64_t t, bool bf)
{
    const char *p = base + t * m.st;
    return bf ? (float)*(const TP_GLOBAL __bf16 *)p : *(const TP_GLOBAL float *)p;
}

// Sum over the 16 lanes of a row group, in all of them.
__device__ __forceinline__ float row_sum(float x)
{
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) x += __shfl_xor(x, m);
    return x;
}

// fp32 rows [G][LD] in LDS as operands: three planes of bf16, or one of fp32.
template <bool BF, int G, int LD>
struct Values {
    typedef typename Tile<BF>::elem E;
    static constexpr int COUNT = (BF ? 3 : 1) * G * LD;     // elements

    static __device__ __forceinline__ void put(E *lds, int row, int col, typename Tile<BF>::val x, int i)
    {
        if constexpr (BF) {
            lds[row * LD + col] = x.hi[i];
            lds[(G + row) * LD + col] = x.mid[i];
            lds[(2 * G + row) * LD + col] = x.lo[i];
        } else {
            lds[row * LD + col] = x[i];
        }
    }
    static __device__ __forceinline__ typename Tile<BF>::val rows(const E *lds, int s, int kt, int lane)
    {
        if constexpr (BF) {
            typename Tile<BF>::val x;
            x.hi = along_row<BF, LD>(lds, s, kt, lane);
            x.mid = along_row<BF, LD>(lds + G * LD, s, kt, lane);
            x.lo = along_row<BF, LD>(lds + 2 * G * LD, s, kt, lane);
            return x;
        } else {
            return along_row<BF, LD>(lds, s, kt, lane);
        }
    }
    template <bool MASK>
    static __device__ __forceinline__ typename Tile<BF>::val cols(const E *lds, int s, int count, int ct, int lane)
    {
        if constexpr (BF) {
            typename Tile<BF>::val x;
            x.hi = along_col<BF, LD, MASK>(lds, s, count, ct, lane);
            x.mid = along_col<BF, LD, MASK>(lds + G * LD, s, count, ct, lane);
            x.lo = along_col<BF, LD, MASK>(lds + 2 * G * LD, s, count, ct, lane);
            return x;
        } else {
            return along_col<BF, LD, MASK>(lds, s, count, ct, lane);
        }
    }
};

template <bool BF, int D>
struct Back {
    static constexpr int G = DELTA_GROUP, NP = G / 16, KT = D / 16;
    typedef Rows<BF, D, G> RW;
    typedef typename RW::E E;
    typedef Tile<BF> TL;
    typedef typename TL::val val;
    static constexpr int LD = RW::LD;
    typedef Values<BF, G, LD> VL;
    // rows read past a piece's end stay inside: what follows each array here
    struct Shared {
        __attribute__((aligned(16))) E q[G * LD], k[G * LD], v[G * LD], dy[G * LD];
        __attribute__((aligned(16))) E U[VL::COUNT], dR[VL::COUNT], pad[16 * LD];
        __attribute__((aligned(16))) val m[NP][3][64];      // T, T^T, P; then the products with K, Q, K
        __attribute__((aligned(16))) PieceRows rows[NP];
        double cum[NP][16];
        float g[G], beta[G], shut[G], idle[G];              // 1 - sigmoid(r), 1 - beta
        float x[G], dbeta[G];
        float dots[RW::NW][G][2];                           // q^.dq^, k^.dk^ of a strip
        float ends[RW::NW];                                 // <G, S> of a strip
        int odd[2];
    };

    // the writes U of a piece, and the state after it, on columns 16w..
    template <bool MASK>
    static __device__ __forceinline__ void forward(Shared &sh, int s, int count, bool ends, int p, int w, int lane,
                                                   floatx4 *S)
    {
        const int r = 4 * (lane >> 4);
        const PieceRows &rows = sh.rows[p];
        floatx4 ks = {}, U = {}, R, W;
#pragma unroll
        for (int kt = 0; kt < KT; kt += 2)
            ks = TL::mm2(along_row<BF, LD>(sh.k, s, kt, lane), along_row<BF, LD>(sh.k, s, kt + 1, lane),
                         TL::split(S[kt]), TL::split(S[kt + 1]), ks);
        const floatx4 vv = TL::wide(along_col<BF, LD, MASK>(sh.v, s, count, w, lane));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            R[i] = !MASK || r + i < count ? rows.beta[r + i] * vv[i] - rows.ak[r + i] * ks[i] : 0.0f;
        U = TL::mm(sh.m[p][1][lane], TL::split(R), U);
        const val u = TL::split(U);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (!MASK || r + i < count) VL::put(sh.U, s + r + i, 16 * w + (lane & 15), u, i);
#pragma unroll
        for (int i = 0; i < 4; ++i) W[i] = !MASK || r + i < count ? U[i] * rows.au[r + i] : 0.0f;
        const val x = TL::split(W);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            S[kt] = TL::mm(along_col<BF, LD, MASK>(sh.k, s, count, kt, lane), x, S[kt] * rows.total);
            if (ends) S[kt] = floatx4{};
        }
    }

    // the transposed state after a piece, on columns 16w.. (keys)
    template <bool MASK>
    static __device__ __forceinline__ void forward_turned(Shared &sh, int s, int count, bool ends, int p, int w,
                                                          int lane, floatx4 *ST)
    {
        const int r = 4 * (lane >> 4);
        const PieceRows &rows = sh.rows[p];
        const floatx4 kc = TL::wide(along_col<BF, LD, MASK>(sh.k, s, count, w, lane));
        floatx4 W;
#pragma unroll
        for (int i = 0; i < 4; ++i) W[i] = kc[i] * rows.au[r + i];
        const val x = TL::split(W);
#pragma unroll
        for (int vt = 0; vt < KT; ++vt) {
            ST[vt] = TL::mm(VL::template cols<MASK>(sh.U, s, count, vt, lane), x, ST[vt] * rows.total);
            if (ends) ST[vt] = floatx4{};
        }
    }

    // dR and dV of a piece, and the gradient of the state before it
    template <bool MASK>
    static __device__ __forceinline__ void backward(Shared &sh, int s, int count, bool ends, int p, int w, int lane,
                                                    floatx4 *Gs)
    {
        const int r = 4 * (lane >> 4), col = 16 * w + (lane & 15);
        const PieceRows &rows = sh.rows[p];
        floatx4 kg = {}, dR = {};
#pragma unroll
        for (int kt = 0; kt < KT; kt += 2) {
            if (ends) Gs[kt] = Gs[kt + 1] = floatx4{};
            kg = TL::mm2(along_row<BF, LD>(sh.k, s, kt, lane), along_row<BF, LD>(sh.k, s, kt + 1, lane),
                         TL::split(Gs[kt]), TL::split(Gs[kt + 1]), kg);
        }
        const auto dyc = along_col<BF, LD, MASK>(sh.dy, s, count, w, lane);
        floatx4 dU;
#pragma unroll
        for (int i = 0; i < 4; ++i) dU[i] = !MASK || r + i < count ? kg[i] * rows.au[r + i] : 0.0f;
        dU = TL::mm(sh.m[p][2][lane], dyc, dU);
        dR = TL::mm(sh.m[p][0][lane], TL::split(dU), dR);
        const val x = TL::split(dR);
        const floatx4 dyw = TL::wide(dyc);
        floatx4 A, B;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            A[i] = dyw[i] * rows.aq[r + i];
            B[i] = !MASK || r + i < count ? -(dR[i] * rows.ak[r + i]) : 0.0f;
            if (!MASK || r + i < count) {
                VL::put(sh.dR, s + r + i, col, x, i);
                sh.v[(s + r + i) * LD + col] = (E)(rows.beta[r + i] * dR[i]);
            }
        }
        const val a = TL::split(A), b = TL::split(B);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            Gs[kt] = TL::mm(along_col<BF, LD, MASK>(sh.q, s, count, kt, lane), a, Gs[kt] * rows.total);
            Gs[kt] = TL::mm(along_col<BF, LD, MASK>(sh.k, s, count, kt, lane), b, Gs[kt]);
        }
    }

    // the gradients of a piece's triangles, as first operands (one wave)
    static __device__ __forceinline__ void triangles(Shared &sh, int s, int count, int p, int lane)
    {
        const int n = lane & 15, r = 4 * (lane >> 4);
        const PieceRows &rows = sh.rows[p];
        floatx4 yu = {}, uy = {}, ru = {}, ur = {};
#pragma unroll
        for (int vt = 0; vt < KT; vt += 2) {
            const auto y = along_row<BF, LD>(sh.dy, s, vt, lane), y1 = along_row<BF, LD>(sh.dy, s, vt + 1, lane);
            const val u = VL::rows(sh.U, s, vt, lane), d = VL::rows(sh.dR, s, vt, lane);
            const val u1 = VL::rows(sh.U, s, vt + 1, lane), d1 = VL::rows(sh.dR, s, vt + 1, lane);
            yu = TL::mm2(y, y1, u, u1, yu);
            uy = TL::mm2(u, u1, y, y1, uy);
            ru = TL::mm2(d, d1, u, u1, ru);
            ur = TL::mm2(u, u1, d, d1, ur);
        }
        floatx4 down, up, mq, mk, mm;
        piece_decays(sh.cum[p], count, lane, down, up);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool below = r + i >= n && r + i < count, above = r + i <= n && n < count;
            mq[i] = above ? uy[i] * up[i] * rows.rk[r + i] : 0.0f;
            mk[i] = below ? yu[i] * down[i] * rows.rq[r + i] : 0.0f;
            mm[i] = r + i == n ? 0.0f
                    : below ? -(ru[i] * down[i] * rows.beta[r + i] * rows.rk[r + i])
                    : above ? -(ur[i] * up[i] * rows.beta[n] * rows.rk[r + i]) : 0.0f;
            if (r + i == n && n < count) sh.dbeta[s + n] = ru[i];
        }
        sh.m[p][0][lane] = TL::split(mq);
        sh.m[p][1][lane] = TL::split(mk);
        sh.m[p][2][lane] = TL::split(mm);
    }

    // dQ^ and dK^ as far as they read the state before a piece
    template <bool MASK>
    static __device__ __forceinline__ void early(Shared &sh, int s, int p, int lane, const floatx4 *ST, floatx4 &dq,
                                                 floatx4 &dk)
    {
        const int r = 4 * (lane >> 4);
        const PieceRows &rows = sh.rows[p];
        floatx4 a = {}, b = {};
#pragma unroll
        for (int vt = 0; vt < KT; vt += 2) {
            const val x = TL::split(ST[vt]), x1 = TL::split(ST[vt + 1]);
            a = TL::mm2(along_row<BF, LD>(sh.dy, s, vt, lane), along_row<BF, LD>(sh.dy, s, vt + 1, lane), x, x1, a);
            b = TL::mm(VL::rows(sh.dR, s, vt, lane), x, b);
            b = TL::mm(VL::rows(sh.dR, s, vt + 1, lane), x1, b);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            dq[i] = a[i] * rows.fade[r + i];
            dk[i] = -(b[i] * rows.beta[r + i] * rows.fade[r + i]);
        }
    }

    // the rest of them, and the transposed gradient of the state before the piece
    template <bool MASK>
    static __device__ __forceinline__ void late(Shared &sh, int s, int count, bool ends, int p, int w, int lane,
                                                floatx4 *GT, floatx4 &dq, floatx4 &dk)
    {
        const int r = 4 * (lane >> 4);
        const PieceRows &rows = sh.rows[p];
        const auto qc = along_col<BF, LD, MASK>(sh.q, s, count, w, lane);
        const auto kc = along_col<BF, LD, MASK>(sh.k, s, count, w, lane);
        const floatx4 qw = TL::wide(qc), kw = TL::wide(kc);
        floatx4 c = {}, A, B;
#pragma unroll
        for (int vt = 0; vt < KT; ++vt) {
            if (ends) GT[vt] = floatx4{};
            c = TL::mm(VL::rows(sh.U, s, vt, lane), TL::split(GT[vt]), c);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            dk[i] += c[i] * rows.rest[r + i];
            A[i] = qw[i] * rows.aq[r + i];
            B[i] = -(kw[i] * rows.ak[r + i]);
        }
        dq = TL::mm(sh.m[p][0][lane], kc, dq);
        dk = TL::mm(sh.m[p][1][lane], qc, dk);
        dk = TL::mm(sh.m[p][2][lane], kc, dk);
        const val a = TL::split(A), b = TL::split(B);
#pragma unroll
        for (int vt = 0; vt < KT; ++vt) {
            GT[vt] = TL::mm(along_col<BF, LD, MASK>(sh.dy, s, count, vt, lane), a, GT[vt] * rows.total);
            GT[vt] = TL::mm(VL::template cols<MASK>(sh.dR, s, count, vt, lane), b, GT[vt]);
        }
        // what the unit rows' gradients need: their products with the rows
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = row_sum(dq[i] * qw[i] * rows.rq[r + i]);
            const float y = row_sum(dk[i] * kw[i] * rows.rk[r + i]);
            if ((lane & 15) == 0 && (!MASK || r + i < count)) {
                sh.dots[w][s + r + i][0] = x;
                sh.dots[w][s + r + i][1] = y;
            }
        }
    }

    // x rq (dq^ - q^ (q^.dq^)) in place of q, and the same of k
    template <bool MASK>
    static __device__ __forceinline__ void finish(Shared &sh, int s, int count, int p, int w, int lane, floatx4 dq,
                                                  floatx4 dk)
    {
        const int r = 4 * (lane >> 4), col = 16 * w + (lane & 15);
        const PieceRows &rows = sh.rows[p];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (MASK && r + i >= count) continue;
            float x = 0.0f, y = 0.0f;
#pragma unroll
            for (int j = 0; j < RW::NW; ++j) {
                x += sh.dots[j][s + r + i][0];
                y += sh.dots[j][s + r + i][1];
            }
            E *q = sh.q + (s + r + i) * LD + col, *k = sh.k + (s + r + i) * LD + col;
            const float rq = rows.rq[r + i], rk = rows.rk[r + i];
            *q = (E)(rq * (dq[i] - (float)*q * rq * x));
            *k = (E)(rk * (dk[i] - (float)*k * rk * y));
            if (w == 0 && (lane & 15) == 0) sh.x[s + r + i] = x + y - 2.0f * sh.dbeta[s + r + i];
        }
    }
};

template <bool BF, int D>
__global__ __launch_bounds__(4 * D, 2) void delta_bwd_kernel(DeltaArgs a)
{
    typedef Back<BF, D> BK;
    typedef typename BK::RW RW;
    constexpr int G = BK::G, NP = BK::NP, KT = BK::KT, LD = BK::LD;
    __shared__ typename BK::Shared sh;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / a.H, h = blockIdx.x - b * a.H;
    const int n = lane & 15, r4 = 4 * (lane >> 4), col = 16 * w + n;
    int len = a.len ? a.len[b] : a.T;
    len = len < 0 ? 0 : len > a.T ? a.T : len;
    const float rate = -8.0f * delta_softplus(a.lam[h]);
    auto base = [&](const DeltaRows &m) { return (char *)m.p + b * m.sb + h * m.sh; };
    const int64_t st = ((int64_t)b * a.H + h) * a.dk * a.dv;

    floatx4 S[KT], ST[KT], Gs[KT], GT[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 16 * kt + r4 + i;
            Gs[kt][i] = a.dh_last && row < a.dk && col < a.dv ? a.dh_last[st + (int64_t)row * a.dv + col] : 0.0f;
            GT[kt][i] = a.dh_last && row < a.dv && col < a.dk ? a.dh_last[st + (int64_t)col * a.dv + row] : 0.0f;
        }
    if (threadIdx.x < 2) sh.odd[threadIdx.x] = 0;
    double lam = 0.0;

    const int last = (a.T - 1) / G;
    for (int grp = last, turn = 0; grp >= 0; --grp, turn ^= 1) {
        const int t0 = grp * G;
        const int count = len - t0 < G ? len - t0 : G, all = a.T - t0 < G ? a.T - t0 : G;
        if (count > 0) {
            Part fq[RW::N], fk[RW::N], fv[RW::N], fy[RW::N];
            RW::fetch(a.q, RW::at(a.q, b, h, t0), count, a.dk, fq);
            RW::fetch(a.k, RW::at(a.k, b, h, t0), count, a.dk, fk);
            RW::fetch(a.v, RW::at(a.v, b, h, t0), count, a.dv, fv);
            RW::fetch(a.dy, RW::at(a.dy, b, h, t0), count, a.dv, fy);
            const uint8_t fd = a.done && lane < count ? a.done[(int64_t)(t0 + lane) * a.B + b] : 0;
            const float *kept = a.saved + (((int64_t)grp * a.B + b) * a.H + h) * D * D;
            auto load_state = [&] {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) S[kt][i] = kept[(16 * kt + r4 + i) * D + col];
                    ST[kt] = *(const floatx4 *)(kept + col * D + 16 * kt + r4);
                }
            };
            load_state();
            float odd = RW::odd(fq) + RW::odd(fk) + RW::odd(fv) + RW::odd(fy);
            workgroup_lds_barrier();                // (the group before is done with)
            if ((int)threadIdx.x < count) {
                const float fr = gate_at(a.r, base(a.r), t0 + threadIdx.x, BF);
                const float fb = gate_at(a.b, base(a.b), t0 + threadIdx.x, BF);
                const float g = rate * delta_sigmoid(fr);
                sh.g[threadIdx.x] = g < -3e38f ? -3e38f : g;
                sh.beta[threadIdx.x] = delta_sigmoid(fb);
                sh.shut[threadIdx.x] = delta_sigmoid(-fr);
                sh.idle[threadIdx.x] = delta_sigmoid(-fb);
                odd += (fr + fb) * 0.0f;
            }
            RW::put(sh.q, fq);
            RW::put(sh.k, fk);
            RW::put(sh.v, fv);
            RW::put(sh.dy, fy);
            if (odd != odd) sh.odd[turn] = 1;
            const uint64_t ends = __ballot(lane < count && fd != 0);
            workgroup_lds_barrier();
            const bool single = __builtin_amdgcn_readfirstlane(sh.odd[turn]) != 0;
            if (threadIdx.x == 0) sh.odd[turn ^ 1] = 0;

            auto run = [&](int c, auto f) {
                if (c == 16) f(std::integral_constant<bool, false>{});
                else f(std::integral_constant<bool, true>{});
            };
            // NP pieces from step s on: where the p-th starts
            auto piece = [&](int s, int p) {
                while (p-- > 0 && s < count) s = piece_end(s, count, ends, single);
                return s;
            };
            auto prepare = [&](int s) {
                if (w >= NP) return;
                const int from = piece(s, w), to = from < count ? piece_end(from, count, ends, single) : from;
                if (to == from) return;
                floatx4 Tt, Tn, Pt, Pn;
                piece_triangles<BF, D, LD, true>(sh.q, sh.k, sh.g, sh.beta, from, to - from, lane, sh.cum[w],
                                                 &sh.rows[w], Tt, Tn, Pt, Pn);
                sh.m[w][0][lane] = Tile<BF>::split(Tn);
                sh.m[w][1][lane] = Tile<BF>::split(Tt);
                sh.m[w][2][lane] = Tile<BF>::split(Pn);
            };
            int batches = 0;
            for (int s = 0; s < count; s = piece(s, NP)) ++batches;
            for (int batch = batches - 1; batch >= 0; --batch) {
                // the state before this batch: from the kept one, over the batches before
                // (more than one where episodes end)
                if (batch != batches - 1) load_state();
                int s = 0;
                for (int j = 0; j < batch; ++j) {
                    prepare(s);
                    workgroup_lds_barrier();
                    for (int p = 0, x = s; p < NP && x < count; ++p) {
                        const int e = piece_end(x, count, ends, single);
                        const bool done = ends >> (e - 1) & 1;
                        BK::template forward<true>(sh, x, e - x, done, p, w, lane, S);
                        x = e;
                    }
                    workgroup_lds_barrier();
                    for (int p = 0, x = s; p < NP && x < count; ++p) {
                        const int e = piece_end(x, count, ends, single);
                        const bool done = ends >> (e - 1) & 1;
                        BK::template forward_turned<true>(sh, x, e - x, done, p, w, lane, ST);
                        x = e;
                    }
                    workgroup_lds_barrier();
                    s = piece(s, NP);
                }
                int at[NP + 1];
                at[0] = s;
#pragma unroll
                for (int p = 0; p < NP; ++p)
                    at[p + 1] = at[p] < count ? piece_end(at[p], count, ends, single) : at[p];
                prepare(s);
                workgroup_lds_barrier();
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const int c = at[p + 1] - at[p];
                    if (c == 0) continue;
                    const bool done = ends >> (at[p + 1] - 1) & 1;
                    run(c, [&](auto m) {
                        BK::template forward<decltype(m)::value>(sh, at[p], c, done, p, w, lane, S);
                    });
                }
                if (batch == batches - 1) {
                    float x = 0.0f;
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x += S[kt][i] * Gs[kt][i];
                    // (an episode that ends here leaves nothing to the next group)
                    if (ends >> (count - 1) & 1) x = 0.0f;
                    x = row_sum(x);
                    x += __shfl_xor(x, 16);
                    x += __shfl_xor(x, 32);
                    if (lane == 0) sh.ends[w] = x;
                }
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) {
                    const int c = at[p + 1] - at[p];
                    if (c == 0) continue;
                    const bool done = ends >> (at[p + 1] - 1) & 1;
                    run(c, [&](auto m) {
                        BK::template backward<decltype(m)::value>(sh, at[p], c, done, p, w, lane, Gs);
                    });
                }
                workgroup_lds_barrier();
                if (w < NP) {
                    const int from = piece(s, w), to = from < count ? piece_end(from, count, ends, single) : from;
                    if (to > from) BK::triangles(sh, from, to - from, w, lane);
                }
                workgroup_lds_barrier();
                floatx4 dq[NP], dk[NP];
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const int c = at[p + 1] - at[p];
                    if (c == 0) continue;
                    const bool done = ends >> (at[p + 1] - 1) & 1;
                    run(c, [&](auto m) {
                        BK::template early<decltype(m)::value>(sh, at[p], p, lane, ST, dq[p], dk[p]);
                        if (p + 1 < NP)
                            BK::template forward_turned<decltype(m)::value>(sh, at[p], c, done, p, w, lane, ST);
                    });
                }
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) {
                    const int c = at[p + 1] - at[p];
                    if (c == 0) continue;
                    const bool done = ends >> (at[p + 1] - 1) & 1;
                    run(c, [&](auto m) {
                        BK::template late<decltype(m)::value>(sh, at[p], c, done, p, w, lane, GT, dq[p], dk[p]);
                    });
                }
                workgroup_lds_barrier();
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const int c = at[p + 1] - at[p];
                    if (c == 0) continue;
                    run(c, [&](auto m) {
                        BK::template finish<decltype(m)::value>(sh, at[p], c, p, w, lane, dq[p], dk[p]);
                    });
                }
                workgroup_lds_barrier();
            }
            // gates: lane t of the first wave has step t
            if (w == 0) {
                float acc = 0.0f, on = 0.0f;
#pragma unroll
                for (int j = 0; j < RW::NW; ++j) on += sh.ends[j];
                // the last step of this step's episode within the group
                const uint64_t m = lane < count ? ends >> lane : 0;
                const int end = m ? lane + __builtin_ctzll(m) : count - 1;
                for (int c = 0; c < count; ++c) acc += c >= lane && c <= end ? sh.x[c] : 0.0f;
                if (lane < count) {
                    if (!m) acc += on;
                    // the first step of an episode has no state to fade
                    if (lane > 0 && (ends >> (lane - 1) & 1)) acc = 0.0f;
                    const float wg = acc * sh.g[lane];
                    lam += (double)wg;
                    sh.x[lane] = wg * sh.shut[lane];
                    sh.dbeta[lane] = sh.dbeta[lane] * sh.idle[lane];
                }
            }
            wave_lds_fence();
        }
        const int done_rows = count > 0 ? count : 0;
        RW::store(a.dq, RW::at(a.dq, b, h, t0), done_rows, all, a.dk, sh.q);
        RW::store(a.dkey, RW::at(a.dkey, b, h, t0), done_rows, all, a.dk, sh.k);
        RW::store(a.dval, RW::at(a.dval, b, h, t0), done_rows, all, a.dv, sh.v);
        if (w == 0 && lane < all) {
            const float x = lane < done_rows ? sh.x[lane] : 0.0f, y = lane < done_rows ? sh.dbeta[lane] : 0.0f;
            char *pr = base(a.dr) + (t0 + lane) * a.dr.st, *pb = base(a.db) + (t0 + lane) * a.db.st;
            if constexpr (BF) {
                *(__bf16 *)pr = (__bf16)x;
                *(__bf16 *)pb = (__bf16)y;
            } else {
                *(float *)pr = x;
                *(float *)pb = y;
            }
        }
    }
    if (w == 0) {
        lam = wave_sum(lam);
        if (lane == 0) a.parts[blockIdx.x] = lam;
    }
    if (a.dh0) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * kt + r4 + i;
                if (row < a.dk && col < a.dv) a.dh0[st + (int64_t)row * a.dv + col] = Gs[kt][i];
            }
    }
}

// dlambda_h = sigmoid(lambda) / softplus(lambda) * sum over sequences of parts, in
// a fixed order.
__global__ __launch_bounds__(256) void delta_lambda_kernel(const double *parts, int B, int H, const float *lam,
                                                           float *dlam)
{
    __shared__ double red[4];
    const int h = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    double s = 0.0;
    for (int b = threadIdx.x; b < B; b += 256) s += parts[(int64_t)b * H + h];
    s = wave_sum(s);
    if (lane == 0) red[w] = s;
    __syncthreads();
    if (threadIdx.x != 0) return;
    s = red[0] + red[1] + red[2] + red[3];
    const double l = (double)lam[h];
    // sigmoid / softplus -> 1 as lambda falls: exp(l) (1 - exp(l)/2) of both
    const double e = exp(-fabs(l)), sp = (l > 0.0 ? l : 0.0) + log1p(e);
    const double sg = l > 0.0 ? 1.0 / (1.0 + e) : e / (1.0 + e);
    dlam[h] = (float)(s * (l < -700.0 ? 1.0 : sg / sp));
}

template <bool BF>
void start_backward(DeltaArgs &a, hipStream_t s)
{
    const int D = delta_width(a.dk, a.dv);
    void (*kernel)(DeltaArgs) = D == 32 ? delta_bwd_kernel<BF, 32> : D == 64 ? delta_bwd_kernel<BF, 64>
                                                                             : delta_bwd_kernel<BF, 128>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.B * a.H)), dim3(4 * D), 0, s, a);
}

}  // namespace

hipError_t launch_delta_backward(DeltaArgs &a, hipStream_t s)
{
    a.parts = (double *)a.work;
    if (a.bf16) start_backward<true>(a, s);
    else start_backward<false>(a, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(delta_lambda_kernel, dim3(a.H), dim3(256), 0, s, a.parts, a.B, a.H, a.lam, a.dlam);
    return hipGetLastError();
}

}  // namespace tpk
