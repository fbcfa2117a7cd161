// Gradients of the gated delta rule (delta.hpp has the forward formulas).  For a
// piece with state S0 before it, G1 the gradient of the state after it, and dY:
//   dU = P^T dY + (gamma_C/gamma) K^ G1,   dR = T^T dU,   dV = beta dR,
//   G0 = gamma_C G1 + (gamma Q^)^T dY - (beta gamma K^)^T dR,
//   M = (dY U^T) o G (lower),  E = -(dR U^T) o beta G (below the diagonal),
//   dQ^ = gamma dY S0^T + M K^,
//   dK^ = -beta gamma dR S0^T + (gamma_C/gamma) U G1^T + M^T Q^ + (E + E^T) K^.
// The pre-activation of beta gets (dR.u)(1 - beta).  The log-decay g_t of a step is in
// what passes from before the step to it or after it, and its gradient is all of that:
//   sum over c >= t > j of (dY U^T)[c][j] P[c][j] - (dR U^T)[c][j] L[c][j]
//   + sum over c >= t of gamma_c (S0^T q^_c).dy_c - beta_c gamma_c (S0^T k^_c).dR_c
//   + sum over j < t of (gamma_C/gamma_j) (G1^T k^_j).u_j  +  gamma_C <G1, S0>.
// Every term has the step's decay as a factor, so the sum is as good as the products
// however strong the decay.  (Summing y.dy - v.dv from the step to the episode's end is
// the same but for rounding: terms that the decay does not touch cancel there, and at
// decays of e^-24 a step 5% of lambda's gradient was lost, at e^-40 up to 75%.)
//
// A workgroup has one head of one sequence (a segment of it, where few heads leave
// CUs without work) and goes through its groups from the last to the first, each
// from the state kept before it.  Wave w has columns 16w.. of the state and of its
// gradient in registers, in fp32, and runs the pieces forward for U and back for dR
// on them.  dq^, dk^ and the triangles' gradients sum over all values' columns: each
// wave multiplies its own, with its states transposed in registers (a product with the
// unit matrix), and the parts meet in LDS, at waves that have columns 16w.. of the keys.
// These products run in fp32, for bf16 outputs too: with operands of two bf16 numbers
// (2^-16 of them lost) 0.5% of dq and dk were not the numbers next to the exact ones,
// now 0.04%; with the forward call 4.36 -> 5.00 ms.
// (States and gradients transposed through LDS, and whole sums in each wave, took six
// barriers more: 4.90 ms where this took 4.76.)
//
// 390 steps of 2,048 sequences of 4 heads of 64 in bf16 take 5.20 ms with the forward
// call, where the bytes (3.8 GB) take 0.8 at the rate of a copy.  A group of 32 steps
// is some 46,000 cycles of a workgroup, two of which a CU holds (75 KiB of LDS and 251
// registers each): what bounds it is the chain of products and splits of a wave, with
// the vector units at work 46% of the time and the matrix units 41% (2,600 vector
// instructions and 380 products a wave and group; fp32, 26% and 47%).  Three workgroups
// (51 KiB, 168 registers) spilled: 5.19 ms against 4.74 then.  The fp32 products as three
// bf16 products over 32 of operands of three numbers: 5.22 ms, heads of 128 6.03 against
// 4.93 (390 x 512), more registers and splits.
//
// Where a group has more than NP pieces (episodes that end in it, or a NaN or an infinity,
// which makes each step a piece), each batch of NP starts from the kept state over the ones
// before it: with an end at one step in 16, 390 x 512 x 4 x 64 in bf16 take 2.5 ms with the
// forward call where they take 1.4 without any, at one in 4 6.8, at every step 38.
#include "delta.hpp"

namespace tpk {
namespace {

template <bool BF, int D>
struct Back {
    static constexpr int G = DELTA_GROUP, KT = D / 16;
    // pieces at a time: the transposes of the states before them stay in registers
    static constexpr int NP = D == 128 ? 1 : 2;
    // the waves' parts of dq^ and of dk^ go through LDS one after the other where it does
    // not hold both beside the rows
    static constexpr int TURNS = D == 128 || (!BF && D == 64) ? 2 : 1;
    typedef Rows<BF, D, G> RW;
    typedef typename RW::E E;
    typedef Tile<BF> TL;
    typedef typename TL::val val;
    typedef typename TL::raw raw;
    typedef Tile<false> F;
    static constexpr int LD = RW::LD, NW = RW::NW;
    static constexpr int HALF = KT + 1, TILES = 2 * HALF / TURNS;
    struct Shared {
        // Rows read past a piece's end stay inside, in what follows each array.  Where
        // such rows are summed over (dy, q, k, times zeros) they are inputs again.
        __attribute__((aligned(16))) E dy[G * LD], q[G * LD], k[G * LD], v[G * LD];
        __attribute__((aligned(16))) floatx4 parts[TILES][NW][64];  // of the waves' columns
        __attribute__((aligned(16))) floatx4 m[NP][3][64];  // T, T^T, P^T
        __attribute__((aligned(16))) val P[NP][64];
        __attribute__((aligned(16))) PieceRows rows[NP];
        __attribute__((aligned(16))) floatx4 L[NP][64];
        // y.dy, v.dv, dR.u of the waves' columns; and what of them passes a step's decay
        // from or to a state: gamma S0^T q^.dy, beta gamma S0^T k^.dR, rest G1^T k^.u
        __attribute__((aligned(16))) float sums[G][6][NW];
        double cum[2 * NP][16];
        float g[G], beta[G], shut[G], idle[G];              // 1 - sigmoid(r), 1 - beta
        float dr[G], dbeta[G];
        __attribute__((aligned(16))) float along[NP][2][16];    // q^.dq^, k^.dk^
        float ends[NP][NW];                                 // gamma_C <G1, S0> of a wave's columns
        float decay[G][3];                                  // parts of the gradients of g
        int odd[2];
    };
    static_assert(16 * LD * sizeof(E) <= sizeof(Shared::parts), "rows past v's end");
    static_assert(sizeof(PieceRows) % 16 == 0 && NP * sizeof(PieceRows) <= sizeof(Shared::parts), "T's rows");
    static_assert(sizeof(Shared) <= LDS_LIMIT, "LDS");

    // f(i) for the rows 4g + i that a piece has.  (PART, here and below: a piece of fewer
    // steps than 16; beside one of one step there may be a NaN or an infinity.)
    template <bool PART, class F>
    static __device__ __forceinline__ void each_row(int count, int r, F f)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (!PART || r + i < count) f(i);
    }

    // (a branch: as many selects would run for every piece)
    static __device__ __forceinline__ void clear(floatx4 *S)
    {
        asm volatile("");
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) S[kt] = floatx4{};
    }

    // The writes U of a piece, the state after it, on columns 16w.., and what the state
    // before it takes from R.  OUT: the rows' parts of y.dy too, and the transpose of the
    // state before it.
    struct Writes {
        floatx4 U, S0;
    };
    template <bool PART, bool OUT>
    static __device__ __forceinline__ Writes forward(Shared &sh, int s, int count, bool ends, int p, int w, int lane,
                                                      floatx4 *S, floatx4 *ST)
    {
        lane = fresh(lane);
        const int r = 4 * (lane >> 4);
        const PieceRows &rows = sh.rows[p];
        // all that comes from LDS first: behind a write nothing is read ahead
        raw kr[KT], qr[OUT ? KT : 1], kc[KT], dyc = {};
        floatx4 P = {};
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            kr[kt] = along_row<BF, LD>(sh.k, s, kt, lane);
            if constexpr (OUT) qr[kt] = along_row<BF, LD>(sh.q, s, kt, lane);
        }
        const floatx4 vv = TL::wide(along_col<BF, LD, PART>(sh.v, s, count, w, lane));
        const floatx4 be = *(const floatx4 *)(rows.beta + r), ak = *(const floatx4 *)(rows.ak + r);
        const floatx4 aq = *(const floatx4 *)(rows.aq + r), au = *(const floatx4 *)(rows.au + r);
        const float total = rows.total;
        const floatx4 Tt = sh.m[p][1][lane];
        if constexpr (OUT) {
            P = sh.m[p][2][lane];
            dyc = along_col<BF, LD, PART>(sh.dy, s, count, w, lane);
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) kc[kt] = along_col<BF, LD, PART>(sh.k, s, count, kt, lane);
        const raw eye = TL::eye(lane);
        typename TL::sum2 ks, qs;
        floatx4 R, W, from;
#pragma unroll
        for (int kt = 0; kt < KT; kt += 2) {
            const val x0 = TL::split(S[kt]), x1 = TL::split(S[kt + 1]);
            ks = TL::mm2(kr[kt], kr[kt + 1], x0, x1, ks);
            if constexpr (OUT) {
                qs = TL::mm2(qr[kt], qr[kt + 1], x0, x1, qs);
                ST[kt] = TL::turned(x0, eye);
                ST[kt + 1] = TL::turned(x1, eye);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            from[i] = ak[i] * ks[i];
            R[i] = !PART || r + i < count ? be[i] * vv[i] - from[i] : 0.0f;
        }
        const floatx4 U = F::mm(Tt, R, {}).v;
#pragma unroll
        for (int i = 0; i < 4; ++i) W[i] = !PART || r + i < count ? U[i] * au[i] : 0.0f;
        const val y = TL::split(W);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) S[kt] = TL::mm(kc[kt], y, {S[kt] * total}).v;
        if (ends) clear(S);
        if constexpr (OUT) {
            const floatx4 dy = TL::wide(dyc);
            floatx4 o, t, u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[i] = aq[i] * qs[i];
                u[i] = o[i] * dy[i];
            }
            o = F::mm(P, U, {o}).v;
#pragma unroll
            for (int i = 0; i < 4; ++i) t[i] = o[i] * dy[i];
            const float yd = row_sums(t, lane), qd = row_sums(u, lane);
            if ((lane & 15) < 4 && (!PART || r + (lane & 3) < count)) {
                sh.sums[s + r + (lane & 3)][0][w] = yd;
                sh.sums[s + r + (lane & 3)][3][w] = qd;
            }
        }
        return Writes{U, from};
    }

    // What the waves' columns give to the gradients of a piece's triangles and keys.
    struct Mine {
        floatx4 dy;         // rows of dY, as first operand
        floatx4 U, dR;      // transposed, for either
        floatx4 ak, au;
    };

    // dR and dV of a piece, and the gradient of the state before it; of the one after it
    // the transpose.
    template <bool PART>
    static __device__ __forceinline__ Mine backward(Shared &sh, int s, int count, int p, int w, int lane, floatx4 *Gs,
                                                    const Writes &x, floatx4 *GT)
    {
        const floatx4 U = x.U;
        lane = fresh(lane);
        const int r = 4 * (lane >> 4), col = 16 * w + (lane & 15);
        const PieceRows &rows = sh.rows[p];
        Mine mine;
        raw kr[KT], kc[KT], qc[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) kr[kt] = along_row<BF, LD>(sh.k, s, kt, lane);
        mine.dy = TL::wide(along_row<BF, LD>(sh.dy, s, w, lane));
        const raw dyc = along_col<BF, LD, PART>(sh.dy, s, count, w, lane);
        const floatx4 vw = TL::wide(along_col<BF, LD, PART>(sh.v, s, count, w, lane));
        const floatx4 be = *(const floatx4 *)(rows.beta + r), ak = *(const floatx4 *)(rows.ak + r);
        const floatx4 aq = *(const floatx4 *)(rows.aq + r), au = *(const floatx4 *)(rows.au + r);
        const float total = rows.total;
        const val Pn = sh.P[p][lane];
        const floatx4 Tn = sh.m[p][0][lane];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            qc[kt] = along_col<BF, LD, PART>(sh.q, s, count, kt, lane);
            kc[kt] = along_col<BF, LD, PART>(sh.k, s, count, kt, lane);
        }
        const raw eye = TL::eye(lane);
        typename TL::sum2 kg;
        floatx4 dU, A, B;
#pragma unroll
        for (int kt = 0; kt < KT; kt += 2) {
            const val x0 = TL::split(Gs[kt]), x1 = TL::split(Gs[kt + 1]);
            kg = TL::mm2(kr[kt], kr[kt + 1], x0, x1, kg);
            GT[kt] = TL::turned(x0, eye);
            GT[kt + 1] = TL::turned(x1, eye);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) dU[i] = !PART || r + i < count ? kg[i] * au[i] : 0.0f;
        dU = TL::mm(Pn, dyc, {dU}).v;
        const floatx4 dR = F::mm(Tn, dU, {}).v;
        const floatx4 dyw = TL::wide(dyc);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            A[i] = dyw[i] * aq[i];
            B[i] = !PART || r + i < count ? -(dR[i] * ak[i]) : 0.0f;
        }
        const val a = TL::split(A), b = TL::split(B);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) Gs[kt] = TL::mm(kc[kt], b, TL::mm(qc[kt], a, {Gs[kt] * total})).v;
        floatx4 dv, t, u, f, g;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            dv[i] = be[i] * dR[i];
            t[i] = vw[i] * dv[i];
            u[i] = dR[i] * U[i];
            f[i] = dR[i] * x.S0[i];
            g[i] = U[i] * (kg[i] * au[i]);
        }
        const float vd = row_sums(t, lane), ru = row_sums(u, lane);
        const float rs = row_sums(f, lane), ug = row_sums(g, lane);
        const floatx4 one = TL::wide(eye);
        mine.U = F::turned(U, one);
        mine.dR = F::turned(dR, one);
        mine.ak = ak;
        mine.au = au;
        each_row<PART>(count, r, [&](int i) {
            sh.v[(s + r + i) * LD + col] = (E)dv[i];
        });
        if ((lane & 15) < 4 && (!PART || r + (lane & 3) < count)) {
            sh.sums[s + r + (lane & 3)][1][w] = vd;
            sh.sums[s + r + (lane & 3)][2][w] = ru;
            sh.sums[s + r + (lane & 3)][4][w] = rs;
            sh.sums[s + r + (lane & 3)][5][w] = ug;
        }
        return mine;
    }

    // A wave's part of dY S0^T for all keys, and of P's gradient (turn 0), or of
    // rest rk U G1^T - beta gamma rk dR S0^T, and of L's (turn 1).
    static __device__ __forceinline__ void give(Shared &sh, int p, int turn, int w, int lane, const Mine &m,
                                                const floatx4 *ST, const floatx4 *GT)
    {
        lane = fresh(lane);
        const int first = TURNS == 1 ? turn * HALF : 0;
        float e = 0.0f;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            floatx4 x;
            if (turn == 0) {
                x = F::mm(m.dy, ST[kt], {}).v;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) e += ST[kt][i] * GT[kt][i];
                x = F::mm(m.U, GT[kt], {}).v;
                const floatx4 y = F::mm(m.dR, ST[kt], {}).v;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = m.au[i] * x[i] - m.ak[i] * y[i];
            }
            sh.parts[first + kt][w][lane] = x;
        }
        if (turn == 1) {
            e = lanes_sum<64>(e);
            if (lane == 0) sh.ends[p][w] = e * sh.rows[p].total;
        }
        sh.parts[first + KT][w][lane] = F::mm(turn == 0 ? m.dy : m.dR, m.U, {}).v;
    }

    // the sum of all waves' parts of a tile
    static __device__ __forceinline__ floatx4 take(const Shared &sh, int tile, int lane)
    {
        floatx4 x = sh.parts[tile][0][lane];
#pragma unroll
        for (int j = 1; j < NW; ++j) x += sh.parts[tile][j][lane];
        return x;
    }

    // sum of a row's parts of the waves
    static __device__ __forceinline__ float total(const float *parts)
    {
        float x = 0.0f;
#pragma unroll
        for (int j = 0; j < NW; ++j) x += parts[j];
        return x;
    }

    // The gradient of a piece's triangle P (turn 0) or L (turn 1), scaled by both rows'
    // lengths, by one wave: as it is and transposed, or, L's, the sum of both.  They take the
    // place of T and P.  And what of it passes each step's decay: the products with the
    // triangle itself, over the rows from the step on and the columns before it.
    template <bool PART>
    static __device__ __forceinline__ void triangle(Shared &sh, int s, int count, int p, int turn, int lane)
    {
        lane = fresh(lane);
        const int n = lane & 15, r = 4 * (lane >> 4);
        const PieceRows &rows = sh.rows[p];
        const floatx4 sum = take(sh, TURNS == 1 ? turn * HALF + KT : KT, lane);
        const floatx4 rq = *(const floatx4 *)(rows.rq + r), rk = *(const floatx4 *)(rows.rk + r);
        const floatx4 be = *(const floatx4 *)(rows.beta + r);
        const float rkn = rows.rk[n];
        const floatx4 fade = piece_decays(sh.cum[p], lane);
        const floatx4 own = turn == 0 ? TL::whole(sh.P[p][lane]) : sh.L[p][lane];
        floatx4 x, N, from;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = turn == 0 ? rq[i] : -(be[i] * rk[i]);
            const bool in = turn == 0 ? r + i >= n : r + i > n, has = !PART || r + i < count;
            x[i] = in && has ? sum[i] * (fade[i] * rkn) * f : 0.0f;
            N[i] = r + i > n && has ? sum[i] * own[i] : 0.0f;
            from[i] = r + i >= n ? 1.0f : 0.0f;
        }
        floatx4 C = F::mm(from, N, {}).v;
#pragma unroll
        for (int i = 0; i < 4; ++i) C[i] = r + i > n ? C[i] : 0.0f;
        const float c = row_sums(C, lane);
        if (n < 4 && (!PART || r + n < count)) sh.decay[s + r + n][turn] = turn == 0 ? c : -c;
        const floatx4 t = F::turned(x, F::eye(lane));
        if (turn == 0) {
            sh.m[p][0][lane] = x;
            sh.m[p][1][lane] = t;
        } else {
            sh.m[p][2][lane] = x + t;       // (no place has both)
        }
    }

    // q^.dq^ = y.dy (turn 0) or k^.dk^ = 2 dR.u - v.dv of a piece's rows
    static __device__ __forceinline__ void lengths(Shared &sh, int s, int count, int p, int turn, int lane)
    {
        if (lane >= count) return;
        const float (*x)[NW] = sh.sums[s + lane];
        sh.along[p][turn][lane] = turn == 0 ? total(x[0]) : 2.0f * total(x[2]) - total(x[1]);
    }

    // What passes each step's decay from or to a piece's first and last state.
    static __device__ __forceinline__ void states(Shared &sh, int s, int count, int p, int lane)
    {
        const int n = lane & 15;
        const float (*x)[NW] = sh.sums[s + (n < count ? n : 0)];
        float in = n < count ? total(x[3]) - total(x[4]) : 0.0f;        // of the steps from this one on
        float out = n < count ? total(x[5]) : 0.0f;                     // of the ones before it
        in += dpp<DPP_ROW_SHL + 1>(in);
        in += dpp<DPP_ROW_SHL + 2>(in);
        in += dpp<DPP_ROW_SHL + 4>(in);
        in += dpp<DPP_ROW_SHL + 8>(in);
        out = dpp<DPP_ROW_SHR + 1>(out);
        out += dpp<DPP_ROW_SHR + 1>(out);
        out += dpp<DPP_ROW_SHR + 2>(out);
        out += dpp<DPP_ROW_SHR + 4>(out);
        out += dpp<DPP_ROW_SHR + 8>(out);
        if (lane < count) sh.decay[s + lane][2] = in + out + total(sh.ends[p]);
    }

    // What is summed of a piece on its keys' columns 16w..
    struct Sums {
        floatx4 dq, dk;
    };
    template <bool PART>
    static __device__ __forceinline__ void collect(Shared &sh, int s, int count, int p, int turn, int w, int lane,
                                                   Sums &t)
    {
        lane = fresh(lane);
        (turn == 0 ? t.dq : t.dk) = take(sh, TURNS == 1 ? turn * HALF + w : w, lane);
        if (w == (2 * p + turn) % NW) {
            lengths(sh, s, count, p, turn, lane);
            triangle<PART>(sh, s, count, p, turn, lane);
            if (turn == 1) states(sh, s, count, p, lane);
        }
    }

    // rq (dq^ - q^ (q^.dq^)) in place of q, and the same of k.
    template <bool PART>
    static __device__ __forceinline__ void finish(Shared &sh, int s, int count, int p, int w, int lane,
                                                  const Sums &t)
    {
        lane = fresh(lane);
        const int r = 4 * (lane >> 4), col = 16 * w + (lane & 15);
        const PieceRows &rows = sh.rows[p];
        const raw qc = along_col<BF, LD, PART>(sh.q, s, count, w, lane);
        const raw kc = along_col<BF, LD, PART>(sh.k, s, count, w, lane);
        const floatx4 rq = *(const floatx4 *)(rows.rq + r), rk = *(const floatx4 *)(rows.rk + r);
        const floatx4 aq = *(const floatx4 *)(rows.aq + r);
        const floatx4 m = sh.m[p][0][lane], mt = sh.m[p][1][lane], l = sh.m[p][2][lane];
        const floatx4 yd = *(const floatx4 *)(sh.along[p][0] + r), kd = *(const floatx4 *)(sh.along[p][1] + r);
        floatx4 a, b = t.dk;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = aq[i] * t.dq[i];
        const floatx4 qw = TL::wide(qc), kw = TL::wide(kc);
        b = F::mm(l, kw, F::mm(m, qw, {b})).v;
        a = F::mm(mt, kw, {a}).v;
        each_row<PART>(count, r, [&](int i) {
            sh.q[(s + r + i) * LD + col] = (E)(a[i] - qw[i] * rq[i] * rq[i] * yd[i]);
            sh.k[(s + r + i) * LD + col] = (E)(b[i] - kw[i] * rk[i] * rk[i] * kd[i]);
        });
    }
};

template <class F>
__device__ __forceinline__ void pieces_of(int count, F f)
{
    if (count < 16) f(std::integral_constant<bool, true>{});
    else f(std::integral_constant<bool, false>{});
}

template <bool BF, int D>
__global__ __launch_bounds__(4 * D, 2) void delta_bwd_kernel(DeltaArgs a)
{
    typedef Back<BF, D> BK;
    typedef typename BK::RW RW;
    constexpr int G = BK::G, NP = BK::NP, KT = BK::KT, LD = BK::LD, NW = BK::NW;
    __shared__ typename BK::Shared sh;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / a.H, h = blockIdx.x - b * a.H;
    const int n = lane & 15, r4 = 4 * (lane >> 4), col = 16 * w + n;
    int len = a.len ? a.len[b] : a.T;
    len = len < 0 ? 0 : len > a.T ? a.T : len;
    const int begin = blockIdx.y * a.seg_len, end = a.T - begin < a.seg_len ? a.T : begin + a.seg_len;
    len = len < end ? len : end;
    const float rate = -8.0f * delta_softplus(a.lam[h]);
    const int64_t st = (int64_t)blockIdx.x * a.dk * a.dv;
    const int64_t part = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * D * D;

    floatx4 Gs[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 16 * kt + r4 + i;
            if (a.segments > 1) Gs[kt][i] = a.adds[part + row * D + col];
            else Gs[kt][i] = a.dh_last && row < a.dk && col < a.dv ? a.dh_last[st + (int64_t)row * a.dv + col] : 0.0f;
        }
    if (threadIdx.x < 2) sh.odd[threadIdx.x] = 0;
    double lam = 0.0;

    // a group's rows, gates and kept state; the group before's are under way while one
    // is finished
    const int first = begin / G, last = (end - 1) / G;
    floatx4 S[KT];
    Part fq[RW::N], fk[RW::N], fv[RW::N], fy[RW::N];
    float fr = 0.0f, fb = 0.0f;
    uint8_t fd = 0;
    auto load_state = [&](int grp) {
        const DeltaArgs &a = fresh_args();
        const int lane = fresh(threadIdx.x & 63), r4 = 4 * (lane >> 4), col = 16 * w + (lane & 15);
        const float *from = a.saved + (((int64_t)grp * gridDim.x + blockIdx.x) * D + r4) * D + col;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) S[kt][i] = ((const TP_GLOBAL float *)from)[(16 * kt + i) * D];
    };
    auto fetch = [&](int grp) {
        const DeltaArgs &a = fresh_args();
        const int tid = fresh(threadIdx.x), lane = tid & 63;
        const int t0 = grp * G, count = len - t0 < G ? len - t0 : G;
        RW::fetch(a.q, RW::at(a.q, b, h, t0, tid), count, a.dk, tid, fq);
        RW::fetch(a.k, RW::at(a.k, b, h, t0, tid), count, a.dk, tid, fk);
        RW::fetch(a.v, RW::at(a.v, b, h, t0, tid), count, a.dv, tid, fv);
        RW::fetch(a.dy, RW::at(a.dy, b, h, t0, tid), count, a.dv, tid, fy);
        if (lane < count) {                     // (every wave: each takes some of the gates)
            fr = delta_gate((char *)a.r.p + b * a.r.sb + h * a.r.sh + (t0 + lane) * a.r.st, BF);
            fb = delta_gate((char *)a.b.p + b * a.b.sb + h * a.b.sh + (t0 + lane) * a.b.st, BF);
        }
        fd = a.done && lane < count ? *(const TP_GLOBAL uint8_t *)(a.done + (int64_t)(t0 + lane) * a.B + b) : 0;
        load_state(grp);
    };
    if (len > begin) fetch((len - 1) / G);
    for (int grp = last, turn = 0; grp >= first; --grp, turn ^= 1) {
        const int t0 = grp * G;
        const int count = len - t0 < G ? len - t0 : G, all = end - t0 < G ? end - t0 : G;
        if (count > 0) {
            floatx4 ST[NP][KT], GT[KT];
            typename BK::Writes X[NP];
            float odd = RW::odd(fq) + RW::odd(fk) + RW::odd(fv) + RW::odd(fy);
            workgroup_lds_barrier();                // (the group before is done with)
            const int tid = fresh(threadIdx.x);
            if (lane < count) {
                if (w == 0) {
                    const float g = rate * delta_sigmoid(fr);
                    sh.g[lane] = g < -3e38f ? -3e38f : g;
                }
                if (w == 1) sh.beta[lane] = delta_sigmoid(fb);
                if (w == 2 % NW) sh.shut[lane] = delta_sigmoid(-fr);
                if (w == 3 % NW) sh.idle[lane] = delta_sigmoid(-fb);
                odd += (fr + fb) * 0.0f;
            }
            RW::put(sh.q, fq, tid);
            RW::put(sh.k, fk, tid);
            RW::put(sh.v, fv, tid);
            RW::put(sh.dy, fy, tid);
            if (odd != odd) sh.odd[turn] = 1;
            const uint64_t ends = __ballot(lane < count && fd != 0);
            workgroup_lds_barrier();
            const bool single = __builtin_amdgcn_readfirstlane(sh.odd[turn]) != 0;
            if (threadIdx.x == 0) sh.odd[turn ^ 1] = 0;

            // NP pieces from step s on: where the p-th starts
            auto piece = [&](int s, int p) {
                while (p-- > 0 && s < count) s = piece_end(s, count, ends, single);
                return s;
            };
            // T, then P of each piece, a wave each (T's has its rows where the parts will be)
            auto prepare = [&](int s) {
                for (int j = w; j < 2 * NP; j += NW) {
                    const int p = j % NP, from = piece(s, p);
                    if (from >= count) continue;
                    const int c = piece_end(from, count, ends, single) - from;
                    floatx4 Tt, Tn, Pt, Pn;
                    if (j < NP) {
                        piece_triangles<BF, D, LD, WANT_T | WANT_L, true>(sh.q, sh.k, sh.g, sh.beta, from, c, lane, sh.cum[j],
                                                                 (PieceRows *)sh.parts + p, Tt, Tn, Pt, Pn);
                        sh.m[p][0][lane] = Tn;
                        sh.m[p][1][lane] = Tt;
                        sh.L[p][lane] = Pn;
                    } else {
                        piece_triangles<BF, D, LD, WANT_ROWS | WANT_P | WANT_PT, true>(
                            sh.q, sh.k, sh.g, sh.beta, from, c, lane, sh.cum[j], &sh.rows[p], Tt, Tn, Pt, Pn);
                        sh.P[p][lane] = Tile<BF>::split(Pn);
                        sh.m[p][2][lane] = Pt;
                    }
                }
            };
            int batches = 0;
            for (int s = 0; s < count; s = piece(s, NP)) ++batches;
#pragma unroll 1
            for (int batch = batches - 1; batch >= 0; --batch) {
                const int lane = fresh(threadIdx.x & 63);
                // the state before this batch: from the kept one, over the batches before
                // (more than one where episodes end)
                if (batch != batches - 1) load_state(grp);
                int s = 0;
#pragma unroll 1
                for (int j = 0; j < batch; ++j) {
                    prepare(s);
                    workgroup_lds_barrier();
                    for (int p = 0, x = s; p < NP && x < count; ++p) {
                        const int e = piece_end(x, count, ends, single);
                        BK::template forward<true, false>(sh, x, e - x, ends >> (e - 1) & 1, p, w, lane, S,
                                                         (floatx4 *)nullptr);
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
                auto done = [&](int p) { return (bool)(ends >> (at[p + 1] - 1) & 1); };
                prepare(s);
                workgroup_lds_barrier();
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const int c = at[p + 1] - at[p];
                    if (c == 0) continue;
                    pieces_of(c, [&](auto m) {
                        X[p] = BK::template forward<decltype(m)::value, true>(sh, at[p], c, done(p), p, w, lane, S,
                                                                              ST[p]);
                    });
                }
                typename BK::Sums t[NP];
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) {
                    const int c = at[p + 1] - at[p];
                    if (c == 0) continue;
                    if (done(p)) BK::clear(Gs);
                    typename BK::Mine mine;
                    pieces_of(c, [&](auto m) {
                        mine = BK::template backward<decltype(m)::value>(sh, at[p], c, p, w, lane, Gs, X[p], GT);
                    });
                    // the waves' parts to the waves that have the keys' columns
                    if (p + 1 < NP) workgroup_lds_barrier();
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        BK::give(sh, p, x, w, lane, mine, ST[p], GT);
                        if (x == 0 && BK::TURNS == 1) continue;
                        if (x == 1 && p == 0 && batch == 0 && grp > first) fetch(grp - 1);
                        workgroup_lds_barrier();
                        pieces_of(c, [&](auto m) {
                            if (BK::TURNS == 1) BK::template collect<decltype(m)::value>(sh, at[p], c, p, 0, w, lane, t[p]);
                            BK::template collect<decltype(m)::value>(sh, at[p], c, p, x, w, lane, t[p]);
                        });
                        if (x == 0) workgroup_lds_barrier();
                    }
                }
                workgroup_lds_barrier();
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const int c = at[p + 1] - at[p];
                    if (c == 0) continue;
                    pieces_of(c, [&](auto m) {
                        BK::template finish<decltype(m)::value>(sh, at[p], c, p, w, lane, t[p]);
                    });
                }
                workgroup_lds_barrier();
            }
            // gates: lane t of the first wave has step t
            if (w == 0 && lane < count) {
                const float wg = (sh.decay[lane][0] + sh.decay[lane][1] + sh.decay[lane][2]) * sh.g[lane];
                lam += (double)wg;
                sh.dr[lane] = wg * sh.shut[lane];
                sh.dbeta[lane] = BK::total(sh.sums[lane][2]) * sh.idle[lane];
            }
            wave_lds_fence();
        }
        const DeltaArgs &a = fresh_args();
        const int tid = fresh(threadIdx.x), lane = tid & 63;
        const int some = count > 0 ? count : 0;
        RW::store(a.dq, RW::at(a.dq, b, h, t0, tid), some, all, a.dk, tid, sh.q);
        RW::store(a.dkey, RW::at(a.dkey, b, h, t0, tid), some, all, a.dk, tid, sh.k);
        RW::store(a.dval, RW::at(a.dval, b, h, t0, tid), some, all, a.dv, tid, sh.v);
        if (w == 0 && lane < all) {
            const float x = lane < some ? sh.dr[lane] : 0.0f, y = lane < some ? sh.dbeta[lane] : 0.0f;
            char *pr = (char *)a.dr.p + b * a.dr.sb + h * a.dr.sh + (t0 + lane) * a.dr.st;
            char *pb = (char *)a.db.p + b * a.db.sb + h * a.db.sh + (t0 + lane) * a.db.st;
            if constexpr (BF) {
                *(TP_GLOBAL __bf16 *)pr = (__bf16)x;
                *(TP_GLOBAL __bf16 *)pb = (__bf16)y;
            } else {
                *(TP_GLOBAL float *)pr = x;
                *(TP_GLOBAL float *)pb = y;
            }
        }
    }
    if (w == 0) {
        lam = wave_sum(lam);
        if (lane == 0) a.parts[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = lam;
    }
    if (a.dh0 && begin == 0) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * kt + r4 + i;
                if (row < a.dk && col < a.dv) a.dh0[st + (int64_t)row * a.dv + col] = Gs[kt][i];
            }
    }
}

// What a segment makes of the states' gradient after it: the gradient before it is
// map (gradient after) + add.  One pass back without states: dU, dR and G of the
// formulas, with dY on no gradient (add) and without it on the unit ones (map).
template <bool BF, int D>
__global__ __launch_bounds__(4 * D, 2) void delta_bwd_map_kernel(DeltaArgs a)
{
    constexpr int G = DELTA_GROUP, NP = G / 16, KT = D / 16;
    typedef Rows<BF, D, G> RW;
    typedef Tile<BF> TL;
    typedef typename RW::E E;
    typedef typename TL::val val;
    constexpr int LD = RW::LD;
    __shared__ __attribute__((aligned(16))) E buf[(3 * G + 16) * LD];
    __shared__ floatx4 sT[NP][64];
    __shared__ val sP[NP][64];
    __shared__ __attribute__((aligned(16))) PieceRows rows[NP];
    __shared__ double cum[NP][16];
    __shared__ float sg[G], sbeta[G];
    __shared__ int sodd[2];
    E *q = buf, *k = q + G * LD, *dy = k + G * LD;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / a.H, h = blockIdx.x - b * a.H, segment = blockIdx.y + 1;
    const int n = lane & 15, r4 = 4 * (lane >> 4), col = 16 * w + n;
    int len = a.len ? a.len[b] : a.T;
    len = len < 0 ? 0 : len > a.T ? a.T : len;
    const int begin = segment * a.seg_len, end = a.T - begin < a.seg_len ? a.T : begin + a.seg_len;
    len = len < end ? len : end;
    const float rate = -8.0f * delta_softplus(a.lam[h]);
    floatx4 Gs[KT], M[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            Gs[kt][i] = 0.0f;
            M[kt][i] = 16 * kt + r4 + i == col ? 1.0f : 0.0f;
        }
    if (threadIdx.x < 2) sodd[threadIdx.x] = 0;
    bool cut = false;
    Part fq[RW::N], fk[RW::N], fy[RW::N];
    const int tid = threadIdx.x;
    auto fetch = [&](int t0) {
        const int count = len - t0 < G ? len - t0 : G;
        RW::fetch(a.q, RW::at(a.q, b, h, t0, tid), count, a.dk, tid, fq);
        RW::fetch(a.k, RW::at(a.k, b, h, t0, tid), count, a.dk, tid, fk);
        RW::fetch(a.dy, RW::at(a.dy, b, h, t0, tid), count, a.dv, tid, fy);
    };
    const int first = begin / G;
    int grp = (len - 1) / G;                // (len <= begin: no group)
    if (len > begin) fetch(grp * G);
    for (int turn = 0; len > begin && grp >= first; --grp, turn ^= 1) {
        const int t0 = grp * G, count = len - t0 < G ? len - t0 : G;
        float odd = RW::odd(fq) + RW::odd(fk) + RW::odd(fy);
        const uint8_t fd = a.done && lane < count ? a.done[(int64_t)(t0 + lane) * a.B + b] : 0;
        workgroup_lds_barrier();
        if ((int)threadIdx.x < count) {
            const float fr = delta_gate((char *)a.r.p + b * a.r.sb + h * a.r.sh + (t0 + threadIdx.x) * a.r.st, BF);
            const float fb = delta_gate((char *)a.b.p + b * a.b.sb + h * a.b.sh + (t0 + threadIdx.x) * a.b.st, BF);
            const float g = rate * delta_sigmoid(fr);
            sg[threadIdx.x] = g < -3e38f ? -3e38f : g;
            sbeta[threadIdx.x] = delta_sigmoid(fb);
            odd += (fr + fb) * 0.0f;
        }
        RW::put(q, fq, tid);
        RW::put(k, fk, tid);
        RW::put(dy, fy, tid);
        if (odd != odd) sodd[turn] = 1;
        const uint64_t ends = __ballot(lane < count && fd != 0);
        cut = cut || ends != 0;
        workgroup_lds_barrier();
        if (grp > first) fetch(t0 - G);
        const bool single = __builtin_amdgcn_readfirstlane(sodd[turn]) != 0;
        if (threadIdx.x == 0) sodd[turn ^ 1] = 0;
        auto piece = [&](int s, int p) {
            while (p-- > 0 && s < count) s = piece_end(s, count, ends, single);
            return s;
        };
        int batches = 0;
        for (int s = 0; s < count; s = piece(s, NP)) ++batches;
#pragma unroll 1
        for (int batch = batches - 1; batch >= 0; --batch) {
            const int s = piece(0, batch * NP);
            for (int p = w; p < NP; p += RW::NW) {
                const int from = piece(s, p);
                if (from >= count) break;
                floatx4 Tt, Tn, Pt, Pn;
                piece_triangles<BF, D, LD, WANT_ROWS | WANT_T | WANT_P, true>(q, k, sg, sbeta, from,
                                                                  piece_end(from, count, ends, single) - from, lane,
                                                                  cum[p], &rows[p], Tt, Tn, Pt, Pn);
                sT[p][lane] = Tn;
                sP[p][lane] = TL::split(Pn);
            }
            workgroup_lds_barrier();
#pragma unroll 1
            for (int p = NP - 1; p >= 0; --p) {
                const int from = piece(s, p);
                if (from >= count) continue;
                const int c = piece_end(from, count, ends, single) - from;
                const bool done = ends >> (from + c - 1) & 1;
                typename TL::sum2 kg, km;
                floatx4 dU, dM, A, B, C;
                if (done) {
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) Gs[kt] = M[kt] = floatx4{};
                }
#pragma unroll
                for (int kt = 0; kt < KT; kt += 2) {
                    const auto k0 = along_row<BF, LD>(k, from, kt, lane), k1 = along_row<BF, LD>(k, from, kt + 1, lane);
                    kg = TL::mm2(k0, k1, TL::split(Gs[kt]), TL::split(Gs[kt + 1]), kg);
                    km = TL::mm2(k0, k1, TL::split(M[kt]), TL::split(M[kt + 1]), km);
                }
                const auto dyc = along_col<BF, LD, true>(dy, from, c, w, lane);
                const floatx4 dyw = TL::wide(dyc);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    dU[i] = r4 + i < c ? kg[i] * rows[p].au[r4 + i] : 0.0f;
                    dM[i] = r4 + i < c ? km[i] * rows[p].au[r4 + i] : 0.0f;
                }
                dU = TL::mm(sP[p][lane], dyc, {dU}).v;
                const floatx4 dR = Tile<false>::mm(sT[p][lane], dU, {}).v;
                const floatx4 dN = Tile<false>::mm(sT[p][lane], dM, {}).v;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float ak = rows[p].ak[r4 + i];
                    A[i] = dyw[i] * rows[p].aq[r4 + i];
                    B[i] = r4 + i < c ? -(dR[i] * ak) : 0.0f;
                    C[i] = r4 + i < c ? -(dN[i] * ak) : 0.0f;
                }
                const val x = TL::split(A), y = TL::split(B), z = TL::split(C);
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    const auto kc = along_col<BF, LD, true>(k, from, c, kt, lane);
                    const auto qc = along_col<BF, LD, true>(q, from, c, kt, lane);
                    Gs[kt] = TL::mm(kc, y, TL::mm(qc, x, {Gs[kt] * rows[p].total})).v;
                    M[kt] = TL::mm(kc, z, {M[kt] * rows[p].total}).v;
                }
            }
            workgroup_lds_barrier();
        }
    }
    const int64_t part = ((int64_t)segment * gridDim.x + blockIdx.x) * D * D;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 16 * kt + r4 + i;
            a.adds[part + row * D + col] = Gs[kt][i];
            a.maps[part + row * D + col] = M[kt][i];
        }
    if (threadIdx.x == 0) a.cuts[segment * gridDim.x + blockIdx.x] = cut;
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

template <bool BF, int D>
void start_backward(DeltaArgs &a, hipStream_t s)
{
    const unsigned heads = (unsigned)(a.B * a.H);
    if (a.segments > 1) {                   // (nobody needs the first segment's map)
        hipLaunchKernelGGL((delta_bwd_map_kernel<BF, D>), dim3(heads, a.segments - 1), dim3(4 * D), 0, s, a);
        launch_delta_join(a, true, s);
    }
    hipLaunchKernelGGL((delta_bwd_kernel<BF, D>), dim3(heads, a.segments), dim3(4 * D), 0, s, a);
}

template <bool BF>
void start_backward(DeltaArgs &a, hipStream_t s)
{
    const int D = delta_width(a.dk, a.dv);
    if (D == 32) start_backward<BF, 32>(a, s);
    else if (D == 64) start_backward<BF, 64>(a, s);
    else start_backward<BF, 128>(a, s);
}

}  // namespace

hipError_t launch_delta_backward(DeltaArgs &a, hipStream_t s)
{
    delta_carve(a);
    if (a.bf16) start_backward<true>(a, s);
    else start_backward<false>(a, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(delta_lambda_kernel, dim3(a.H), dim3(256), 0, s, a.parts, a.B * a.segments, a.H, a.lam,
                       a.dlam);
    return hipGetLastError();
}

}  // namespace tpk
