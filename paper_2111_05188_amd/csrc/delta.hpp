// Gated delta rule over bars, shared device code.  A head's state S [dk][dv],
// queries and keys of unit length (q^ = q rq, k^ = k rk, r = 1/sqrt(x.x + eps)),
// a decay e^g, a write strength beta:
//   S' = e^g S,  u = beta (v - S'^T k^),  S <- S' + k^ u^T,  y = S^T q^.
//
// Up to 16 steps, a piece, go through the matrix units at once.  With the decays
// gamma_c from before the piece to step c, G[c][j] = gamma_c / gamma_j and S0
// the state before it:
//   L[c][j] = beta_c G[c][j] k^_c.k^_j  (j < c),     T = (I + L)^-1,
//   R = beta (V - gamma K^ S0),  U = T R,
//   Y = gamma Q^ S0 + P U,       P[c][j] = G[c][j] q^_c.k^_j  (j <= c),
//   S1 = gamma_C S0 + sum_c (gamma_C / gamma_c) k^_c u_c^T.
// A piece ends with an episode, so that neither its decays nor a NaN reach over
// an episode's end; steps with a NaN or an infinity near them are pieces of one
// step, so that nothing reaches the steps before.
//
// Products run on 16 x 16 tiles.  Lane l = 16 g + n of a wave holds rows 4g..4g+3
// of column n of a result, and that is also what the second operand of a product
// over those rows wants, so states and writes never leave the registers; the same
// registers taken as the first operand stand for the transposed tile.  In bf16 an
// operand that is not an input is three bf16 numbers that add up to it: states and
// writes go through many products one after the other, and keep fp32's precision
// so (with two numbers states were off by 4e-6, lambda's gradient by 3e-5).  A
// product over 16 fills half of the instruction's 32; where nothing else fits, the
// half-rate product over 16 saves the copies that would fill it.  T's and P's products
// with what is no input run in fp32: as many cycles as those of three numbers by three,
// and nothing to split.
#pragma once

#include "device.hpp"
#include "internal.hpp"

namespace tpk {
namespace {

constexpr float DELTA_LOG2E = 1.44269504088896341f;

// ---------------------------------------------------------------------------
// operands of a product over 16: Raw an input's own values, Val any fp32 values
// ---------------------------------------------------------------------------
template <bool BF> struct Tile;

// An accumulator of products over K.  It takes products of one kind only, and starts from
// zeros or a value that vector instructions made: hipcc puts no wait between two products
// on one accumulator, whatever their kinds (its listing has them back to back), and of unlike
// kinds the second read it before the first had written it (a product over 32 after one over
// 16: y off by an ulp of bf16, not always the same ones).
template <int K> struct Sum {
    floatx4 v = {};
    __device__ __forceinline__ float operator[](int i) const { return v[i]; }
};

template <> struct Tile<false> {
    typedef float elem;
    typedef floatx4 raw;
    typedef floatx4 val;
    static constexpr int PAD = 4;               // elements after a row in LDS
    static __device__ __forceinline__ val split(floatx4 x) { return x; }
    static __device__ __forceinline__ floatx4 wide(raw x) { return x; }
    static __device__ __forceinline__ floatx4 whole(val x) { return x; }
    typedef Sum<4> sum, sum2;                   // of products over 16 and over 32
    static __device__ __forceinline__ sum mm(floatx4 a, floatx4 b, sum c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c.v = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c.v, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ sum2 mm2(val a0, val a1, val b0, val b1, sum2 c)
    {
        return mm(a1, b1, mm(a0, b0, c));
    }
    // The transposed tile: a product with the unit matrix, which loses nothing.
    static __device__ __forceinline__ raw eye(int lane)
    {
        raw x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = 4 * (lane >> 4) + i == (lane & 15) ? 1.0f : 0.0f;
        return x;
    }
    static __device__ __forceinline__ floatx4 turned(val x, raw eye) { return mm(x, eye, {}).v; }
};

template <> struct Tile<true> {
    typedef __bf16 elem;
    typedef bf16x4 raw;
    struct val {
        bf16x4 hi, mid, lo;
    };
    static constexpr int PAD = 8;
    // The upper 8 bits of a significand, the next 8 and the last: nothing is lost.
    // (Rounding to the nearest, with the conversion instruction, takes as many
    // instructions and is slower: 390 x 4,096 x 4 x 64 forward 1.94 ms against 1.82.)
    static __device__ __forceinline__ val split(floatx4 x)
    {
        val v;
        uint32_t h[4], m[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = __float_as_uint(x[i]);
            const float r = x[i] - __uint_as_float(h[i] & 0xFFFF0000u);
            m[i] = __float_as_uint(r);
            l[i] = __float_as_uint(r - __uint_as_float(m[i] & 0xFFFF0000u));
        }
        v.hi = upper(h);
        v.mid = upper(m);
        v.lo = upper(l);
        return v;
    }
    static __device__ __forceinline__ bf16x4 upper(const uint32_t *w)
    {
        const uint32_t p[2] = {__builtin_amdgcn_perm(w[1], w[0], 0x07060302u),
                               __builtin_amdgcn_perm(w[3], w[2], 0x07060302u)};
        bf16x4 v;
        __builtin_memcpy(&v, p, sizeof v);
        return v;
    }
    static __device__ __forceinline__ floatx4 wide(raw x) { return __builtin_convertvector(x, floatx4); }
    static __device__ __forceinline__ floatx4 whole(const val &x) { return wide(x.hi) + (wide(x.mid) + wide(x.lo)); }
    static __device__ __forceinline__ bf16x8 join(bf16x4 a, bf16x4 b)
    {
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    typedef Sum<16> sum;
    typedef Sum<32> sum2;
    static __device__ __forceinline__ sum2 go(bf16x8 a, bf16x8 b, sum2 c)
    {
        return {__builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c.v, 0, 0, 0)};
    }
    // Half the rate of the products over 32, but no register is copied to fill one.
    static __device__ __forceinline__ sum go(bf16x4 a, bf16x4 b, sum c)
    {
        typedef short s4 __attribute__((ext_vector_type(4)));
        s4 x, y;
        __builtin_memcpy(&x, &a, sizeof x);
        __builtin_memcpy(&y, &b, sizeof y);
        return {__builtin_amdgcn_mfma_f32_16x16x16bf16_1k(x, y, c.v, 0, 0, 0)};
    }
    // (the least products first)
    static __device__ __forceinline__ sum mm(raw a, val b, sum c)
    {
        return go(a, b.hi, go(a, b.mid, go(a, b.lo, c)));
    }
    static __device__ __forceinline__ sum mm(val a, raw b, sum c)
    {
        return go(a.hi, b, go(a.mid, b, go(a.lo, b, c)));
    }
    static __device__ __forceinline__ raw eye(int lane)
    {
        raw x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (__bf16)(4 * (lane >> 4) + i == (lane & 15) ? 1.0f : 0.0f);
        return x;
    }
    static __device__ __forceinline__ floatx4 turned(val x, raw eye)
    {
        return go(x.hi, eye, go(x.mid, eye, go(x.lo, eye, {}))).v;
    }
    // products over 32
    static __device__ __forceinline__ sum2 mm2(raw a0, raw a1, val b0, val b1, sum2 c)
    {
        c = go(join(a0, a1), join(b0.lo, b1.lo), c);
        c = go(join(a0, a1), join(b0.mid, b1.mid), c);
        return go(join(a0, a1), join(b0.hi, b1.hi), c);
    }
    static __device__ __forceinline__ sum2 mm2(raw a0, raw a1, raw b0, raw b1, sum2 c)
    {
        return go(join(a0, a1), join(b0, b1), c);
    }
};

// ---------------------------------------------------------------------------
// rows of inputs in LDS: [G rows][D + PAD], 16-byte parts moved by the threads
// ---------------------------------------------------------------------------
typedef uint32_t Part __attribute__((ext_vector_type(4)));

template <bool BF, int D, int G>
struct Rows {
    typedef typename Tile<BF>::elem E;
    static constexpr int NT = 4 * D;                        // threads: a wave for 16 columns
    static constexpr int NW = D / 16;
    static constexpr int LD = D + Tile<BF>::PAD;
    static constexpr int PER = 16 / (int)sizeof(E);         // elements of a part
    static constexpr int PARTS = D / PER;                   // of a row
    static constexpr int N = G * PARTS / NT;                // parts of a thread
    static_assert(G * PARTS % NT == 0 && N >= 1 && NT % PARTS == 0, "threads share the rows evenly");

    // a thread's first part: its row and first column; the others are HOP rows on
    static constexpr int HOP = NT / PARTS;
    static __device__ __forceinline__ int row(int tid) { return tid / PARTS; }
    static __device__ __forceinline__ int col(int tid) { return tid % PARTS * PER; }

    // where a thread's first part of rows t0.. is
    static __device__ __forceinline__ char *at(const DeltaRows &m, int b, int h, int64_t t0, int tid)
    {
        return (char *)m.p + b * m.sb + h * m.sh + (t0 + row(tid)) * m.st + col(tid) * (int64_t)sizeof(E);
    }

    // rows of an array into registers; zeros past `count` rows and d columns
    static __device__ __forceinline__ void fetch(const DeltaRows &m, const char *at, int count, int d, int tid,
                                                 Part *reg)
    {
        const int64_t hop = HOP * m.st;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            Part p = {};
            const int r = row(tid) + i * HOP, c = col(tid);
            const char *from = at + i * hop;
            if (r < count && c < d) {
                if (m.vec) {
                    p = *(const TP_GLOBAL Part *)from;
                } else {
                    E e[PER];
#pragma unroll
                    for (int j = 0; j < PER; ++j) e[j] = c + j < d ? ((const TP_GLOBAL E *)from)[j] : (E)0.0f;
                    __builtin_memcpy(&p, e, sizeof p);
                }
            }
            reg[i] = p;
        }
    }

    static __device__ __forceinline__ void put(E *lds, const Part *reg, int tid)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) *(Part *)(lds + (row(tid) + i * HOP) * LD + col(tid)) = reg[i];
    }

    // the rows' values as they lie in LDS, zeros from row `count` to row `all`
    static __device__ __forceinline__ void store(const DeltaRows &m, char *at, int count, int all, int d, int tid,
                                                 const E *lds)
    {
        const int64_t hop = HOP * m.st;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = row(tid) + i * HOP, c = col(tid);
            if (r >= all || c >= d) continue;
            Part p = {};
            if (r < count) p = *(const Part *)(lds + r * LD + c);
            char *to = at + i * hop;
            if (m.vec) {
                *(TP_GLOBAL Part *)to = p;
            } else {
                E e[PER];
                __builtin_memcpy(e, &p, sizeof p);
#pragma unroll
                for (int j = 0; j < PER; ++j)
                    if (c + j < d) ((TP_GLOBAL E *)to)[j] = e[j];
            }
        }
    }

    // NaN if a NaN or an infinity is among this thread's parts, else 0
    static __device__ __forceinline__ float odd(const Part *reg)
    {
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (BF) {
                    typedef __bf16 two __attribute__((ext_vector_type(2)));
                    const uint32_t w = reg[i][j];
                    two v, z = {};
                    __builtin_memcpy(&v, &w, sizeof v);
                    x = __builtin_amdgcn_fdot2_f32_bf16(v, z, x, false);
                } else {
                    x = fmaf(__uint_as_float(reg[i][j]), 0.0f, x);
                }
            }
        return x;
    }
};

// rows s.. of a tile as the operand of a product over columns (k-tile kt)
template <bool BF, int LD, class E>
__device__ __forceinline__ typename Tile<BF>::raw along_row(const E *lds, int s, int kt, int lane)
{
    return *(const typename Tile<BF>::raw *)(lds + (s + (lane & 15)) * LD + 16 * kt + 4 * (lane >> 4));
}

// columns 16 ct.. of rows s.. as the operand of a product over the rows; rows
// from `count` on are zero where MASK.  In bf16 one transposing read: the 16 lanes
// of a group ask for 4 rows of 16 in parts of 4, and each gets a column of them.
template <bool BF, int LD, bool MASK, class E>
__device__ __forceinline__ typename Tile<BF>::raw along_col(const E *lds, int s, int count, int ct, int lane)
{
    typename Tile<BF>::raw v;
    const int n = lane & 15, r = 4 * (lane >> 4);
    if constexpr (BF) {
        typedef short s4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s4 *at;
        const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (at)(lds + (s + r + (n >> 2)) * LD + 16 * ct + 4 * (n & 3)));
        __builtin_memcpy(&v, &x, sizeof v);
    } else {
        const E *p = lds + (s + r) * LD + 16 * ct + n;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = p[i * LD];
    }
    if constexpr (MASK) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = r + i < count ? v[i] : (E)0.0f;
    }
    return v;
}

// The lane's number, as if it were not known yet: what is compared and computed from
// it stays inside the loop.  Outside, the compiler keeps some hundred lane masks and
// addresses alive, more than there are registers for.
__device__ __forceinline__ int fresh(int lane)
{
    asm volatile("" : "+v"(lane));
    return lane;
}

// The kernel's arguments, read anew: eleven arrays' pointers and strides are more than
// the scalar registers hold, and what the compiler keeps of them in others, through
// memory, waits for the loads under way.
__device__ __forceinline__ const DeltaArgs &fresh_args()
{
    auto p = (const __attribute__((address_space(4))) char *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const DeltaArgs *)(const char *)p;
}

// ---------------------------------------------------------------------------
// a piece's decays and triangles (one wave)
// ---------------------------------------------------------------------------

__device__ __forceinline__ float delta_gate(const char *p, bool bf)
{
    return bf ? (float)*(const TP_GLOBAL __bf16 *)p : *(const TP_GLOBAL float *)p;
}

// scalars of a piece's rows, and the decay over all of it
struct __attribute__((aligned(16))) PieceRows {
    float beta[16];
    float rq[16], rk[16];
    float aq[16], ak[16], au[16];   // gamma rq, beta gamma rk, (gamma_C / gamma) rk
    float total;
};

__device__ __forceinline__ float delta_softplus(float x)
{
    return (x > 0.0f ? x : 0.0f) + log1pf(expf(-fabsf(x))) + (x != x ? x : 0.0f);
}

__device__ __forceinline__ float delta_sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

__device__ __forceinline__ float delta_exp(float x) { return __builtin_amdgcn_exp2f(x * DELTA_LOG2E); }

// Decays between the steps of a piece, in the layout of a result: fade[i] between
// steps 4g+i and n, whichever is first.  Sums of g run in 64 bits, so that a closed
// gate does not blur the decays after it.
__device__ __forceinline__ floatx4 piece_decays(const double *cum, int lane)
{
    const int n = lane & 15, r = 4 * (lane >> 4);
    const double cn = cum[n];
    floatx4 fade;
#pragma unroll
    for (int i = 0; i < 4; ++i) fade[i] = delta_exp(-fabsf((float)(cum[r + i] - cn)));
    return fade;
}

// Sums of the log-decays over a piece's steps, by its wave, in the wave's own LDS.
__device__ __forceinline__ double piece_sums(const float *g, int count, int lane, double *cum)
{
    const int n = lane & 15;
    double c = n < count ? (double)g[n] : 0.0;
    c += dpp_f64<DPP_ROW_SHR + 1>(c);
    c += dpp_f64<DPP_ROW_SHR + 2>(c);
    c += dpp_f64<DPP_ROW_SHR + 4>(c);
    c += dpp_f64<DPP_ROW_SHR + 8>(c);
    if (lane < 16) cum[n] = c;
    wave_lds_fence();
    return c;
}

// What one wave prepares of a piece.  (`rows` has the rows' scalars with WANT_ROWS, else
// it is the wave's own while it works.)
// WANT_L: L, with T, in Pn's place.
enum : int { WANT_T = 1, WANT_PT = 2, WANT_P = 4, WANT_ROWS = 8, WANT_L = 16 };

// K K^T and Q K^T tiles of a piece, the rows' lengths, T and P in both layouts (as
// far as they are wanted).  L is nilpotent; its inverse grows from blocks of 1, 2, 4,
// 8 on the diagonal: T <- T - T L_off T with the part of L that joins two blocks, so
// no power of L is formed whose entries cancel.  Rows past the piece's end have
// length 0 and no decay, whatever LDS holds there: an output or a gradient may be a NaN.
template <bool BF, int D, int LD, int WANT, bool BOTH, class E>
__device__ __forceinline__ void piece_triangles(const E *q, const E *k, const float *g, const float *beta, int s,
                                                int count, int lane, double *cum, PieceRows *rows,
                                                floatx4 &Tt, floatx4 &Tn, floatx4 &Pt, floatx4 &Pn)
{
    constexpr float EPS = 1e-6f;
    lane = fresh(lane);
    constexpr bool Q = (WANT & (WANT_P | WANT_PT | WANT_ROWS)) != 0, B = (WANT & (WANT_T | WANT_ROWS)) != 0;
    const int n = lane & 15, grp = lane >> 4, r = 4 * grp;
    typename Tile<BF>::sum2 kk, qq, kq, qk;
#pragma unroll
    for (int kt = 0; kt < D / 16; kt += 2) {
        const auto a0 = along_row<BF, LD>(k, s, kt, lane), b0 = along_row<BF, LD>(Q ? q : k, s, kt, lane);
        const auto a1 = along_row<BF, LD>(k, s, kt + 1, lane), b1 = along_row<BF, LD>(Q ? q : k, s, kt + 1, lane);
        kk = Tile<BF>::mm2(a0, a1, a0, a1, kk);
        if constexpr (Q) qq = Tile<BF>::mm2(b0, b1, b0, b1, qq);
        if constexpr (WANT & WANT_P) qk = Tile<BF>::mm2(b0, b1, a0, a1, qk);
        if constexpr (WANT & WANT_PT) kq = Tile<BF>::mm2(a0, a1, b0, b1, kq);
    }
    const float be = B && n < count ? beta[s + n] : 0.0f;
    const double c = piece_sums(g + s, count, lane, cum);
    if (count < 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool it = r + i < count && n < count;
            kk.v[i] = it ? kk[i] : 0.0f;
            qq.v[i] = it ? qq[i] : 0.0f;
            kq.v[i] = it ? kq[i] : 0.0f;
            qk.v[i] = it ? qk[i] : 0.0f;
        }
    }
    // lengths from the diagonals: lane 16 (n/4) + n has row n's
    if (grp == n >> 2) {
        const float dk = n & 2 ? (n & 1 ? kk[3] : kk[2]) : (n & 1 ? kk[1] : kk[0]);
        const float dq = n & 2 ? (n & 1 ? qq[3] : qq[2]) : (n & 1 ? qq[1] : qq[0]);
        rows->rk[n] = n < count ? __builtin_amdgcn_rsqf(dk + EPS) : 0.0f;
        if constexpr (Q) rows->rq[n] = n < count ? __builtin_amdgcn_rsqf(dq + EPS) : 0.0f;
        if constexpr (B) rows->beta[n] = be;
    }
    const floatx4 fade = piece_decays(cum, lane);
    wave_lds_fence();
    const float rkn = rows->rk[n], rqn = rows->rq[n];
    const floatx4 rkr = *(const floatx4 *)(rows->rk + r), rqr = *(const floatx4 *)(rows->rq + r);
    if constexpr (WANT & WANT_ROWS) {
        if (lane < 16) {
            const double all = cum[15];
            const float since = n < count ? delta_exp((float)c) : 0.0f;
            const float rest = n < count ? delta_exp((float)(all - c)) : 0.0f;
            if (n == 0) rows->total = delta_exp((float)all);
            rows->aq[n] = since * rqn;
            rows->ak[n] = be * since * rkn;
            rows->au[n] = rest * rkn;
        }
    }
    if constexpr (WANT & WANT_T) {
        const floatx4 ber = *(const floatx4 *)(rows->beta + r);
        const bool same4 = grp == n >> 2, same8 = grp >> 1 == n >> 3;
        floatx4 Lt, off;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = kk[i] * rkr[i] * (rkn * fade[i]);
            const float Ln = r + i > n ? x * ber[i] : 0.0f;     // row r+i after column n
            Lt[i] = r + i < n ? x * be : 0.0f;                  // transposed
            if constexpr (WANT & WANT_L) Pn[i] = Ln;
            // blocks of two: I - L inside them
            const float unit = r + i == n ? 1.0f : 0.0f;
            const bool same2 = 2 * grp + i / 2 == n >> 1;
            Tn[i] = same2 ? unit - Ln : 0.0f;
            Tt[i] = same2 ? unit - Lt[i] : 0.0f;
            off[i] = same4 && !same2 ? -Lt[i] : 0.0f;
        }
#pragma unroll
        for (int w = 2; w < 16; w *= 2) {
            if (w > 2)
#pragma unroll
                for (int i = 0; i < 4; ++i) off[i] = (w == 4 ? same8 && !same4 : !same8) ? -Lt[i] : 0.0f;
            const floatx4 Y = Tile<false>::mm(off, Tn, {}).v;       // -L_off T
            const floatx4 t = Tile<false>::mm(Y, Tt, {Tt}).v;       // T^T - (L_off T)^T T^T
            if (BOTH || w < 8) Tn = Tile<false>::mm(Tt, Y, {Tn}).v;
            Tt = t;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (WANT & WANT_P) Pn[i] = r + i >= n ? qk[i] * rqr[i] * (rkn * fade[i]) : 0.0f;
        if constexpr (WANT & WANT_PT) Pt[i] = r + i <= n ? kq[i] * rkr[i] * (rqn * fade[i]) : 0.0f;
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}

// Sums over the 16 lanes of a row group: lane n gets that of x[n % 4].  (Lanes swap halves
// of what they have, so that the four sums go on in one register.)
__device__ __forceinline__ float row_sums(floatx4 x, int lane)
{
    const bool odd = lane & 1, upper = lane & 2;
    const float a = (odd ? x[1] : x[0]) + dpp<0xB1>(odd ? x[0] : x[1]);
    const float b = (odd ? x[3] : x[2]) + dpp<0xB1>(odd ? x[2] : x[3]);
    float c = (upper ? b : a) + dpp<0x4E>(upper ? a : b);
    c += dpp<0x124>(c);
    return c + dpp<0x128>(c);
}

// The next piece from step s of a group of `count` steps: it ends with a whole
// tile, an episode, the group or the steps that a kept state is for.
__device__ __forceinline__ int piece_end(int s, int count, uint64_t ends, bool single)
{
    int e = single ? s + 1 : s + 16;
    const int mark = (s / DELTA_GROUP + 1) * DELTA_GROUP;
    if (e > mark) e = mark;
    if (e > count) e = count;
    const uint64_t m = ends >> s;
    if (m) {
        const int d = s + __builtin_ctzll(m) + 1;
        if (d < e) e = d;
    }
    return e;
}

}  // namespace
}  // namespace tpk
