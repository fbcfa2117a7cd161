// Gated delta rule: whole sequences forward, and one step (delta.hpp has the
// formulas).
//
// Forward, a workgroup has one head of one sequence; wave w has columns 16w.. of
// its state, all rows of them, in registers.  Groups of steps go through LDS:
// the next group's loads are under way while one is worked on.  Each wave first
// prepares one piece of the group (its triangles, which do not need the state),
// then all waves run the pieces on their columns.
//
// 390 steps of 4,096 sequences of 4 heads of 64 in bf16: 1.70 ms, 3.8 GB at 2.3 TB/s.
// Vector instructions (62% of the time) and the matrix units (40%) bound it, above
// all the splits of the state into three bf16 numbers, once a piece.  Three workgroups a
// CU; four (128 registers) or groups of 32 steps gain nothing (1.69 - 1.94 ms), nor do gates shared out over the waves (1.76).
//
// Where few heads leave most CUs without work, a sequence is split into segments.
// What a segment does to the state is linear: a first launch runs every segment on
// no state, for what it adds, and without values on the unit states, for its map;
// then each segment's first state comes from them, one product a segment, or, for many,
// over blocks of them.  24,570 steps of 4 heads of 128 in bf16: 270 us (6.6 ms
// without segments), of which maps 106, join 86, outputs 92; each of the three
// is a chain, of six groups of 64 steps or of eight segments' maps at a time.
#include "delta.hpp"

namespace tpk {
namespace {

// one piece on the state's columns of this wave; OUT: its outputs, in place of v
template <bool BF, int D, int LD, bool MASK, bool OUT, class E>
__device__ __forceinline__ void run_piece(const E *q, const E *k, E *v, int s, int count, bool ends,
                                          const PieceRows &rows, const floatx4 &Tt, const floatx4 &Pt, int w,
                                          int lane, floatx4 *S)
{
    typedef Tile<BF> TL;
    constexpr int KT = D / 16;
    lane = fresh(lane);
    const int r = 4 * (lane >> 4);
    typename TL::sum2 ks, qs;
#pragma unroll
    for (int kt = 0; kt < KT; kt += 2) {
        const auto x0 = TL::split(S[kt]), x1 = TL::split(S[kt + 1]);
        ks = TL::mm2(along_row<BF, LD>(k, s, kt, lane), along_row<BF, LD>(k, s, kt + 1, lane), x0, x1, ks);
        if constexpr (OUT)
            qs = TL::mm2(along_row<BF, LD>(q, s, kt, lane), along_row<BF, LD>(q, s, kt + 1, lane), x0, x1, qs);
    }
    const floatx4 vv = TL::wide(along_col<BF, LD, MASK>(v, s, count, w, lane));
    const floatx4 be = *(const floatx4 *)(rows.beta + r), ak = *(const floatx4 *)(rows.ak + r);
    const floatx4 aq = *(const floatx4 *)(rows.aq + r), au = *(const floatx4 *)(rows.au + r);
    floatx4 R, o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        R[i] = !MASK || r + i < count ? be[i] * vv[i] - ak[i] * ks[i] : 0.0f;
        o[i] = aq[i] * qs[i];
    }
    const floatx4 U = Tile<false>::mm(Tt, R, {}).v;
    if constexpr (OUT) {
        o = Tile<false>::mm(Pt, U, {o}).v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (!MASK || r + i < count) v[(s + r + i) * LD + 16 * w + (lane & 15)] = (E)o[i];
    }
    if (ends) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) S[kt] = floatx4{};
        return;
    }
    floatx4 W;
#pragma unroll
    for (int i = 0; i < 4; ++i) W[i] = !MASK || r + i < count ? U[i] * au[i] : 0.0f;
    const auto x = TL::split(W);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
        S[kt] = TL::mm(along_col<BF, LD, MASK>(k, s, count, kt, lane), x, {S[kt] * rows.total}).v;
}

// what a piece does to the unit states (a value's columns are zero)
template <bool BF, int D, int LD, bool MASK, class E>
__device__ __forceinline__ void map_piece(const E *k, int s, int count, bool ends, const PieceRows &rows,
                                          const floatx4 &Tt, int lane, floatx4 *S)
{
    typedef Tile<BF> TL;
    constexpr int KT = D / 16;
    lane = fresh(lane);
    const int r = 4 * (lane >> 4);
    typename TL::sum2 ks;
    floatx4 R, W;
#pragma unroll
    for (int kt = 0; kt < KT; kt += 2)
        ks = TL::mm2(along_row<BF, LD>(k, s, kt, lane), along_row<BF, LD>(k, s, kt + 1, lane), TL::split(S[kt]),
                     TL::split(S[kt + 1]), ks);
#pragma unroll
    for (int i = 0; i < 4; ++i) R[i] = !MASK || r + i < count ? -(rows.ak[r + i] * ks[i]) : 0.0f;
    const floatx4 U = Tile<false>::mm(Tt, R, {}).v;
#pragma unroll
    for (int i = 0; i < 4; ++i) W[i] = !MASK || r + i < count ? U[i] * rows.au[r + i] : 0.0f;
    const auto x = TL::split(W);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        S[kt] = TL::mm(along_col<BF, LD, MASK>(k, s, count, kt, lane), x, {S[kt] * rows.total}).v;
        if (ends) S[kt] = floatx4{};
    }
}

// MAP: a segment's map and what it adds, instead of outputs
template <bool BF, int D, int G, bool MAP>
__global__ __launch_bounds__(4 * D, D == 128 ? 2 : 3) void delta_fwd_kernel(DeltaArgs a)
{
    constexpr int NP = G / 16, KT = D / 16;
    typedef Rows<BF, D, G> RW;
    typedef typename RW::E E;
    constexpr int LD = RW::LD, NW = RW::NW;
    __shared__ __attribute__((aligned(16))) E buf[(3 * G + 16) * LD];
    __shared__ floatx4 sT[NP][64], sP[NP][64];
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
    // this segment's steps
    const int begin = blockIdx.y * a.seg_len, end = a.T - begin < a.seg_len ? a.T : begin + a.seg_len;
    len = len < end ? len : end;
    const float rate = -8.0f * delta_softplus(a.lam[h]);
    const int64_t st = ((int64_t)b * a.H + h) * a.dk * a.dv;
    const int64_t part = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * D * D;
    const int col = 16 * w + n;
    floatx4 S[KT], M[MAP ? KT : 1];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 16 * kt + r4 + i;
            if constexpr (MAP) {
                S[kt][i] = 0.0f;
                M[kt][i] = row == col ? 1.0f : 0.0f;
            } else if (a.segments > 1) {
                S[kt][i] = a.adds[part + row * D + col];
            } else {
                S[kt][i] = a.h0 && row < a.dk && col < a.dv ? a.h0[st + (int64_t)row * a.dv + col] : 0.0f;
            }
        }
    bool cut = false;

    const int tid = threadIdx.x;
    const char *pq = RW::at(a.q, b, h, begin, tid), *pk = RW::at(a.k, b, h, begin, tid), *pv = RW::at(a.v, b, h, begin, tid);
    char *py = !MAP && a.y.p ? RW::at(a.y, b, h, begin, tid) : nullptr;
    const char *pr = (char *)a.r.p + b * a.r.sb + h * a.r.sh + (begin + (int64_t)threadIdx.x) * a.r.st;
    const char *pb = (char *)a.b.p + b * a.b.sb + h * a.b.sh + (begin + (int64_t)threadIdx.x) * a.b.st;
    const uint8_t *pd = a.done ? a.done + (int64_t)(begin + lane) * a.B + b : nullptr;
    float *ps = !MAP && a.saved
                    ? a.saved + ((int64_t)(begin / DELTA_GROUP) * gridDim.x + blockIdx.x) * D * D + r4 * D + col
                    : nullptr;
    Part fq[RW::N], fk[RW::N], fv[RW::N];
    float fr = 0.0f, fb = 0.0f;
    uint8_t fd = 0;
    auto fetch = [&](int count) {
        if constexpr (!MAP) RW::fetch(a.q, pq, count, a.dk, tid, fq);
        RW::fetch(a.k, pk, count, a.dk, tid, fk);
        RW::fetch(a.v, pv, count, a.dv, tid, fv);
        pq += G * a.q.st;
        pk += G * a.k.st;
        pv += G * a.v.st;
        if ((int)threadIdx.x < count) {
            fr = delta_gate(pr, BF);
            fb = delta_gate(pb, BF);
        }
        pr += G * a.r.st;
        pb += G * a.b.st;
        if (pd) {
            fd = lane < count ? *(const TP_GLOBAL uint8_t *)pd : 0;
            pd += G * (int64_t)a.B;
        }
    };
    fetch(len - begin < G ? len - begin : G);
    if (threadIdx.x < 2) sodd[threadIdx.x] = 0;
    workgroup_lds_barrier();
    for (int t0 = begin, turn = 0; t0 < end; t0 += G, turn ^= 1) {
        const int count = len - t0 < G ? len - t0 : G, all = end - t0 < G ? end - t0 : G;
        if (count > 0) {
            if constexpr (!MAP) RW::put(q, fq, tid);
            RW::put(k, fk, tid);
            RW::put(v, fv, tid);
            float odd = (MAP ? 0.0f : RW::odd(fq)) + RW::odd(fk) + RW::odd(fv);
            if ((int)threadIdx.x < count) {
                const float g = rate * delta_sigmoid(fr);
                sg[threadIdx.x] = g < -3e38f ? -3e38f : g;
                sbeta[threadIdx.x] = delta_sigmoid(fb);
                odd += (fr + fb) * 0.0f;
            }
            const uint64_t ends = __ballot(lane < count && fd != 0);
            if (odd != odd) sodd[turn] = 1;
            workgroup_lds_barrier();
            if (t0 + G < len) fetch(len - t0 - G < G ? len - t0 - G : G);
            const bool single = __builtin_amdgcn_readfirstlane(sodd[turn]) != 0;
            if (threadIdx.x == 0) sodd[turn ^ 1] = 0;
            for (int s = 0; s < count;) {
                for (int p = w; p < NP; p += NW) {
                    int from = s;
                    for (int j = 0; j < p && from < count; ++j) from = piece_end(from, count, ends, single);
                    if (from >= count) break;
                    floatx4 Tt, Tn, Pt, Pn;
                    piece_triangles<BF, D, LD, WANT_ROWS | (MAP ? WANT_T : WANT_T | WANT_PT), false>(MAP ? k : q, k, sg, sbeta, from,
                                                      piece_end(from, count, ends, single) - from, lane, cum[p],
                                                      &rows[p], Tt, Tn, Pt, Pn);
                    sT[p][lane] = Tt;
                    if constexpr (!MAP) sP[p][lane] = Pt;
                }
                workgroup_lds_barrier();
#pragma unroll 1
                for (int p = 0; p < NP && s < count; ++p) {
                    const int e = piece_end(s, count, ends, single);
                    const bool done = ends >> (e - 1) & 1;
                    if (ps && s % DELTA_GROUP == 0) {
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                            for (int i = 0; i < 4; ++i) ((TP_GLOBAL float *)ps)[(16 * kt + i) * D] = S[kt][i];
                        ps += (int64_t)gridDim.x * D * D;
                    }
                    if constexpr (MAP) {
                        cut = cut || done;
                        if (e - s == 16) {
                            run_piece<BF, D, LD, false, !MAP>(q, k, v, s, 16, done, rows[p], sT[p][lane], sP[p][lane],
                                                        w, lane, S);
                            map_piece<BF, D, LD, false>(k, s, 16, done, rows[p], sT[p][lane], lane, M);
                        } else {
                            run_piece<BF, D, LD, true, !MAP>(q, k, v, s, e - s, done, rows[p], sT[p][lane], sP[p][lane],
                                                       w, lane, S);
                            map_piece<BF, D, LD, true>(k, s, e - s, done, rows[p], sT[p][lane], lane, M);
                        }
                    } else if (e - s == 16)
                        run_piece<BF, D, LD, false, !MAP>(q, k, v, s, 16, done, rows[p], sT[p][lane], sP[p][lane], w,
                                                    lane, S);
                    else
                        run_piece<BF, D, LD, true, !MAP>(q, k, v, s, e - s, done, rows[p], sT[p][lane], sP[p][lane], w,
                                                   lane, S);
                    s = e;
                }
                workgroup_lds_barrier();
            }
        }
        if (py) {
            RW::store(a.y, py, count > 0 ? count : 0, all, a.dv, tid, v);
            py += G * a.y.st;
        }
    }
    if constexpr (MAP) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * kt + r4 + i;
                a.adds[part + row * D + col] = S[kt][i];
                a.maps[part + row * D + col] = M[kt][i];
            }
        if (threadIdx.x == 0) a.cuts[blockIdx.y * gridDim.x + blockIdx.x] = cut;
    } else if (a.h_last && end == a.T) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * kt + r4 + i;
                if (row < a.dk && col < a.dv) a.h_last[st + (int64_t)row * a.dv + col] = S[kt][i];
            }
    }
}

// The state after a run of segments, or before every one of them.  In the order of
// their positions (backward: from the last segment on) they are split into blocks of
// `per`.  FOLD: a block's own map and what it adds, from its segments' (columns of the
// unit states, then of no state).  Else the first state of every segment, in the place of
// what it adds, from `first`, or from each block's in `starts`.
struct DeltaJoin {
    const float *maps;
    float *adds;
    const int32_t *cuts;
    int n, per;
    bool backward;
    const float *first, *starts;
    int dk, dv;
    float *block_maps, *block_adds;
    int32_t *block_cuts;
};

// A workgroup has 16 columns of one head's states, wave w the rows 16w.. of
// them; all waves read all rows of the state before from LDS.
template <int D, bool FOLD>
__global__ __launch_bounds__(4 * D) void delta_join_kernel(DeltaJoin a)
{
    constexpr int KT = D / 16;
    __shared__ floatx4 state[2][KT][64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, r4 = 4 * (lane >> 4), heads = gridDim.x;
    const bool unit = FOLD && blockIdx.y < KT;
    const int col = (FOLD && !unit ? blockIdx.y - KT : blockIdx.y) * 16 + n;
    const int from = blockIdx.z * a.per, count = a.n - from < a.per ? a.n - from : a.per;
    const int64_t block = ((int64_t)blockIdx.z * heads + blockIdx.x) * D * D;
    const int64_t st = (int64_t)blockIdx.x * a.dk * a.dv;
    floatx4 S;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 16 * w + r4 + i;
        if constexpr (FOLD) S[i] = unit && row == col ? 1.0f : 0.0f;
        else if (a.starts) S[i] = a.starts[block + row * D + col];
        else S[i] = a.first && row < a.dk && col < a.dv ? a.first[st + (int64_t)row * a.dv + col] : 0.0f;
    }
    // products: of all segments but, where nothing follows, the last
    const int steps = FOLD ? count : count - 1;
    struct Segment {
        floatx4 add, map[KT];
        int cut;
    };
    auto place = [&](int x) {
        const int seg = a.backward ? a.n - 1 - from - x : from + x;
        return (int64_t)seg * heads + blockIdx.x;
    };
    auto fetch = [&](int x, Segment &g) {
        const int64_t at = place(x) * D * D;
        g.cut = a.cuts[place(x)];
#pragma unroll
        for (int i = 0; i < 4; ++i) g.add[i] = unit ? 0.0f : a.adds[at + (16 * w + r4 + i) * D + col];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
            g.map[kt] = *(const floatx4 *)(a.maps + at + (16 * w + n) * D + 16 * kt + r4);
    };
    bool cut = false;
    // the state before segment x goes to its place; the one after it, with the loads of
    // the next but one on their way
    auto step = [&](int x, Segment &g) {
        const int64_t at = place(x) * D * D;
        if constexpr (!FOLD) {
#pragma unroll
            for (int i = 0; i < 4; ++i) a.adds[at + (16 * w + r4 + i) * D + col] = S[i];
        }
        state[x & 1][w][lane] = S;
        if (x >= steps) return;
        cut = cut || g.cut != 0;
        workgroup_lds_barrier();
        Sum<4> one{g.add}, half;            // (two chains of products)
        if (g.cut == 0)
#pragma unroll
            for (int kt = 0; kt < KT; kt += 2) {
                one = Tile<false>::mm(g.map[kt], state[x & 1][kt][lane], one);
                half = Tile<false>::mm(g.map[kt + 1], state[x & 1][kt + 1][lane], half);
            }
        S = one.v + half.v;
        if (x + 2 < steps) fetch(x + 2, g);
    };
    Segment even, odd;
    if (steps > 0) fetch(0, even);
    if (steps > 1) fetch(1, odd);
    for (int x = 0; x < count; x += 2) {
        step(x, even);
        if (x + 1 < count) step(x + 1, odd);
    }
    if constexpr (FOLD) {
        float *to = (unit ? a.block_maps : a.block_adds) + block;
#pragma unroll
        for (int i = 0; i < 4; ++i) to[(16 * w + r4 + i) * D + col] = S[i];
        if (blockIdx.y == 0 && threadIdx.x == 0) a.block_cuts[(int64_t)blockIdx.z * heads + blockIdx.x] = cut;
    }
}

// One step: a workgroup has one head of one sequence, its state in registers
// between the one read and the one write.  y = e^g S^T q^ + (k^.q^) u, so both
// products are of the state as it came.  The states' two passes through memory
// bound it: 4,096 accounts of 8 heads of 64, 195 us (5.6 TB/s).
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
                                  delta_sigmoid(delta_gate(base(a.r), BF)));
    const float beta = delta_sigmoid(delta_gate(base(a.b), BF));
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

template <bool BF, int D>
void start_forward(DeltaArgs &a, hipStream_t s)
{
    constexpr int G = BF ? 64 : 32;
    const unsigned heads = (unsigned)(a.B * a.H);
    if (a.segments > 1) {                   // (nobody needs the last segment's map)
        hipLaunchKernelGGL((delta_fwd_kernel<BF, D, G, true>), dim3(heads, a.segments - 1), dim3(4 * D), 0, s, a);
        launch_delta_join(a, false, s);
    }
    hipLaunchKernelGGL((delta_fwd_kernel<BF, D, G, false>), dim3(heads, a.segments), dim3(4 * D), 0, s, a);
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
    // steps past the last group, and the threads of all sequences' heads, in 32 bits
    return T <= 1 << 30 && (int64_t)B * H < (int64_t)1 << 23;
}

size_t delta_saved_bytes(int T, int B, int H, int dk, int dv)
{
    const size_t D = delta_width(dk, dv);
    return (size_t)((T + DELTA_GROUP - 1) / DELTA_GROUP) * B * H * D * D * sizeof(float);
}

static int delta_segments(int T, int B, int H, int &seg_len)
{
    const int64_t heads = (int64_t)B * H, groups = ((int64_t)T + 63) / 64;
    int64_t want = heads < 256 ? 512 / heads : 1;
    if (want > 64) want = 64;
    if (want > groups / 2) want = groups / 2;
    if (want < 2) want = 1;
    const int64_t per = (groups + want - 1) / want;
    seg_len = (int)(per * 64);
    return (int)((groups + per - 1) / per);
}

// blocks of segments (1: the join takes them one after the other), and of how many
static int delta_blocks(int segments, int &per)
{
    per = segments;
    if (segments <= 24) return 1;
    per = 1;
    while (per * per < segments) ++per;
    return (segments + per - 1) / per;
}

static size_t delta_round(size_t bytes) { return (bytes + 255) / 256 * 256; }

// lambda's parts, one a head and segment; the maps of segments, and of blocks of them
size_t delta_workspace_bytes(int T, int B, int H, int dk, int dv)
{
    int seg_len, per;
    const int segments = delta_segments(T, B, H, seg_len), blocks = delta_blocks(segments, per);
    const size_t heads = (size_t)B * H, D = delta_width(dk, dv), state = 2 * D * D * sizeof(float);
    size_t bytes = delta_round(segments * heads * sizeof(double));
    if (segments > 1) bytes += delta_round(segments * heads * sizeof(int32_t)) + segments * heads * state;
    if (blocks > 1) bytes += delta_round(blocks * heads * sizeof(int32_t)) + blocks * heads * state;
    return bytes;
}

void delta_carve(DeltaArgs &a)
{
    a.segments = delta_segments(a.T, a.B, a.H, a.seg_len);
    const size_t n = (size_t)a.segments * a.B * a.H, D = delta_width(a.dk, a.dv);
    char *p = (char *)a.work;
    a.parts = (double *)p;
    p += delta_round(n * sizeof(double));
    a.cuts = (int32_t *)p;
    p += delta_round(n * sizeof(int32_t));
    a.maps = (float *)p;
    a.adds = a.maps + n * D * D;
}

template <int D>
static void start_join(const DeltaArgs &a, bool backward, hipStream_t s)
{
    const unsigned heads = (unsigned)(a.B * a.H);
    DeltaJoin j = {};
    j.maps = a.maps;
    j.adds = a.adds;
    j.cuts = a.cuts;
    j.n = a.segments;
    j.backward = backward;
    j.first = backward ? a.dh_last : a.h0;
    j.dk = a.dk;
    j.dv = a.dv;
    const unsigned blocks = delta_blocks(a.segments, j.per);
    if (blocks > 1) {
        const size_t n = (size_t)blocks * heads;
        char *p = (char *)(a.adds + (size_t)a.segments * heads * D * D);
        j.block_cuts = (int32_t *)p;
        j.block_maps = (float *)(p + delta_round(n * sizeof(int32_t)));
        j.block_adds = j.block_maps + n * D * D;
        hipLaunchKernelGGL((delta_join_kernel<D, true>), dim3(heads, D / 8, blocks - 1), dim3(4 * D), 0, s, j);
        DeltaJoin o = j;
        o.maps = j.block_maps;
        o.adds = j.block_adds;
        o.cuts = j.block_cuts;
        o.n = o.per = blocks;
        o.backward = false;
        hipLaunchKernelGGL((delta_join_kernel<D, false>), dim3(heads, D / 16), dim3(4 * D), 0, s, o);
        j.starts = j.block_adds;
    }
    hipLaunchKernelGGL((delta_join_kernel<D, false>), dim3(heads, D / 16, blocks), dim3(4 * D), 0, s, j);
}

void launch_delta_join(const DeltaArgs &a, bool backward, hipStream_t s)
{
    const int D = delta_width(a.dk, a.dv);
    if (D == 32) start_join<32>(a, backward, s);
    else if (D == 64) start_join<64>(a, backward, s);
    else start_join<128>(a, backward, s);
}

template <bool BF>
static void start_forward(DeltaArgs &a, hipStream_t s)
{
    const int D = delta_width(a.dk, a.dv);
    if (D == 32) start_forward<BF, 32>(a, s);
    else if (D == 64) start_forward<BF, 64>(a, s);
    else start_forward<BF, 128>(a, s);
}

hipError_t launch_delta_forward(DeltaArgs &a, hipStream_t s)
{
    delta_carve(a);
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
