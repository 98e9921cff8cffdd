// Gated delta rule, backward.  With the notation of the forward pass, dS1 the gradient of the state after a chunk of 32 steps:
//     dU  = A^T dO + diag(exp(G_C - G)) K dS1
//     Z   = ((I + diag(beta) N)^-1)^T dU                                    the gradient of what each step writes;  dV = diag(beta) Z
//     dS0 = exp(G_C) dS1 + (scale diag(exp G) Q)^T dO - (diag(exp G) K)^T diag(beta) Z
// k_delta_adjoint walks the chunks backwards with that (the forward states do not enter).  Z, like E, does not depend on where chunks are cut, so
// k_delta_grads takes slots of 64 steps, all side by side, with the states S0 and dS1 at their ends (D_ij = exp(G_i - G_j)):
//     F = scale (dO U^T) o D  (j <= i),      H = -(diag(beta) Z U^T) o D  (j < i)
//     dQ = scale diag(exp G) dO S0^T + F K
//     dK = -diag(exp G) diag(beta) Z S0^T + (H + H^T) K + F^T Q + diag(exp(G_C - G)) U dS1^T
//     dbeta_t = z_t . e_t,     dg_t = sum of dG_i over i >= t,
//     dG_i = sum_j M_ij - sum_j M_ji + q_i . (state part of dQ_i) + k_i . (-.. Z S0^T part) - k_i . (U dS1^T part),   M = F o Q K^T + H o K K^T
//     and at the slot's last step also the sum of k . (U dS1^T part) and exp(G_C) <S0, dS1>.
// Row and column sums of M are taken in float32, without the diagonal, which cancels.
#include "delta_common.hpp"

namespace lrnnx {

// ---------------------------------------------------------------- the walk backwards
// As in the forward walk a wavefront owns 16 columns of dS, or two share them, and everything it computes of them stays in its registers.  Bound by the
// latency of a chunk: 4 x 4096 steps of 16 heads of 128 x 128, bfloat16, 128 chunks in 254 us (343 with one wavefront to 16 columns).
template <int NPI, int NP, int DK, int NBUF, int DS> struct AdjLds {
    struct Buf {
        uint16_t k[NPI][32][DK + 8], kt[NPI][DK][40], qt[NPI][DK][40];
        uint16_t th[NP][256], tw[NP][512], ah[NP][256], aw[NP][512];           // (as they lie in memory)
        float scal[96];
    } buf[NBUF];
    f32x4 halves[DS == 2 ? 8 : 1][64];
};

// DEEP: loads two chunks ahead, for launches of at most a workgroup a compute unit, where registers are there for it and nothing else hides memory
// (the same case: 285 us without; the forward walk gains nothing by it, with one or two wavefronts to 16 columns).
template <int NPI, int NP, int DK, int DS, bool EXACT, bool AGG, bool DEEP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DEEP && (DS == 1 || NP == 3) ? 1 : 2, DEEP && (DS == 1 || NP == 3) ? 1 : 2))) void k_delta_adjoint(const DeltaParams p) {
    constexpr int NT = 256, CW = 4 / DS, KS = DK / 32 / DS, MT = DK / 16 / DS, OT = 2 / DS;          // tiles that are a wavefront's own
    constexpr int NBUF = NPI == 3 && DK == 128 ? 1 : 2;
    extern __shared__ __align__(16) char lds_raw[];
    using Lds = AdjLds<NPI, NP, DK, NBUF, DS>;
    Lds &lds = *reinterpret_cast<Lds *>(lds_raw);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row16 = lane & 15, g4 = lane >> 4;
    DeltaUnit un;
    if (!delta_unit(p, AGG ? p.nseg - 1 : p.nseg, un)) return;
    const int h = un.h, hk = h / (p.Hv / p.Hk), b = un.b, seg = AGG ? un.seg + 1 : un.seg;
    const DeltaSeq sq = delta_seq(p, b);
    const int dh = DS == 2 ? wave & 1 : 0, d0 = dh * (DK / 2), first = DS == 2 ? dh : 0;
    const int c0 = (un.group * CW + wave / DS) * 16, n0 = c0 + row16;
    const bool col_in = n0 < p.dv, mine = c0 < p.dvp;
    const int64_t nchunk = (sq.len + 31) / 32, ch0 = p.nseg > 1 ? (int64_t)seg * p.seg_chunks : 0;
    const int64_t ch1 = p.nseg > 1 && nchunk > ch0 + p.seg_chunks ? ch0 + p.seg_chunks : nchunk;
    if (ch0 >= nchunk && seg > 0) return;
    const int64_t head = (int64_t)b * p.Hv + h;
    const NegId neg = neg_id();

    f32x4 S[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = d0 + 16 * m + 4 * g4 + r;
            if (AGG) S[m][r] = d == n0 - p.dvp ? 1.0f : 0.0f;
            else if (ch1 < nchunk) S[m][r] = mine ? p.entry[((head * p.nseg + seg) * DK + d) * p.dvp + n0] : 0.0f;
            else S[m][r] = p.ds_last && col_in && d < p.dk ? p.ds_last[(head * p.dk + d) * p.dv + n0] : 0.0f;
        }

    const uint16_t *kp = p.k.p + sq.ib * p.k.sb + sq.at * p.k.sl + hk * p.k.sh, *qp = p.q.p + sq.ib * p.q.sb + sq.at * p.q.sl + hk * p.q.sh;
    const uint16_t *dp = p.dout.p + sq.ib * p.dout.sb + sq.at * p.dout.sl + h * p.dout.sh;

    constexpr int QUADS = 8 * (DK / 4), MATS = chunk_words(NP, NP) / 8;
    constexpr int IQ = (QUADS + NT - 1) / NT, IM = (MATS + NT - 1) / NT;
    struct Stage {
        uint2 k[IQ][NPI][4], q[IQ][NPI][4];
        uint4 m[IM];
        uint16_t d[NPI][2][4];
    };
    const uint32_t krow = (uint32_t)p.k.sl * 2, qrow = (uint32_t)p.q.sl * 2, drow = (uint32_t)p.dout.sl * 2;
    const uint32_t doff = mine ? 4 * g4 * drow + n0 * 2u : kOutside;
    auto fetch = [&](int64_t ch, Stage &st) __attribute__((always_inline)) {
        const bool in = ch >= ch0 && ch < ch1;
        const int64_t t0 = in ? ch * 32 : 0, last = (sq.len - t0 < 32 ? sq.len - t0 : 32) - 1;
#pragma unroll
        for (int pl = 0; pl < NPI; ++pl) {
            const Buffer kb = buffer_of(kp + pl * p.k.plane + t0 * p.k.sl, in ? last * krow + 2 * DK : 0);
            const Buffer qb = buffer_of(qp + pl * p.q.plane + t0 * p.q.sl, in ? last * qrow + 2 * DK : 0);
            const Buffer db = buffer_of(dp + pl * p.dout.plane + t0 * p.dout.sl, in ? last * drow + 2 * p.dvp : 0);
#pragma unroll
            for (int x = 0; x < IQ; ++x) {
                const int i = tid + x * NT, tq = i / (DK / 4), dq = i % (DK / 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    st.k[x][pl][e] = buffer_load8(kb, QUADS % NT && i >= QUADS ? kOutside : (4 * tq + e) * krow + 8 * dq);
                    st.q[x][pl][e] = buffer_load8(qb, QUADS % NT && i >= QUADS ? kOutside : (4 * tq + e) * qrow + 8 * dq);
                }
            }
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) buffer_load(db, doff + (16 * m + r) * drow, st.d[pl][m][r]);
        }
        const int64_t mat = in ? ((sq.slot + (ch >> 1)) * p.Hv + h) * 2 + (ch & 1) : 0;
        const Buffer mb = buffer_of(p.mats_adj + mat * (MATS * 8), in ? MATS * 16 : 0);
#pragma unroll
        for (int x = 0; x < IM; ++x) st.m[x] = buffer_load16(mb, (tid + x * NT) * 16);
    };
    auto put = [&](typename Lds::Buf &B, const Stage &st) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < IQ; ++x) {
            const int i = tid + x * NT, tq = i / (DK / 4), dq = i % (DK / 4);
            if (QUADS % NT && i >= QUADS) continue;
            const int col = (dq >> 3) * 32 + quad_place(dq & 7), place = quad_place(tq);
#pragma unroll
            for (int pl = 0; pl < NPI; ++pl) {
                uint2 kc[4], qc[4];
                transpose_quad(st.k[x][pl], kc);
                transpose_quad(st.q[x][pl], qc);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    *reinterpret_cast<uint2 *>(&B.k[pl][4 * tq + e][col]) = st.k[x][pl][e];
                    *reinterpret_cast<uint2 *>(&B.kt[pl][4 * dq + e][turned(4 * dq, place)]) = kc[e];
                    *reinterpret_cast<uint2 *>(&B.qt[pl][4 * dq + e][turned(4 * dq, place)]) = qc[e];
                }
            }
        }
        uint4 *mats = reinterpret_cast<uint4 *>(&B.th[0][0]);
#pragma unroll
        for (int x = 0; x < IM; ++x)
            if (MATS % NT == 0 || tid + x * NT < MATS) mats[tid + x * NT] = st.m[x];
    };

    auto step = [&](int64_t ch, Stage &cur, Stage &next) __attribute__((always_inline)) {
        const typename Lds::Buf &B = lds.buf[NBUF == 2 ? ch & 1 : 0];
        const int64_t t0 = ch * 32;
        const int n = (int)(sq.len - t0 < 32 ? sq.len - t0 : 32);
        Frag dof[NPI];
        f32x4 dO[2] = {};
#pragma unroll
        for (int pl = 0; pl < NPI; ++pl) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) dO[m][r] += load_io(&cur.d[pl][m][r]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                dof[pl].u[e] = (uint32_t)cur.d[pl][e >> 1][2 * (e & 1)] | (uint32_t)cur.d[pl][e >> 1][2 * (e & 1) + 1] << 16;
        }
        fetch(ch - (DEEP ? 2 : 1), cur);

        const int64_t sh = (sq.slot + (ch >> 1)) * p.Hv + h;
        const int G = p.dvp / 16;
        float *units = p.dunits + sh * 6 * G + c0 / 16;
        if (!AGG && ((ch & 1) || ch == nchunk - 1) && mine)
            save_state<EXACT, DK>(S, p.dstates, (sh * p.dvp + n0) * DK + d0 + 4 * g4, units + dh * G, G);
        constexpr bool EARLY = NPI == 1;                    // operands read well before they are used
        Frag kf[EARLY ? KS : 1][2][NPI], tf[2][NP], ktf[EARLY ? MT : 1][NPI], qtf[EARLY ? MT : 1][NPI], af[2][NP], tt[OT][NP];
        f32x4 gam[2], be[2], en[2];
        if constexpr (EARLY)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int m = 0; m < 2; ++m) kf[ks][m][0].v = *reinterpret_cast<const uint4 *>(&B.k[0][16 * m + row16][d0 + 32 * ks + 8 * g4]);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            en[m] = *reinterpret_cast<const f32x4 *>(&B.scal[32 + 16 * m + 4 * g4]);
#pragma unroll
            for (int i = 0; i < NP; ++i) af[m][i] = m ? half_tile<true>(B.ah[i], lane) : whole_tile(B.aw[i], lane);
#pragma unroll
            for (int i = 0; i < NP; ++i) tf[m][i] = m ? half_tile<true>(B.th[i], lane) : whole_tile(B.tw[i], lane);
        }
        if constexpr (EARLY) reads_first();
        // dU
        f32x4 X[2] = {}, Y[2] = {};
#pragma unroll
        for (int m = 0; m < 2; ++m) Y[m] = mm(af[m], dof, Y[m]);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            Frag s[NP];
            split_tiles<NP>(S[2 * ks], S[2 * ks + 1], s, neg);
            const int at = EARLY ? ks : 0;
            if constexpr (!EARLY)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int i = 0; i < NPI; ++i) kf[0][m][i].v = *reinterpret_cast<const uint4 *>(&B.k[i][16 * m + row16][d0 + 32 * ks + 8 * g4]);
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < NPI; ++j)
#pragma unroll
                    for (int m = 0; m < 2; ++m)
                        if (i + j < NP) X[m] = mfma(kf[at][m][j], s[i], X[m]);
        }
        if constexpr (DS == 2) {
            lds.halves[2 * wave][lane] = X[0];
            lds.halves[2 * wave + 1][lane] = X[1];
            lds_barrier();
            X[0] += lds.halves[2 * (wave ^ 1)][lane];
            X[1] += lds.halves[2 * (wave ^ 1) + 1][lane];
        }
        if constexpr (!AGG)
#pragma unroll
            for (int m = 0; m < OT; ++m)
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    if constexpr (DS == 2) triangle_tile<true>(dh == 1, B.th[i], B.tw[i], lane, tt[m][i]);
                    else tt[m][i] = tf[m][i];
                }
        if constexpr (EARLY)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                ktf[m][0].v = *reinterpret_cast<const uint4 *>(&B.kt[0][d0 + 16 * m + row16][turned(d0 + 16 * m, 8 * g4)]);
                qtf[m][0].v = *reinterpret_cast<const uint4 *>(&B.qt[0][d0 + 16 * m + row16][turned(d0 + 16 * m, 8 * g4)]);
            }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            be[m] = *reinterpret_cast<const f32x4 *>(&B.scal[64 + 16 * m + 4 * g4]);
            gam[m] = *reinterpret_cast<const f32x4 *>(&B.scal[16 * m + 4 * g4]);
        }
        const float gend = B.scal[31];
        if constexpr (EARLY) reads_first();
        // scale exp(G) dO, which waits for nothing, into dS0 first
        f32x4 W[2];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) { W[m][r] = p.scale * gam[m][r] * dO[m][r]; X[m][r] = __builtin_fmaf(en[m][r], X[m][r], Y[m][r]); }
        Frag uf[NP], wf[NP];
        split_tiles<NP>(X[0], X[1], uf, neg);
        split_tiles<NP>(W[0], W[1], wf, neg);
        f32x4 Z[2] = {}, Zt[OT] = {};
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < NP; ++j)
                if (i + j < NP)
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        Z[m] = mfma(tf[m][i], uf[j], Z[m]);
                        if (!AGG && m < OT) Zt[m] = mfma(uf[j], tt[m][i], Zt[m]);                      // a step to a lane, for wide stores
                    }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[m][r] *= gend;
        if constexpr (EARLY) mm_each(qtf, wf, S);
        else
#pragma unroll
            for (int m = 0; m < MT; ++m) {
#pragma unroll
                for (int i = 0; i < NPI; ++i) qtf[0][i].v = *reinterpret_cast<const uint4 *>(&B.qt[i][d0 + 16 * m + row16][turned(d0 + 16 * m, 8 * g4)]);
                S[m] = mm(qtf[0], wf, S[m]);
            }
        f32x4 R[2];                                         // -exp(G) beta z
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) R[m][r] = -gam[m][r] * be[m][r] * Z[m][r];
        Frag rf[NP];
        split_tiles<NP>(R[0], R[1], rf, neg);
        if constexpr (EARLY) mm_each(ktf, rf, S);
        else
#pragma unroll
            for (int m = 0; m < MT; ++m) {
#pragma unroll
                for (int i = 0; i < NPI; ++i) ktf[0][i].v = *reinterpret_cast<const uint4 *>(&B.kt[i][d0 + 16 * m + row16][turned(d0 + 16 * m, 8 * g4)]);
                S[m] = mm(ktf[0], rf, S[m]);
            }
        if (!AGG && mine)
            save_rows<EXACT>(Zt, p.z, ((sq.row + t0 + 16 * first + row16) * p.Hv + h) * p.dvp + c0 + 4 * g4, (int64_t)16 * p.Hv * p.dvp,
                             n - 16 * first, units + (2 + 2 * (ch & 1) + first) * G, G);
        if (NBUF == 1) lds_barrier();
        put(lds.buf[NBUF == 2 ? (ch - 1) & 1 : 0], next);
        lds_barrier();
    };
    Stage one;
    fetch(ch1 - 1, one);
    put(lds.buf[NBUF == 2 ? (ch1 - 1) & 1 : 0], one);
    if constexpr (DEEP) {
        Stage two;
        fetch(ch1 - 2, two);
        lds_barrier();
        for (int64_t ch = ch1 - 1; ch >= ch0;) {
            step(ch, one, two);
            if (--ch < ch0) break;
            step(ch, two, one);
            --ch;
        }
    } else {
        lds_barrier();
        for (int64_t ch = ch1 - 1; ch >= ch0; --ch) step(ch, one, one);
    }
    if constexpr (AGG) {
        if (mine) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) p.entry[((head * p.nseg + un.seg) * DK + 16 * m + 4 * g4 + r) * p.dvp + n0] = S[m][r];
        } else if (c0 < p.dvp + DK) store_trans<NP, DK>(S, p.trans + (head * (p.nseg - 1) + un.seg) * NP * DK * DK, n0 - p.dvp, g4);
    } else if (p.ds0 && col_in && ch0 == 0)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = d0 + 16 * m + 4 * g4 + r;
                if (d < p.dk) p.ds0[(head * p.dk + d) * p.dv + n0] = S[m][r];
            }
}

// ---------------------------------------------------------------- the gradients of a slot
// A workgroup takes the 64 steps of a slot and a value head (where value heads share a key head, k_delta_share adds up their parts of dQ and dK); a
// wavefront owns 16 of the steps, one to a lane of each group of 16, and every product is arranged so that its results lie a step to a lane: gates are a number to a lane, F and H go from one product's
// results into the next one's operand without leaving the lane, and rows of dQ and dK come out four neighbouring elements at a time.  Both
// orientations of F and H are computed (one as products with the rows of others, one the other way round), which costs less than turning them.
// The columns of v come through LDS 32 at a time (rows of dO, E, Z and of both states, the next ones under way meanwhile), then K and Q, as rows
// and turned, in the same place: 72 KB for dk = 128 in bfloat16, two workgroups a compute unit.  Bound by memory: 4 x 4096 steps of 16 heads of
// 128 x 128, 805 MB in 227 us (3.5 TB/s; a copy would take 152); with what is kept in float32 1.21 GB in 466, one workgroup a compute unit (98 KB).
template <int NPI, int NPE, int DK> struct GradLds {
    static constexpr int ROWS = NPI == 3 ? 0 : 1;
    union {
        struct { uint16_t e[NPE][64][40], z[NPE][64][40], d[NPI][64][40], s0[NPE][DK][40], s1[NPE][DK][40]; } v;
        struct { uint16_t kt[NPI][DK][72], qt[NPI][DK][72], kr[ROWS + 1][ROWS ? 64 : 1][DK + 8]; } k;      // kr: rows of K and of Q
    };
    double G[64];
    float beta[64], dG[64], ends[4], dots[4], most[4];
};

// Rows of a packed axis outside every sequence, zeros in the gradients: there are at most as many as slots have steps, and a slot's workgroup clears the 64 of
// them that come at its place in their order.
template <class IO> __device__ void clear_outside(const DeltaParams &p, int64_t slot, int h, int hk) {
    const int64_t lo = delta_clamp(p.cu[0], p.L), end = delta_clamp(p.cu[p.B], p.L), hi = end > lo ? end : lo, count = lo + (p.L - hi) - slot * kDeltaSlot;
    const bool keys = h % (p.Hv / p.Hk) == 0;
    for (int i = threadIdx.x >> 6; i < (count < kDeltaSlot ? count : kDeltaSlot); i += 4) {
        const int64_t at = slot * kDeltaSlot + i, row = at < lo ? at : hi + (at - lo);
        const int lane = threadIdx.x & 63;
        for (int c = lane; c < p.dv; c += 64) store_io(reinterpret_cast<IO *>(p.dvv) + (row * p.Hv + h) * p.dv + c, 0.0f);
        if (keys)
            for (int c = lane; c < p.dk; c += 64) {
                store_io(reinterpret_cast<IO *>(p.dq) + (row * p.Hk + hk) * p.dk + c, 0.0f);
                store_io(reinterpret_cast<IO *>(p.dkk) + (row * p.Hk + hk) * p.dk + c, 0.0f);
            }
        if (lane == 0)
            for (void *gate : {p.dg, p.dbeta}) {
                if (p.gate_io && p.io) store_io(reinterpret_cast<uint16_t *>(gate) + row * p.Hv + h, 0.0f);
                else store_io(reinterpret_cast<float *>(gate) + row * p.Hv + h, 0.0f);
            }
    }
}

// NPI: planes of an input, NPE: of E, Z and the states, which lie in memory as float32 (3) or as 16-bit floating point with a power of two a block (1; dO too
// is brought to that here).
template <class IO, int NPI, int NPE, int DK>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(NPE == 1 ? 2 : 1, 2))) void k_delta_grads(const DeltaParams p) {
    constexpr int KS = DK / 32, MT = DK / 16, NPF = NPI == 3 ? 3 : 2;
    constexpr bool UNITS = NPE == 1;
    using Kept = std::conditional_t<UNITS, uint16_t, float>;
    constexpr int KE = sizeof(Kept) / 2;
    constexpr bool ROWS = NPI == 1;                         // rows of K and Q in LDS too; else from memory
    extern __shared__ __align__(16) char lds_raw[];
    GradLds<NPI, NPE, DK> &lds = *reinterpret_cast<GradLds<NPI, NPE, DK> *>(lds_raw);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row16 = lane & 15, g4 = lane >> 4;
    const int64_t slot = blockIdx.x / (unsigned)p.Hv;
    const int h = (int)(blockIdx.x - slot * p.Hv), hk = h / (p.Hv / p.Hk);
    DeltaSeq sq;
    int64_t t0;
    int b;
    const int n = delta_slot(p, slot, sq, t0, b);
    if (p.cu) clear_outside<IO>(p, slot, h, hk);
    if (n == 0) return;
    const int64_t at = sq.at + t0, row0 = sq.row + t0, rows = (int64_t)(p.cu ? 1 : p.B) * p.L;
    const uint16_t *kp = p.k.p + sq.ib * p.k.sb + at * p.k.sl + hk * p.k.sh, *qp = p.q.p + sq.ib * p.q.sb + at * p.q.sl + hk * p.q.sh;
    const uint32_t krow = (uint32_t)p.k.sl * 2, qrow = (uint32_t)p.q.sl * 2, drow = (uint32_t)p.dout.sl * 2, erow = (uint32_t)p.Hv * p.dvp * (uint32_t)sizeof(Kept);
    const int own = 16 * wave + row16;
    const bool own_in = own < n;

    f32x4 dq[MT], dk[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) dq[m] = dk[m] = f32x4{};

    const uint16_t *dp = p.dout.p + sq.ib * p.dout.sb + at * p.dout.sl + h * p.dout.sh;
    // E's and Z's rows: in float32 those of the wavefront's 16 steps (all 64 of a slot may span more than a descriptor does)
    const int from = UNITS ? 0 : 16 * wave, to = UNITS || n < from + 16 ? n : from + 16;
    const int64_t first = ((row0 + from) * p.Hv + h) * p.dvp;
    const int64_t ebytes = to > from ? (to - from - 1) * (int64_t)erow + p.dvp * (int64_t)sizeof(Kept) : 0;
    const Kept *ep = reinterpret_cast<const Kept *>(p.err) + first, *zp = reinterpret_cast<const Kept *>(p.z) + first;
    const Kept *s0p = reinterpret_cast<const Kept *>(p.states) + (slot * p.Hv + h) * DK * p.dvp;
    const Kept *s1p = reinterpret_cast<const Kept *>(p.dstates) + (slot * p.Hv + h) * DK * p.dvp;
    const int ksv = p.dvp / 32;

    // 32 columns of v on their way: a thread brings eight elements of a row of dO (of each plane), E and Z, and of the states, which lie a column of v to
    // a row, four rows by four elements (the first 2 DK threads)
    uint4 ereg[KE], zreg[KE], dreg[NPI];
    uint2 areg[KE][4], breg[KE][4];
    const int tr = tid >> 2, tc = (tid & 3) * 16, sq4 = tid / (DK / 4), sd4 = tid % (DK / 4);
    auto fetch = [&](int ks) {
#pragma unroll
        for (int i = 0; i < KE; ++i) {
            const uint32_t off = (UNITS ? tr : tr & 15) * erow + KE * (64 * ks + tc) + 16 * i;
            ereg[i] = buffer_load16(buffer_of(ep, ebytes), off);
            zreg[i] = buffer_load16(buffer_of(zp, ebytes), off);
        }
#pragma unroll
        for (int i = 0; i < NPI; ++i)
            dreg[i] = buffer_load16(buffer_of(dp + i * p.dout.plane, (int64_t)(n - 1) * drow + 2 * p.dvp), tr * drow + 64 * ks + tc);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const uint32_t off = tid < 2 * DK ? (uint32_t)(((32 * ks + 4 * sq4 + x) * DK + 4 * sd4) * (int)sizeof(Kept)) : kOutside;
            const Buffer ab = buffer_of(s0p, DK * p.dvp * (int)sizeof(Kept)), bb = buffer_of(s1p, DK * p.dvp * (int)sizeof(Kept));
            if constexpr (UNITS) { areg[0][x] = buffer_load8(ab, off); breg[0][x] = buffer_load8(bb, off); }
            else {
                const uint4 a = buffer_load16(ab, off), b = buffer_load16(bb, off);
                areg[0][x] = make_uint2(a.x, a.y); areg[KE - 1][x] = make_uint2(a.z, a.w);
                breg[0][x] = make_uint2(b.x, b.y); breg[KE - 1][x] = make_uint2(b.z, b.w);
            }
        }
    };
    // the blocks' units: a slot's largest of each kind, and the others' share of it
    float zunit = 1.0f;
    float uE = 1.0f, uZ = 1.0f, uD = 1.0f, uA = 1.0f, uB = 1.0f, rE = 1.0f, rZ = 1.0f, rA = 1.0f, rB = 1.0f;
    const int G = p.dvp / 16;
    if constexpr (UNITS) {
        const float *fu = p.units + (slot * p.Hv + h) * 6 * G, *bu = p.dunits + (slot * p.Hv + h) * 6 * G;
        const int in = (n > 32 ? 4 : 2) * G;
        buffer_load(buffer_of(fu, 8 * G), 4 * lane, rA);
        buffer_load(buffer_of(fu + 2 * G, 4 * in), 4 * lane, rE);
        buffer_load(buffer_of(bu, 8 * G), 4 * lane, rB);
        buffer_load(buffer_of(bu + 2 * G, 4 * in), 4 * lane, rZ);
    }
    fetch(0);
    if constexpr (UNITS) {
        // the largest of dO, whose rows are read once more for it
        const Buffer db = buffer_of(dp, (int64_t)(n - 1) * drow + 2 * p.dvp);
        uint32_t most = 0x00800080u;
        for (int ks = 0; ks < ksv; ks += 4) {
            uint4 d[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) d[x] = buffer_load16(db, ks + x < ksv ? tr * drow + 64 * (ks + x) + tc : kOutside);
#pragma unroll
            for (int x = 0; x < 4; ++x) most = max_finite(max_finite(max_finite(max_finite(most, d[x].x), d[x].y), d[x].z), d[x].w);
        }
        most -= 0x00800080u;
        most = most << 16 > (most & 0x7fff0000u) ? most << 16 : most & 0x7fff0000u;
        const float whole = wave_max(__uint_as_float(most));
        if (lane == 0) lds.most[wave] = whole;
        uA = wave_max(rA); uE = wave_max(rE); uB = wave_max(rB); uZ = wave_max(rZ);
        zunit = rZ;
        rA *= inverse_unit(uA); rE *= inverse_unit(uE); rB *= inverse_unit(uB); rZ *= inverse_unit(uZ);
    }
    if (wave == 0) {
        const bool in = lane < n;
        const int64_t t = at + (in ? lane : 0);
        const float gr = load_gate(p.g, sq.ib * p.g_sb + t * p.g_sl + h * p.g_sh, p.io, p.gate_io);
        const float be = load_gate(p.beta, sq.ib * p.be_sb + t * p.be_sl + h * p.be_sh, p.io, p.gate_io);
        double G = in ? gate_log(gr) : 0.0;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const double o = __shfl_up(G, m, 64);
            if (lane >= m) G += o;
        }
        lds.G[lane] = G;
        lds.beta[lane] = in ? be : 0.0f;
    }

    // Products with 16 others' steps at a time: earlier ones wrote what this wavefront's read (e_j . dO_own, e_j . z_own), later ones read what it wrote
    // (dO_i . e_own, z_i . e_own); its own 16 are both, the second kind of them apart.
    f32x4 P1[4] = {}, P2[4] = {}, P1own = {}, P2own = {};
    f32x4 qs[MT], kr[MT], kw[MT];                                // S0 dO, S0 z, dS1 e of the lane's step
#pragma unroll
    for (int m = 0; m < MT; ++m) qs[m] = kr[m] = kw[m] = f32x4{};
    auto mv = [](const auto &a, const auto &b, f32x4 c) __attribute__((always_inline)) -> f32x4 {
        if constexpr (UNITS) return mfma16(a[0], b[0], c);
        else return mm(a, b, c);
    };
    float dbeta = 0.0f, sdot = 0.0f, bown = 0.0f;
    // K and Q of the slot, 16 quads of steps by DK / 4 quads of columns, under way during the last 32 columns
    constexpr int IQ = DK / 64;
    uint2 kw4[NPI][IQ * 4], qw4[NPI][IQ * 4];
    auto fetch_kq = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int pl = 0; pl < NPI; ++pl) {
            const Buffer kb = buffer_of(kp + pl * p.k.plane, (int64_t)(n - 1) * krow + 2 * DK), qb = buffer_of(qp + pl * p.q.plane, (int64_t)(n - 1) * qrow + 2 * DK);
#pragma unroll
            for (int x = 0; x < IQ; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = tid + 256 * x, tq = i / (DK / 4), dc = i % (DK / 4);
                    kw4[pl][4 * x + e] = buffer_load8(kb, (4 * tq + e) * krow + 8 * dc);
                    qw4[pl][4 * x + e] = buffer_load8(qb, (4 * tq + e) * qrow + 8 * dc);
                }
        }
    };
    auto columns = [&](int ks, auto last) __attribute__((always_inline)) {
        lds_barrier();                                  // what was there in LDS has been read
        auto &L = lds.v;
        if constexpr (UNITS) uD = block_unit(fmaxf(fmaxf(lds.most[0], lds.most[1]), fmaxf(lds.most[2], lds.most[3])));
        uint2 pE = {}, pZ = {}, pA = {}, pB = {};
        const int ge = 2 * ks + ((tid >> 1) & 1) + (tr >> 4) * G;
        // Brought to the slot's units, where 11 bits are left of numbers down to 2^-29 of the slot's largest and nothing below 2^-39 (a sum in float32 has
        // lost such a term by 2^-24).  The power itself may be below what 16 bits hold: two factors, of 2^-14 and 2^-24 at least.
        if constexpr (UNITS) {
            const int gs = 2 * ks + (sq4 >> 2 & 1) + (8 * sd4 >= DK ? G : 0);
            auto factors = [](float f) __attribute__((always_inline)) -> uint2 {
                const float a = fmaxf(f, 0x1p-14f), b = fminf(f * 0x1p14f, 1.0f);
                return make_uint2(pack_f16(a, a), pack_f16(b, b));
            };
            pE = factors(__shfl(rE, ge, 64)); pZ = factors(__shfl(rZ, ge, 64)); pA = factors(__shfl(rA, gs, 64)); pB = factors(__shfl(rB, gs, 64));
        }
        auto times = [&](uint32_t x, uint2 f) __attribute__((always_inline)) -> uint32_t {
            return UNITS ? __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, x) * __builtin_bit_cast(f16x2, f.x) * __builtin_bit_cast(f16x2, f.y)) : x;
        };
        // dV = beta z, a row's eight columns a thread: of 16 bits as they lie in memory, with their own block's unit
        auto put_dv = [&](int row, int column, const f32x4 (&z)[2], float f) __attribute__((always_inline)) {
            if (row >= n) return;
            IO *to = reinterpret_cast<IO *>(p.dvv) + ((row0 + row) * p.Hv + h) * p.dv + column;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const f32x4 v = z[x] * f;
                if (p.o_vec && column + 4 * x + 4 <= p.dv) store4(to + 4 * x, v);
                else
#pragma unroll
                    for (int r = 0; r < 4; ++r) if (column + 4 * x + r < p.dv) store_io(to + 4 * x + r, v[r]);
            }
        };
        if constexpr (UNITS) {
            Frag z;
            z.v = zreg[0];
            f32x4 zs[2];
#pragma unroll
            for (int x = 0; x < 8; ++x) zs[x >> 2][x & 3] = (float)z.h16[x];
            put_dv(tr, 32 * ks + 8 * (tid & 3), zs, lds.beta[tr] * __shfl(zunit, ge, 64));
        }
        if constexpr (UNITS) {
            const uint4 e = ereg[0], z = zreg[0];
            *reinterpret_cast<uint4 *>(&L.e[0][tr][tc / 2]) = make_uint4(times(e.x, pE), times(e.y, pE), times(e.z, pE), times(e.w, pE));
            *reinterpret_cast<uint4 *>(&L.z[0][tr][tc / 2]) = make_uint4(times(z.x, pZ), times(z.y, pZ), times(z.z, pZ), times(z.w, pZ));
        } else {
            auto planes = [](const uint4 &lo, const uint4 &hi, uint32_t (&w)[4][NPE]) __attribute__((always_inline)) {
                split2<NPE>(__uint_as_float(lo.x), __uint_as_float(lo.y), w[0]);
                split2<NPE>(__uint_as_float(lo.z), __uint_as_float(lo.w), w[1]);
                split2<NPE>(__uint_as_float(hi.x), __uint_as_float(hi.y), w[2]);
                split2<NPE>(__uint_as_float(hi.z), __uint_as_float(hi.w), w[3]);
            };
            uint32_t e[4][NPE], z[4][NPE];
            planes(ereg[0], ereg[KE - 1], e);
            planes(zreg[0], zreg[KE - 1], z);
#pragma unroll
            for (int i = 0; i < NPE; ++i) {
                *reinterpret_cast<uint4 *>(&L.e[i][tr][tc / 2]) = make_uint4(e[0][i], e[1][i], e[2][i], e[3][i]);
                *reinterpret_cast<uint4 *>(&L.z[i][tr][tc / 2]) = make_uint4(z[0][i], z[1][i], z[2][i], z[3][i]);
            }
        }
#pragma unroll
        for (int i = 0; i < NPI; ++i) {
            uint4 d = dreg[i];
            if constexpr (UNITS) {
                const float inv = inverse_unit(uD);
                auto conv = [&](uint32_t x) __attribute__((always_inline)) { return pack_f16(__uint_as_float(x << 16) * inv, hi_part(__uint_as_float(x)) * inv); };
                d = make_uint4(conv(d.x), conv(d.y), conv(d.z), conv(d.w));
            }
            *reinterpret_cast<uint4 *>(&L.d[i][tr][tc / 2]) = d;
        }
        uint2 ap[NPE][4], bp[NPE][4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if constexpr (UNITS) { ap[0][x] = areg[0][x]; bp[0][x] = breg[0][x]; }
            else {
                uint32_t a[2][NPE], b[2][NPE];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    split2<NPE>(__uint_as_float(areg[y * (KE - 1)][x].x), __uint_as_float(areg[y * (KE - 1)][x].y), a[y]);
                    split2<NPE>(__uint_as_float(breg[y * (KE - 1)][x].x), __uint_as_float(breg[y * (KE - 1)][x].y), b[y]);
                }
#pragma unroll
                for (int i = 0; i < NPE; ++i) { ap[i][x] = make_uint2(a[0][i], a[1][i]); bp[i][x] = make_uint2(b[0][i], b[1][i]); }
            }
        }
#pragma unroll
        for (int i = 0; i < NPE; ++i)
            if (tid < 2 * DK) {
                uint2 c[4], d[4];
                transpose_quad(ap[i], c);
                transpose_quad(bp[i], d);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    *reinterpret_cast<uint2 *>(&L.s0[i][4 * sd4 + x][turned(4 * sd4, 4 * sq4)]) = make_uint2(times(c[x].x, pA), times(c[x].y, pA));
                    *reinterpret_cast<uint2 *>(&L.s1[i][4 * sd4 + x][turned(4 * sd4, 4 * sq4)]) = make_uint2(times(d[x].x, pB), times(d[x].y, pB));
                }
            }
        if constexpr (last) fetch_kq();
        else fetch(ks + 1);
        lds_barrier();
        bown = lds.beta[own];
        Frag dO[NPI], e[NPE], z[NPE];
#pragma unroll
        for (int i = 0; i < NPI; ++i) dO[i].v = *reinterpret_cast<const uint4 *>(&L.d[i][own][8 * g4]);
#pragma unroll
        for (int i = 0; i < NPE; ++i) {
            e[i].v = *reinterpret_cast<const uint4 *>(&L.e[i][own][8 * g4]);
            z[i].v = *reinterpret_cast<const uint4 *>(&L.z[i][own][8 * g4]);
        }
        // the states' products, and <S0, dS1> of a quarter of their rows
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            Frag s0[NPE], s1[NPE];
#pragma unroll
            for (int i = 0; i < NPE; ++i) {
                s0[i].v = *reinterpret_cast<const uint4 *>(&L.s0[i][16 * m + row16][turned(16 * m, 8 * g4)]);
                s1[i].v = *reinterpret_cast<const uint4 *>(&L.s1[i][16 * m + row16][turned(16 * m, 8 * g4)]);
            }
            qs[m] = mv(s0, dO, qs[m]);
            kr[m] = mv(s0, z, kr[m]);
            kw[m] = mv(s1, e, kw[m]);
            if (m & 1) reads_first();
        }
#pragma unroll
        for (int y = 0; y < MT / 4; ++y) {
            const int m = 4 * y + wave;
            Frag s0[NPE], s1[NPE];
#pragma unroll
            for (int i = 0; i < NPE; ++i) {
                s0[i].v = *reinterpret_cast<const uint4 *>(&L.s0[i][16 * m + row16][turned(16 * m, 8 * g4)]);
                s1[i].v = *reinterpret_cast<const uint4 *>(&L.s1[i][16 * m + row16][turned(16 * m, 8 * g4)]);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if constexpr (UNITS) sdot = __builtin_amdgcn_fdot2(s0[0].p16[x], s1[0].p16[x], sdot, false);
                else {
                    float al = 0.0f, ah = 0.0f, cl = 0.0f, chh = 0.0f;
#pragma unroll
                    for (int i = NPE - 1; i >= 0; --i) {
                        al += __uint_as_float(s1[i].u[x] << 16); ah += hi_part(__uint_as_float(s1[i].u[x]));
                        cl += __uint_as_float(s0[i].u[x] << 16); chh += hi_part(__uint_as_float(s0[i].u[x]));
                    }
                    sdot = __builtin_fmaf(al, cl, __builtin_fmaf(ah, chh, sdot));
                }
            }
        }
        // with the other steps
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            Frag r1[NPE], r2[NPE], c1[NPE], c2[NPE];
#pragma unroll
            for (int i = 0; i < NPE; ++i) {
                const int j = i < NPI ? i : 0;              // (of one plane each product of E with dO takes it)
                r1[i].v = *reinterpret_cast<const uint4 *>(&(m <= wave ? L.e : L.d)[NPI == NPE || m <= wave ? i : j][16 * m + row16][8 * g4]);
                r2[i].v = *reinterpret_cast<const uint4 *>(&(m <= wave ? L.e : L.z)[i][16 * m + row16][8 * g4]);
#pragma unroll
                for (int x = 0; x < 4; ++x) { c1[i].u[x] = m <= wave ? dO[j].u[x] : e[i].u[x]; c2[i].u[x] = m <= wave ? z[i].u[x] : e[i].u[x]; }
            }
            if constexpr (NPI == NPE) P1[m] = mv(r1, c1, P1[m]);
            else
#pragma unroll
                for (int i = 0; i < NPE; ++i) P1[m] = mfma(r1[i], c1[i], P1[m]);
            P2[m] = mv(r2, c2, P2[m]);
        }
        P1own = mv(dO, e, P1own);
        P2own = mv(z, e, P2own);
        // dbeta = z . e
        if constexpr (UNITS) {
#pragma unroll
            for (int x = 0; x < 4; ++x) dbeta = __builtin_amdgcn_fdot2(z[0].p16[x], e[0].p16[x], dbeta, false);
        } else {
            f32x4 zs[2] = {}, es[2] = {};
#pragma unroll
            for (int x = 0; x < 8; ++x)
#pragma unroll
                for (int i = NPE - 1; i >= 0; --i) {
                    zs[x >> 2][x & 3] += __uint_as_float(x & 1 ? z[i].u[x >> 1] & 0xffff0000u : z[i].u[x >> 1] << 16);
                    es[x >> 2][x & 3] += __uint_as_float(x & 1 ? e[i].u[x >> 1] & 0xffff0000u : e[i].u[x >> 1] << 16);
                }
#pragma unroll
            for (int x = 0; x < 8; ++x) dbeta = __builtin_fmaf(zs[x >> 2][x & 3], es[x >> 2][x & 3], dbeta);
            put_dv(own, 32 * ks + 8 * g4, zs, bown);
        }
    };
#pragma unroll 1
    for (int ks = 0; ks < ksv - 1; ++ks) columns(ks, std::false_type{});
    columns(ksv - 1, std::true_type{});
    if constexpr (UNITS) { dbeta = dbeta * uZ * uE; sdot = sdot * uA * uB; }
    const double Gown = lds.G[own];
    const float gam = __expf((float)Gown), en = __expf((float)(lds.G[63] - Gown));

    // K and Q into LDS, turned, and as rows
    lds_barrier();
#pragma unroll
    for (int pl = 0; pl < NPI; ++pl)
#pragma unroll
        for (int x = 0; x < IQ; ++x) {
            const int i = tid + 256 * x, tq = i / (DK / 4), dc = i % (DK / 4), place = (tq >> 3) * 32 + quad_place(tq & 7);
            uint2 w[4], u[4], c[4], d[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) { w[e] = kw4[pl][4 * x + e]; u[e] = qw4[pl][4 * x + e]; }
            transpose_quad(w, c);
            transpose_quad(u, d);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                *reinterpret_cast<uint2 *>(&lds.k.kt[pl][4 * dc + e][turned(4 * dc, place)]) = c[e];
                *reinterpret_cast<uint2 *>(&lds.k.qt[pl][4 * dc + e][turned(4 * dc, place)]) = d[e];
                if constexpr (ROWS) {
                    *reinterpret_cast<uint2 *>(&lds.k.kr[0][4 * tq + e][4 * dc]) = w[e];
                    *reinterpret_cast<uint2 *>(&lds.k.kr[1][4 * tq + e][4 * dc]) = u[e];
                }
            }
        }
    lds_barrier();
    // rows of K (which = 0) and Q as operands
    auto row_of = [&](int which, int t, int ks, Frag (&f)[NPI]) {
        if constexpr (ROWS) f[0].v = *reinterpret_cast<const uint4 *>(&lds.k.kr[which][t][32 * ks + 8 * g4]);
        else
#pragma unroll
            for (int i = 0; i < NPI; ++i) {
                const Buffer rb = which ? buffer_of(qp + i * p.q.plane, (int64_t)(n - 1) * qrow + 2 * DK) : buffer_of(kp + i * p.k.plane, (int64_t)(n - 1) * krow + 2 * DK);
                f[i].v = buffer_load16(rb, t * (which ? qrow : krow) + 64 * ks + 16 * g4);
            }
    };
    auto four_of = [&](int which, int m) -> f32x4 {      // of this lane's step, columns 16 m + 4 g4 ..
        f32x4 v = {};
#pragma unroll
        for (int i = NPI - 1; i >= 0; --i) {
            uint2 a;
            if constexpr (ROWS) a = *reinterpret_cast<const uint2 *>(&lds.k.kr[which][own][16 * m + 4 * g4]);
            else {
                const Buffer rb = which ? buffer_of(qp + i * p.q.plane, (int64_t)(n - 1) * qrow + 2 * DK) : buffer_of(kp + i * p.k.plane, (int64_t)(n - 1) * krow + 2 * DK);
                a = buffer_load8(rb, own * (which ? qrow : krow) + 32 * m + 8 * g4);
            }
            v += f32x4{__uint_as_float(a.x << 16), hi_part(__uint_as_float(a.x)), __uint_as_float(a.y << 16), hi_part(__uint_as_float(a.y))};
        }
        return v;
    };
    // the states' part of dQ and dK
    float dG = 0.0f, ends = 0.0f;
    {
        const float cq = p.scale * gam, ck = -gam * bown, cw = en * bown, vq = uA * uD, vk = uA * uZ, vw = uB * uE;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const f32x4 kv = four_of(0, m), qv = four_of(1, m);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float a = cq * (vq * qs[m][r]), c = ck * (vk * kr[m][r]), w = cw * (vw * kw[m][r]);
                dq[m][r] += a; dk[m][r] += c + w;
                dG = __builtin_fmaf(qv[r], a, __builtin_fmaf(kv[r], c, dG));
                ends = __builtin_fmaf(kv[r], w, ends);
            }
        }
        dG -= ends;
    }
    // F, H in both orientations, M's row and column sums
    f32x4 HH[4], Ft[4], F[4];
    {
        const float vf = uD * uE, vh = uZ * uE;
        Frag kf[KS][NPI], qf[KS][NPI];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) { row_of(0, own, ks, kf[ks]); row_of(1, own, ks, qf[ks]); }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            f32x4 QKt = {}, QK = {}, KK = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                Frag kx[NPI], qx[NPI];
                row_of(0, 16 * m + row16, ks, kx);
                row_of(1, 16 * m + row16, ks, qx);
                KK = mm(kx, kf[ks], KK);
                QKt = mm(kx, qf[ks], QKt);
                QK = mm(qx, kf[ks], QK);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int o = 16 * m + 4 * g4 + r;
                const double Go = lds.G[o];
                const float bo = lds.beta[o];
                const float D = __expf((float)(o <= own ? Gown - Go : Go - Gown));
                const float ds = p.scale * D * vf, db = -D * bown * bo * vh;
                const float ft = o <= own ? ds * bo * P1[m][r] : 0.0f;          // this step reads what step o wrote
                const float f = o >= own ? ds * bown * (m == wave ? P1own[r] : P1[m][r]) : 0.0f;        // step o reads what this step wrote
                const float hl = o < own ? db * P2[m][r] : 0.0f, hx = o > own ? db * (m == wave ? P2own[r] : P2[m][r]) : 0.0f;
                const float hh = hl + hx;
                dG += (o < own ? ft * QKt[r] : 0.0f) + hl * KK[r];            // (a step's own term would be added and taken off again)
                dG -= (o > own ? f * QK[r] : 0.0f) + hx * KK[r];
                Ft[m][r] = ft; F[m][r] = f; HH[m][r] = hh;
            }
        }
    }
    // dQ += F K, dK += (H + H^T) K + F^T Q
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        Frag ft[NPF], f[NPF], hh[NPF];
        split_tiles<NPF>(Ft[2 * x], Ft[2 * x + 1], ft);
        split_tiles<NPF>(F[2 * x], F[2 * x + 1], f);
        split_tiles<NPF>(HH[2 * x], HH[2 * x + 1], hh);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            Frag kt[NPI], qt[NPI];
#pragma unroll
            for (int i = 0; i < NPI; ++i) {
                kt[i].v = *reinterpret_cast<const uint4 *>(&lds.k.kt[i][16 * m + row16][turned(16 * m, 32 * x + 8 * g4)]);
                qt[i].v = *reinterpret_cast<const uint4 *>(&lds.k.qt[i][16 * m + row16][turned(16 * m, 32 * x + 8 * g4)]);
            }
            dq[m] = mm(kt, ft, dq[m]);
            dk[m] = mm(kt, hh, dk[m]);
            dk[m] = mm(qt, f, dk[m]);
        }
    }
    if (!own_in) { dG = 0.0f; ends = 0.0f; }
    // over the four lane groups of a step, then over the steps
#pragma unroll
    for (int m = 16; m < 64; m <<= 1) {
        dG += __shfl_xor(dG, m, 64);
        dbeta += __shfl_xor(dbeta, m, 64);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        ends += __shfl_xor(ends, m, 64);
        sdot += __shfl_xor(sdot, m, 64);
    }
    if (lane < 16) {
        lds.dG[own] = dG;
        if (own_in) {
            const int64_t i = (row0 + own) * p.Hv + h;
            if (p.gate_io && p.io) store_io(reinterpret_cast<uint16_t *>(p.dbeta) + i, dbeta);
            else store_io(reinterpret_cast<float *>(p.dbeta) + i, dbeta);
        }
    }
    if (lane == 0) { lds.ends[wave] = ends; lds.dots[wave] = sdot; }
    lds_barrier();
    if (wave == 0) {
        float x = lds.dG[lane];
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const float o = __shfl_down(x, m, 64);
            if (lane + m < 64) x += o;
        }
        x += (lds.ends[0] + lds.ends[1]) + (lds.ends[2] + lds.ends[3]);
        x += __expf((float)lds.G[63]) * ((lds.dots[0] + lds.dots[1]) + (lds.dots[2] + lds.dots[3]));
        if (lane < n) {
            const int64_t i = (row0 + lane) * p.Hv + h;
            if (p.gate_io && p.io) store_io(reinterpret_cast<uint16_t *>(p.dg) + i, x);
            else store_io(reinterpret_cast<float *>(p.dg) + i, x);
        }
    }
    if (!own_in) return;
    if (p.part) {
        float *qo = p.part + ((row0 + own) * p.Hv + h) * DK + 4 * g4, *ko = qo + rows * p.Hv * DK;
#pragma unroll
        for (int m = 0; m < MT; ++m) { store4(qo + 16 * m, dq[m]); store4(ko + 16 * m, dk[m]); }
        return;
    }
    IO *qo = reinterpret_cast<IO *>(p.dq) + ((row0 + own) * p.Hk + hk) * p.dk, *ko = reinterpret_cast<IO *>(p.dkk) + ((row0 + own) * p.Hk + hk) * p.dk;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int d = 16 * m + 4 * g4;
        if (p.dk % 4 == 0 && p.o_vec) {
            if (d < p.dk) { store4(qo + d, dq[m]); store4(ko + d, dk[m]); }
        } else
#pragma unroll
            for (int r = 0; r < 4; ++r) if (d + r < p.dk) { store_io(qo + d + r, dq[m][r]); store_io(ko + d + r, dk[m][r]); }
    }
}

// dQ and dK of a shared key head: its value heads' parts in their order.  A workgroup takes a quarter of a slot's steps and a key head, a thread four columns; bound
// by the parts' bytes.  (With a workgroup for all value heads of a key head no parts would be written, but the registers of both sums do not fit
// beside the rest, and where heads are few the chip is left empty: float32, 239 steps of 12 value heads on 4 of 128 x 128, 2 entries: 280 us a
// training step so, 170 with parts.)
template <class IO, int DK> __global__ __launch_bounds__(256) void k_delta_share(const DeltaParams p) {
    const int64_t slot = blockIdx.x / (unsigned)p.Hk;
    const int hk = (int)(blockIdx.x - slot * p.Hk), d = threadIdx.x % (DK / 4) * 4, share = p.Hv / p.Hk;
    DeltaSeq sq;
    int64_t t0;
    int b;
    const int n = delta_slot(p, slot, sq, t0, b);
    const float *part = p.part + (blockIdx.y & 1 ? (int64_t)(p.cu ? 1 : p.B) * p.L * p.Hv * DK : 0);
    void *out = blockIdx.y & 1 ? p.dkk : p.dq;
    for (int t = (blockIdx.y >> 1) * (1024 / DK) + threadIdx.x / (DK / 4); t < n; t += 4 * (1024 / DK)) {
        const int64_t row = sq.row + t0 + t;
        const float *from = part + (row * p.Hv + hk * share) * DK + d;
        IO *to = reinterpret_cast<IO *>(out) + (row * p.Hk + hk) * p.dk + d;
        f32x4 x = {};
        for (int i = 0; i < share; ++i) x += *reinterpret_cast<const f32x4 *>(from + i * DK);
        if (p.dk % 4 == 0 && p.o_vec) {
            if (d < p.dk) store4(to, x);
        } else
#pragma unroll
            for (int r = 0; r < 4; ++r) if (d + r < p.dk) store_io(to + r, x[r]);
    }
}

// ---------------------------------------------------------------- launches
template <int NPI, int NP, int DK, int DS, bool EXACT, bool AGG> static hipError_t launch_adjoint_one(DeltaParams p, hipStream_t s) {
    constexpr int NBUF = NPI == 3 && DK == 128 ? 1 : 2;
    constexpr size_t bytes = sizeof(AdjLds<NPI, NP, DK, NBUF, DS>);
    static_assert(bytes <= 160 * 1024, "LDS");
    p.groups = ((AGG ? p.dvp + DK : p.dvp) / 16 + 4 / DS - 1) / (4 / DS);
    const unsigned blocks = delta_blocks(p, AGG ? p.nseg - 1 : p.nseg);
    auto k = blocks <= 256 ? k_delta_adjoint<NPI, NP, DK, DS, EXACT, AGG, true> : k_delta_adjoint<NPI, NP, DK, DS, EXACT, AGG, false>;
    if (bytes > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(k, dim3(blocks), dim3(256), bytes, s, p);
    return hipGetLastError();
}
template <int NPI, int NP, int DK> static hipError_t launch_adjoint_dk(const DeltaParams &p, hipStream_t s) {
    if (p.nseg > 1) {
        if (const hipError_t e = launch_adjoint_one<NPI, NP, DK, 1, false, true>(p, s)) return e;
        if (const hipError_t e = launch_delta_join(p, true, s)) return e;
    }
    const bool split = delta_rows_split(p);
    if constexpr (NP == 3)
        if (p.exact) return split ? launch_adjoint_one<NPI, NP, DK, 2, true, false>(p, s) : launch_adjoint_one<NPI, NP, DK, 1, true, false>(p, s);
    if constexpr (NPI == 1)
        if (!p.exact) return split ? launch_adjoint_one<NPI, NP, DK, 2, false, false>(p, s) : launch_adjoint_one<NPI, NP, DK, 1, false, false>(p, s);
    return hipErrorInvalidValue;
}
hipError_t launch_delta_adjoint(const DeltaParams &p, hipStream_t s) {
    if (!p.io) return p.dk > 64 ? launch_adjoint_dk<3, 3, 128>(p, s) : launch_adjoint_dk<3, 3, 64>(p, s);
    if (p.np == 3) return p.dk > 64 ? launch_adjoint_dk<1, 3, 128>(p, s) : launch_adjoint_dk<1, 3, 64>(p, s);
    return p.dk > 64 ? launch_adjoint_dk<1, 2, 128>(p, s) : launch_adjoint_dk<1, 2, 64>(p, s);
}
template <class IO, int NPI, int NPE, int DK> static hipError_t launch_grads_one(const DeltaParams &p, hipStream_t s) {
    constexpr size_t bytes = sizeof(GradLds<NPI, NPE, DK>);
    static_assert(bytes <= 160 * 1024, "LDS");
    auto k = k_delta_grads<IO, NPI, NPE, DK>;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k, dim3((unsigned)(p.nslots * p.Hv)), dim3(256), bytes, s, p);
    if (const hipError_t e = hipGetLastError()) return e;
    if (p.part) hipLaunchKernelGGL((k_delta_share<IO, DK>), dim3((unsigned)(p.nslots * p.Hk), 8), dim3(256), 0, s, p);
    return hipGetLastError();
}
hipError_t launch_delta_grads(const DeltaParams &p, hipStream_t s) {
    if (!p.io) return p.dk > 64 ? launch_grads_one<float, 3, 3, 128>(p, s) : launch_grads_one<float, 3, 3, 64>(p, s);
    if (p.exact) return p.dk > 64 ? launch_grads_one<uint16_t, 1, 3, 128>(p, s) : launch_grads_one<uint16_t, 1, 3, 64>(p, s);
    return p.dk > 64 ? launch_grads_one<uint16_t, 1, 1, 128>(p, s) : launch_grads_one<uint16_t, 1, 1, 64>(p, s);
}

}  // namespace lrnnx
