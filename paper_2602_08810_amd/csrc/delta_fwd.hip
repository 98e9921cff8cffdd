// Gated delta rule, forward.  With G the running sum of the log decays within a chunk of C = 32 steps and S0 the state before it:
//     N_ij  = exp(G_i - G_j) k_i . k_j   (j < i)          A_ij = scale exp(G_i - G_j) q_i . k_j   (j <= i)
//     E     = (I + N diag(beta))^-1 (V - diag(exp G) K S0)       the corrections: what the state does not yet say of each value
//     U     = diag(beta) E
//     O     = scale diag(exp G) Q S0 + A U
//     S1    = exp(G_C) S0 + (diag(exp(G_C - G)) K)^T U
// Every exponent is a sum of log decays, at most 0 for decays: nothing overflows, and differences are taken of sums in double precision.
// k_delta_prep forms the inverse and A of every chunk, all chunks side by side; k_delta_scan then walks the chunks of a sequence.
#include "delta_common.hpp"

namespace lrnnx {

// ---------------------------------------------------------------- operands in planes
// A float32 operand, or rows that are not as the matrix kernels read them (width not padded, unaligned), as planes of aligned rows: one launch for
// all operands of a call, eight elements a thread (q, k and the gradient of 3 x 531 steps of 6 heads in float32: 6 us, a latency).
template <class IO> __global__ __launch_bounds__(256) void k_delta_pack(const DeltaPacks all) {
    const DeltaPack &p = all.p[blockIdx.z];
    const unsigned sub = p.rows > 1 ? p.by_items(threadIdx.x) : 0, first = threadIdx.x - sub * p.items;
    if (sub >= p.rows) return;
    const int64_t b = blockIdx.y, step = (int64_t)gridDim.x * p.rows;
    for (int64_t t = (int64_t)blockIdx.x * p.rows + sub; t < all.L; t += step)
        for (unsigned rest = first; rest < p.items; rest += 256) {
            const unsigned h = p.by_head(rest), c = (rest - h * (p.dp / 8)) * 8;
            const int64_t from = b * p.sb + t * p.sl + h * p.sh + c;
            float x[8] = {};
            const IO *f = reinterpret_cast<const IO *>(p.src) + from;
            if (p.vec && c + 8 <= (unsigned)p.d) {
                uint32_t u[2 * sizeof(IO)];
#pragma unroll
                for (int i = 0; i < (int)sizeof(IO) / 2; ++i) {
                    const uint4 v = reinterpret_cast<const uint4 *>(f)[i];
                    u[4 * i] = v.x; u[4 * i + 1] = v.y; u[4 * i + 2] = v.z; u[4 * i + 3] = v.w;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(sizeof(IO) == 4 ? u[e % (2 * sizeof(IO))] : e & 1 ? u[e >> 1] & 0xffff0000u : u[e >> 1] << 16);
            } else if (c < (unsigned)p.d) {
                IO raw[8];                                   // (all loads under way before the first is looked at)
#pragma unroll
                for (int e = 0; e < 8; ++e) raw[e] = f[c + e < (unsigned)p.d ? e : 0];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = c + e < (unsigned)p.d ? load_io(&raw[e]) : 0.0f;
            }
            uint16_t *to = p.dst + ((b * all.L + t) * p.H + h) * p.dp + c;
            Frag g[3];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t u[3];
                split2<3>(x[2 * e], x[2 * e + 1], u);
#pragma unroll
                for (int k = 0; k < 3; ++k) g[k].u[e] = u[k];
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) if (k < all.planes) *reinterpret_cast<uint4 *>(to + k * p.plane) = g[k].v;
        }
}
hipError_t launch_delta_pack(const DeltaPacks &p, hipStream_t s) {
    unsigned rows = 256;
    for (int i = 0; i < p.n; ++i) rows = p.p[i].rows < rows ? p.p[i].rows : rows;
    const int64_t blocks = (p.L + rows - 1) / rows;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536), (unsigned)p.B, (unsigned)p.n);
    if (p.io) hipLaunchKernelGGL(k_delta_pack<uint16_t>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(k_delta_pack<float>, grid, dim3(256), 0, s, p);
    return hipGetLastError();
}

template <class T> __global__ __launch_bounds__(256) void k_delta_gather(const DeltaGather p) {
    const int64_t per_row = (int64_t)p.H * p.d, n = (int64_t)p.B * p.L * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row, b = row / p.L, t = row - b * p.L;
        const int rest = (int)(i - row * per_row), h = rest / p.d;
        reinterpret_cast<T *>(p.dst)[i] = reinterpret_cast<const T *>(p.src)[b * p.sb + t * p.sl + h * p.sh + (rest - h * p.d)];
    }
}
hipError_t launch_delta_gather(const DeltaGather &p, hipStream_t s) {
    const int64_t n = (int64_t)p.B * p.L * p.H * p.d, blocks = (n + 255) / 256;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536));
    if (p.io) hipLaunchKernelGGL(k_delta_gather<uint16_t>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(k_delta_gather<float>, grid, dim3(256), 0, s, p);
    return hipGetLastError();
}

// ---------------------------------------------------------------- the matrices of a chunk
// One wavefront takes a chunk of one value head, rows read straight from memory.  Products K K^T and Q K^T are taken in the orientation in which their
// tiles are operands as they come (A: a step to a lane, its terms in the lane), for the adjoint in the other one too; only N goes through LDS, for the
// solve: a row of the inverse to a lane, each element found and at once taken off the ones before it (496 multiply-adds a lane that do not wait for each
// other).  Substitution is stable where powers of N would cancel.  The upper 32 lanes solve for the adjoint's inverse, which is the same with the steps
// counted from the chunk's end.
// Bound by what it reads and writes, few chunks by latency: 4 x 2048 steps of 16 heads of 128, bfloat16, 23 us where 100 MB are 19 at the rate of a copy;
// 4 x 4096 with the adjoint's matrices 61 us of 46 (71 with a wavefront for two chunks); 2 x 77 steps of 6 heads, float32, 9 (11).
template <int NPI, int NP, int DK, int ADJ> __global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(NPI == 3 ? 2 : 4))) void k_delta_prep(const DeltaParams p) {
    constexpr int KS = DK / 32, W = 36, NPA = NPI == 3 ? 3 : 2, MW = chunk_words(NP, NPA), AW = chunk_words(ADJ, ADJ);
    __shared__ __align__(16) float Ns[ADJ > 0 ? 2 : 1][32][W];           // N by rows; by columns, both counted from the end
    __shared__ double Gs[32];
    __shared__ __align__(16) float Bs[32];
    const int c = blockIdx.x & 1;
    const int64_t unit = blockIdx.x >> 1, slot = unit / (unsigned)p.Hv;
    const int h = (int)(unit - slot * p.Hv), hk = h / (p.Hv / p.Hk);
    const int lane = threadIdx.x, row16 = lane & 15, g4 = lane >> 4, own = lane & 31;
    const bool up = lane >= 32;
    DeltaSeq sq;
    int64_t t0;
    int b;
    const int n = delta_slot(p, slot, sq, t0, b) - 32 * c;   // steps from the chunk's first on
    if (n <= 0) return;
    const int64_t at = sq.at + t0 + 32 * c, mat = unit * 2 + c;
    const uint32_t krow = (uint32_t)p.k.sl * 2, qrow = (uint32_t)p.q.sl * 2;
    const uint16_t *kp = p.k.p + sq.ib * p.k.sb + at * p.k.sl + hk * p.k.sh, *qp = p.q.p + sq.ib * p.q.sb + at * p.q.sl + hk * p.q.sh;
    const bool in = own < n;
    const int64_t tg = at + (in ? own : 0), last = (n < 32 ? n : 32) - 1;
    const float gr = load_gate(p.g, sq.ib * p.g_sb + tg * p.g_sl + h * p.g_sh, p.io, p.gate_io);
    const float be = load_gate(p.beta, sq.ib * p.be_sb + tg * p.be_sl + h * p.be_sh, p.io, p.gate_io);

    // tiles of K K^T and Q K^T: [step written j][step reading i], and [i][j] for the adjoint
    f32x4 kk[3] = {}, qk[3] = {}, qa[3] = {}, ka = {};
    {
        Frag K[KS][2][NPI], Q[KS][2][NPI];
#pragma unroll
        for (int i = 0; i < NPI; ++i) {
            const Buffer kb = buffer_of(kp + i * p.k.plane, last * krow + 2 * DK), qb = buffer_of(qp + i * p.q.plane, last * qrow + 2 * DK);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const uint32_t t = 16 * m + row16;
                    K[ks][m][i].v = buffer_load16(kb, t * krow + 64 * ks + 16 * g4);
                    Q[ks][m][i].v = buffer_load16(qb, t * qrow + 64 * ks + 16 * g4);
                }
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
            for (int x = 0; x < 3; ++x) {                     // (0,0), (0,1), (1,1)
                kk[x] = mm(K[ks][x > 1], K[ks][x > 0], kk[x]);
                qk[x] = mm(K[ks][x > 1], Q[ks][x > 0], qk[x]);
                if (ADJ > 0) qa[x] = mm(Q[ks][x > 0], K[ks][x > 1], qa[x]);
            }
            if (ADJ > 0) ka = mm(K[ks][1], K[ks][0], ka);     // (the tiles on the diagonal are their own transposes)
        }
    }
    // running sums of the log decays, the same in both halves of the wavefront
    {
        double G = in ? gate_log(gr) : 0.0;
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) {
            const double o = __shfl_up(G, m, 32);
            if (own >= m) G += o;
        }
        const double end = __shfl(G, 31, 32);
        const float bv = in ? be : 0.0f, eg = __expf((float)G), ee = __expf((float)(end - G));
        if (!up) {
            Gs[own] = G; Bs[own] = bv;
            float *sc = reinterpret_cast<float *>(p.mats + (mat + 1) * MW - 192) + own;
            sc[0] = eg; sc[32] = ee; sc[64] = bv;
        } else if constexpr (ADJ > 0) {
            float *sc = reinterpret_cast<float *>(p.mats_adj + (mat + 1) * AW - 192) + own;
            sc[0] = eg; sc[32] = ee; sc[64] = bv;
        }
    }
    lds_barrier();
    auto store = [&](const f32x4 &lo, const f32x4 &hi, int m, auto np, auto upper, uint16_t *to) {       // tile m of an operand (triangle_tile)
        constexpr int P = decltype(np)::value;
        constexpr bool UP = decltype(upper)::value;
        Frag f[P];
        split_tiles<P>(lo, hi, f);
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (m == UP) *reinterpret_cast<uint2 *>(to + i * 256 + lane * 4) = f[i].h[UP];
            else *reinterpret_cast<uint4 *>(to + (P + 2 * i) * 256 + lane * 8) = f[i].v;
    };
    using ForA = std::integral_constant<int, NPA>;
    {
        float rows[2] = {0.0f, 0.0f};                        // of the lane's row of either half: 0, or NaN
        f32x4 A[3], At[3];
#pragma unroll
        for (int x = 0; x < 3; ++x) {
            {                                                // a reading step to a lane
                const int i = 16 * (x > 0) + row16, j0 = 16 * (x > 1) + 4 * g4;
                const double Gi = Gs[i];
                f32x4 N;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float d = j0 + r <= i ? __expf((float)(Gi - Gs[j0 + r])) : 0.0f;
                    N[r] = j0 + r < i ? d * kk[x][r] : 0.0f;
                    A[x][r] = j0 + r <= i ? p.scale * d * qk[x][r] : 0.0f;
                    rows[x > 0] = __builtin_fmaf(N[r], 0.0f, rows[x > 0]);
                }
                *reinterpret_cast<f32x4 *>(&Ns[0][i][j0]) = N;
            }
            if constexpr (ADJ > 0) {                         // a written step to a lane
                const int j = 16 * (x > 1) + row16, i0 = 16 * (x > 0) + 4 * g4;
                const double Gj = Gs[j];
                f32x4 N;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float d = j <= i0 + r ? __expf((float)(Gs[i0 + r] - Gj)) : 0.0f;
                    N[3 - r] = j < i0 + r ? d * (x == 1 ? ka[r] : kk[x][r]) : 0.0f;
                    At[x][r] = j <= i0 + r ? p.scale * d * qa[x][r] : 0.0f;
                }
                *reinterpret_cast<f32x4 *>(&Ns[1][31 - j][28 - i0]) = N;
            }
        }
        const f32x4 none = {};
        uint16_t *to = p.mats + mat * MW + NP * 768;
        store(A[0], none, 0, ForA(), std::false_type(), to);
        store(A[1], A[2], 1, ForA(), std::false_type(), to);
        if constexpr (ADJ > 0) {
            to = p.mats_adj + mat * AW + ADJ * 768;
            store(At[0], At[1], 0, std::integral_constant<int, ADJ>(), std::true_type(), to);
            store(none, At[2], 1, std::integral_constant<int, ADJ>(), std::true_type(), to);
        }
        const uint64_t lower = __ballot(rows[0] != 0.0f), upper = __ballot(rows[1] != 0.0f), strong = __ballot(Bs[own] - Bs[own] != 0.0f);
        if (lower | upper | strong) {                        // rows from the first that is not finite on: none of N, the walk finds NaN in exp(G)
            auto fold = [](uint64_t m) { return (uint32_t)(m | m >> 16 | m >> 32 | m >> 48) & 0xffffu; };
            const int sound = __builtin_ctz(fold(lower) | fold(upper) << 16 | (uint32_t)strong);
            lds_barrier();
            if (!up && own >= sound) {
                Bs[own] = 0.0f;
                for (int j = 0; j < 32; ++j) Ns[0][own][j] = 0.0f;
                *(reinterpret_cast<float *>(p.mats + (mat + 1) * MW - 192) + own) = __builtin_nanf("");
            }
            if (ADJ > 0 && up)
                for (int j = 0; j < 32; ++j) Ns[ADJ > 0][own][j] = __builtin_nanf("");
        }
    }
    lds_barrier();

    // X (I + N diag(beta)) = I, from the last column to the first; row `own`, of the adjoint counted from the end
    const int from = ADJ > 0 && up ? 32 * W : 0;
    const float *N = &Ns[0][0][0] + from;
    {
        float x[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) x[j] = 0.0f;            // the sums over later columns first, then the element
#pragma unroll
        for (int l = 31; l >= 0; --l) {
            x[l] = (l == own ? 1.0f : 0.0f) - Bs[ADJ > 0 && up ? 31 - l : l] * x[l];
#pragma unroll
            for (int j = 0; j < l; j += 4) {
                const f32x4 v = *reinterpret_cast<const f32x4 *>(N + l * W + j);
#pragma unroll
                for (int e = 0; e < 4; ++e) if (j + e < l) x[j + e] = __builtin_fmaf(x[l], v[e], x[j + e]);
            }
        }
        lds_barrier();                                       // through LDS into the operands' order
        float *row = &Ns[0][0][0] + (ADJ > 0 && up ? (32 + 31 - own) * W : own * W);
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
            const f32x4 v = {x[j], x[j + 1], x[j + 2], x[j + 3]};
            *reinterpret_cast<f32x4 *>(row + (ADJ > 0 && up ? 28 - j : j)) = ADJ > 0 && up ? f32x4{v[3], v[2], v[1], v[0]} : v;
        }
    }
    lds_barrier();
    auto half = [&](int which, int m, int k) { return *reinterpret_cast<const f32x4 *>(&Ns[which][16 * m + row16][16 * k + 4 * g4]); };
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        store(half(0, m, 0), half(0, m, 1), m, std::integral_constant<int, NP>(), std::false_type(), p.mats + mat * MW);
        if constexpr (ADJ > 0) store(half(1, m, 0), half(1, m, 1), m, std::integral_constant<int, ADJ>(), std::true_type(), p.mats_adj + mat * AW);
    }
}

// ---------------------------------------------------------------- the walk over the chunks
// A wavefront owns 16 columns of a head's state, dk x 16 in float32 accumulators, for the whole sequence.  A result tile of a matrix instruction
// holds a column of four rows in each lane, which is what the second operand of the next instruction wants of its terms, so K S0 -> E -> U ->
// K^T U runs from registers to registers: no exchange between lanes or wavefronts on the path that the next chunk waits for.  The wavefronts of
// a workgroup share what is the same for all columns (K, Q, K^T, the chunk's matrices) in LDS.
template <int NPI, int NP, int DK, int NBUF, int DS> struct ScanLds {
    static constexpr int NPA = NPI == 3 ? 3 : 2;
    struct Buf {
        uint16_t k[NPI][32][DK + 8], q[NPI][32][DK + 8], kt[NPI][DK][40];
        uint16_t th[NP][256], tw[NP][512], ah[NPA][256], aw[NPA][512];         // (as they lie in memory)
        float scal[96];
    } buf[NBUF];
    f32x4 halves[DS == 2 ? 12 : 1][64];
};

// Bound by the latency of a chunk's chain of products and of the rows it brings: 4 x 2048 steps of 16 heads of 128 x 128, bfloat16 with the last state in
// float32, 64 chunks in 124 us; 4 x 4096 with what the backward pass is left, 260 us where 540 MB are 102 at the rate of a copy.
// DS = 2: two wavefronts share 16 columns, each with half of the rows of S: half of the products and registers each, for one exchange through LDS (the
// halves of K S0 and Q S0 are added) and twice the workgroups (the two cases above with one wavefront: 139 and 335 us).
// AGG: what a segment makes of the state that enters it, S -> M S + N, without outputs: N is the walk from a state of zero, and the columns of M, behind those
// of v, are walks from the columns of I with v = 0.  k_delta_join then chains the segments, and each is walked again from its true state.
template <class IO, int NPI, int NP, int DK, int DS, bool SAVE, bool EXACT, bool AGG>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_delta_scan(const DeltaParams p) {
    constexpr int NT = 256, CW = 4 / DS, KS = DK / 32 / DS, MT = DK / 16 / DS, OT = 2 / DS;          // tiles that are a wavefront's own
    constexpr int NPA = NPI == 3 ? 3 : 2;
    constexpr int NBUF = NPI == 3 && DK == 128 ? 1 : 2;
    constexpr int NPO = NPI == 3 ? 3 : 2;                 // planes of what only enters o
    extern __shared__ __align__(16) char lds_raw[];
    using Lds = ScanLds<NPI, NP, DK, NBUF, DS>;
    Lds &lds = *reinterpret_cast<Lds *>(lds_raw);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row16 = lane & 15, g4 = lane >> 4;
    DeltaUnit un;
    if (!delta_unit(p, AGG ? p.nseg - 1 : p.nseg, un)) return;
    const int h = un.h, hk = h / (p.Hv / p.Hk), b = un.b;
    const DeltaSeq sq = delta_seq(p, b);
    const int dh = DS == 2 ? wave & 1 : 0, d0 = dh * (DK / 2);         // this wavefront's half of the rows of S
    const int c0 = (un.group * CW + wave / DS) * 16, n0 = c0 + row16;  // this wavefront's columns, this lane's
    const bool col_in = n0 < p.dv;
    const int64_t nchunk = (sq.len + 31) / 32, ch0 = p.nseg > 1 ? (int64_t)un.seg * p.seg_chunks : 0;
    const int64_t ch1 = p.nseg > 1 && nchunk > ch0 + p.seg_chunks ? ch0 + p.seg_chunks : nchunk;
    if (ch0 >= nchunk && un.seg > 0) return;
    const int64_t head = (int64_t)b * p.Hv + h;
    const NegId neg = neg_id();
    const bool wide = p.o_vec && c0 + 16 <= p.dv;                      // o in stores of four elements

    f32x4 S[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = d0 + 16 * m + 4 * g4 + r;
            if (AGG) S[m][r] = d == n0 - p.dvp ? 1.0f : 0.0f;
            else if (un.seg > 0) S[m][r] = c0 < p.dvp ? p.entry[((head * p.nseg + un.seg) * DK + d) * p.dvp + n0] : 0.0f;
            else S[m][r] = p.s0 && col_in && d < p.dk ? p.s0[(head * p.dk + d) * p.dv + n0] : 0.0f;
        }

    const uint16_t *kp = p.k.p + sq.ib * p.k.sb + sq.at * p.k.sl + hk * p.k.sh, *qp = p.q.p + sq.ib * p.q.sb + sq.at * p.q.sl + hk * p.q.sh;
    const IO *vp = reinterpret_cast<const IO *>(p.v) + sq.ib * p.v_sb + sq.at * p.v_sl + h * p.v_sh;
    IO *op = reinterpret_cast<IO *>(p.o) + sq.ib * p.o_sb + sq.at * p.o_sl + h * p.o_sh + c0 + 4 * g4;

    // what a thread brings into LDS: quads of four steps by four columns of K, 16 bytes of Q, 16 bytes of the chunk's matrices
    constexpr int QUADS = 8 * (DK / 4), QROWS = 32 * (DK / 8), MATS = chunk_words(NP, NPA) / 8;
    constexpr int IQ = (QUADS + NT - 1) / NT, IR = (QROWS + NT - 1) / NT, IM = (MATS + NT - 1) / NT;
    struct Stage {
        uint2 k[IQ][NPI][4];
        uint4 q[IR][NPI], m[IM];
    };
    constexpr bool LATE = NPI == 1 && (AGG || DK == 64 || (DS == 2 && !(SAVE && NP == 3)));
    struct Values { IO v[2][4]; float gend; };             // rows of v and exp(G_C), wanted in their own chunk
    const uint32_t krow = (uint32_t)p.k.sl * 2, qrow = (uint32_t)p.q.sl * 2, vrow = (uint32_t)p.v_sl * sizeof(IO);
    const uint32_t voff = col_in ? 4 * g4 * vrow + n0 * (uint32_t)sizeof(IO) : kOutside;
    // (a chunk past the segment's end: nothing is read, without a branch that would have to wait for the registers)
    auto fetch = [&](int64_t ch, Stage &st, Values &vs) __attribute__((always_inline)) {
        const bool in = ch < ch1;
        const int64_t t0 = in ? ch * 32 : 0, last = (sq.len - t0 < 32 ? sq.len - t0 : 32) - 1;
#pragma unroll
        for (int pl = 0; pl < NPI; ++pl) {
            const Buffer kb = buffer_of(kp + pl * p.k.plane + t0 * p.k.sl, in ? last * krow + 2 * DK : 0);
            const Buffer qb = buffer_of(qp + pl * p.q.plane + t0 * p.q.sl, in ? last * qrow + 2 * DK : 0);
#pragma unroll
            for (int x = 0; x < IQ; ++x) {
                const int i = tid + x * NT, tq = i / (DK / 4), dq = i % (DK / 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) st.k[x][pl][e] = buffer_load8(kb, QUADS % NT && i >= QUADS ? kOutside : (4 * tq + e) * krow + 8 * dq);
            }
#pragma unroll
            for (int x = 0; x < (AGG ? 0 : IR); ++x) {
                const int i = tid + x * NT, t = i / (DK / 8), d8 = i % (DK / 8);
                st.q[x][pl] = buffer_load16(qb, QROWS % NT && i >= QROWS ? kOutside : t * qrow + 16 * d8);
            }
        }
        const int64_t mat = in ? ((sq.slot + (ch >> 1)) * p.Hv + h) * 2 + (ch & 1) : 0;
        const Buffer mb = buffer_of(p.mats + mat * (MATS * 8), in ? MATS * 16 : 0);
#pragma unroll
        for (int x = 0; x < IM; ++x) st.m[x] = buffer_load16(mb, (tid + x * NT) * 16);
        const Buffer vb = buffer_of(vp + t0 * p.v_sl, in ? last * vrow + p.dv * (int)sizeof(IO) : 0);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) buffer_load(vb, voff + (16 * m + r) * vrow, vs.v[m][r]);
        if constexpr (!LATE) buffer_load(mb, MATS * 16 - 4 * (96 - 31), vs.gend);
    };
    auto put = [&](typename Lds::Buf &B, const Stage &st) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < IQ; ++x) {
            const int i = tid + x * NT, tq = i / (DK / 4), dq = i % (DK / 4);
            if (QUADS % NT && i >= QUADS) continue;
            const int col = (dq >> 3) * 32 + quad_place(dq & 7), place = quad_place(tq);
#pragma unroll
            for (int pl = 0; pl < NPI; ++pl) {
                uint2 c[4];
                transpose_quad(st.k[x][pl], c);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    *reinterpret_cast<uint2 *>(&B.k[pl][4 * tq + e][col]) = st.k[x][pl][e];
                    *reinterpret_cast<uint2 *>(&B.kt[pl][4 * dq + e][turned(4 * dq, place)]) = c[e];
                }
            }
        }
#pragma unroll
        for (int x = 0; x < (AGG ? 0 : IR); ++x) {
            const int i = tid + x * NT, t = i / (DK / 8), d8 = i % (DK / 8);
            if (QROWS % NT && i >= QROWS) continue;
            const int q0 = (2 * d8) & 7, base = (d8 >> 2) * 32;
#pragma unroll
            for (int pl = 0; pl < NPI; ++pl) {
                *reinterpret_cast<uint2 *>(&B.q[pl][t][base + quad_place(q0)]) = make_uint2(st.q[x][pl].x, st.q[x][pl].y);
                *reinterpret_cast<uint2 *>(&B.q[pl][t][base + quad_place(q0 + 1)]) = make_uint2(st.q[x][pl].z, st.q[x][pl].w);
            }
        }
        uint4 *mats = reinterpret_cast<uint4 *>(&B.th[0][0]);
#pragma unroll
        for (int x = 0; x < IM; ++x)
            if (MATS % NT == 0 || tid + x * NT < MATS) mats[tid + x * NT] = st.m[x];
    };

    // What is not finite in v, k or the gates of the chunk (there exp(G) is NaN) must not meet the zeros that stand in T and A for later steps: from a
    // column's first such step on R and beta, and so U, are taken as zeros, o, what is saved and the state after the chunk as NaN.  LATE: looked for in R;
    // else at the start of the step, in v and exp(G_C), which then is another copy of the code (`rare`): a branch amid a step costs up to 3 % and 30 registers,
    // and where they spill 8 % (8 heads of 128 x 128 on 32768 steps, the second walk 151 -> 163 us) or, in float32, 80 %; the other way costs 2 to 4 %.
    auto step = [&](int64_t ch, Stage &st, const Values &v, Values &vnext, auto rare) __attribute__((always_inline)) {
        const typename Lds::Buf &B = lds.buf[NBUF == 2 ? ch & 1 : 0];
        const int64_t t0 = ch * 32;
        const int n = (int)(sq.len - t0 < 32 ? sq.len - t0 : 32);
        constexpr bool ONE = SAVE && DS == 1;
        f32x4 V[2];                                         // (with SAVE there are no registers for a second set of rows under way)
        if constexpr (ONE)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) V[m][r] = load_io(&v.v[m][r]);
        fetch(ch + 1, st, vnext);

        const int64_t sh = (sq.slot + (ch >> 1)) * p.Hv + h;
        if (SAVE && !(ch & 1) && c0 < p.dvp) {
            const int G = p.dvp / 16;
            save_state<EXACT, DK>(S, p.states, (sh * p.dvp + n0) * DK + d0 + 4 * g4, p.units + (sh * 6 + dh) * G + c0 / 16, G);
        }

        // K S0 and (transposed: a step to a lane) Q S0
        constexpr bool EARLY = NPI == 1 || DK == 64;        // operands read well before they are used
        Frag kf[EARLY ? KS : 1][2][NPI], qf[EARLY ? KS : 1][2][NPI], tf[2][NP], ktf[EARLY ? MT : 1][NPI], af[OT][NPA], tt[OT][NP];
        f32x4 gam[2], be[2], en[2];
        auto read_kq = [&](int ks, int at) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int i = 0; i < NPI; ++i) {
                    kf[at][m][i].v = *reinterpret_cast<const uint4 *>(&B.k[i][16 * m + row16][d0 + 32 * ks + 8 * g4]);
                    if constexpr (!AGG) qf[at][m][i].v = *reinterpret_cast<const uint4 *>(&B.q[i][16 * m + row16][d0 + 32 * ks + 8 * g4]);
                }
        };
        if constexpr (EARLY)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) read_kq(ks, ks);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            gam[m] = *reinterpret_cast<const f32x4 *>(&B.scal[16 * m + 4 * g4]);
#pragma unroll
            for (int i = 0; i < NP; ++i) tf[m][i] = m ? whole_tile(B.tw[i], lane) : half_tile<false>(B.th[i], lane);
        }
        if constexpr (EARLY) reads_first();
        f32x4 P[2] = {}, O[2] = {};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            Frag s[NP];
            split_tiles<NP>(S[2 * ks], S[2 * ks + 1], s, neg);
            const int at = EARLY ? ks : 0;
            if constexpr (!EARLY) read_kq(ks, 0);
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < NPI; ++j)
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        if (i + j < NP) P[m] = mfma(kf[at][m][j], s[i], P[m]);
                        if (!AGG && i < NPO && i + j < NPO) O[m] = mfma(s[i], qf[at][m][j], O[m]);
                    }
        }
        f32x4 Oown[OT];                                     // and the tiles of the chunk's steps whose o (and E) it writes
        const int first = DS == 2 ? dh : 0;
        if constexpr (DS == 2) {
            lds.halves[3 * wave][lane] = P[0];
            lds.halves[3 * wave + 1][lane] = P[1];
            if constexpr (!AGG) lds.halves[3 * wave + 2][lane] = dh ? O[0] : O[1];
            lds_barrier();
            P[0] += lds.halves[3 * (wave ^ 1)][lane];
            P[1] += lds.halves[3 * (wave ^ 1) + 1][lane];
            Oown[0] = dh ? O[1] : O[0];
            if constexpr (!AGG) Oown[0] += lds.halves[3 * (wave ^ 1) + 2][lane];
        } else
#pragma unroll
            for (int m = 0; m < OT; ++m) Oown[m] = O[m];
        if constexpr (EARLY) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < NPI; ++i) ktf[m][i].v = *reinterpret_cast<const uint4 *>(&B.kt[i][d0 + 16 * m + row16][turned(d0 + 16 * m, 8 * g4)]);
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            be[m] = *reinterpret_cast<const f32x4 *>(&B.scal[64 + 16 * m + 4 * g4]);
            en[m] = *reinterpret_cast<const f32x4 *>(&B.scal[32 + 16 * m + 4 * g4]);
        }
        if constexpr (!AGG)
#pragma unroll
            for (int m = 0; m < OT; ++m) {
#pragma unroll
                for (int i = 0; i < NPA; ++i) triangle_tile<false>(first + m == 0, B.ah[i], B.aw[i], lane, af[m][i]);
                if constexpr (SAVE)
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        if constexpr (DS == 2) triangle_tile<false>(dh == 0, B.th[i], B.tw[i], lane, tt[m][i]);
                        else tt[m][i] = tf[m][i];
                    }
            }
        if constexpr (EARLY) reads_first();
        // E = (I + N beta)^-1 (V - exp(G) K S0)
        f32x4 R[2], E[2] = {}, Et[OT] = {};
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) R[m][r] = __builtin_fmaf(-gam[m][r], P[m][r], ONE ? V[m][r] : load_io(&v.v[m][r]));
        float gend = B.scal[31];
        bool fix = decltype(rare)::value;
        if constexpr (LATE) fix = __any(!__builtin_isfinite(((R[0][0] + R[0][1]) + (R[0][2] + R[0][3])) + ((R[1][0] + R[1][1]) + (R[1][2] + R[1][3]))));
        if (__builtin_expect(fix, 0)) {
            int bad = 32;
#pragma unroll
            for (int t = 7; t >= 0; --t) bad = __builtin_isfinite(R[t >> 2][t & 3]) ? bad : 16 * (t >> 2) + 4 * g4 + (t & 3);
            bad = min(bad, __shfl_xor(bad, 16, 64));
            bad = min(bad, __shfl_xor(bad, 32, 64));
            if (bad < 32) gend = __builtin_nanf("");
#pragma unroll
            for (int t = 0; t < 8; ++t)
                if (16 * (t >> 2) + 4 * g4 + (t & 3) >= bad) { R[t >> 2][t & 3] = 0.0f; be[t >> 2][t & 3] = 0.0f; }
            if constexpr (!AGG)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int column = __shfl(bad, 4 * g4 + r, 64);
#pragma unroll
                    for (int m = 0; m < OT; ++m)
                        if (16 * (first + m) + row16 >= column) Oown[m][r] = Et[m][r] = __builtin_nanf("");
                }
        }
        Frag rf[NP];
        split_tiles<NP>(R[0], R[1], rf, neg);
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < NP; ++j)
                if (i + j < NP)
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        E[m] = mfma(tf[m][i], rf[j], E[m]);
                        if (SAVE && m < OT) Et[m] = mfma(rf[j], tt[m][i], Et[m]);  // a step to a lane, for wide stores
                    }
        // U = beta E, and U decayed to the end of the chunk
        f32x4 U[2], D[2];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) { U[m][r] = be[m][r] * E[m][r]; D[m][r] = en[m][r] * U[m][r]; }
        Frag uf[NPO], df[NP];
        split_tiles<NP>(D[0], D[1], df, neg);
        if constexpr (!AGG) split_tiles<NPO>(U[0], U[1], uf, neg);
        // S1
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[m][r] *= gend;
        if constexpr (EARLY) mm_each(ktf, df, S);
        else
#pragma unroll
            for (int m = 0; m < MT; ++m) {
#pragma unroll
                for (int i = 0; i < NPI; ++i) ktf[0][i].v = *reinterpret_cast<const uint4 *>(&B.kt[i][d0 + 16 * m + row16][turned(d0 + 16 * m, 8 * g4)]);
                S[m] = mm(ktf[0], df, S[m]);
            }
        if (SAVE && c0 < p.dvp) {
            const int G = p.dvp / 16;
            save_rows<EXACT>(Et, p.err, ((sq.row + t0 + 16 * first + row16) * p.Hv + h) * p.dvp + c0 + 4 * g4, (int64_t)16 * p.Hv * p.dvp,
                             n - 16 * first, p.units + (sh * 6 + 2 + 2 * (ch & 1) + first) * G + c0 / 16, G);
        }
        if constexpr (!AGG) {                               // O
#pragma unroll
            for (int m = 0; m < OT; ++m) {
                const float gs = p.scale * B.scal[16 * (first + m) + row16];
#pragma unroll
                for (int r = 0; r < 4; ++r) Oown[m][r] *= gs;
            }
#pragma unroll
            for (int i = 0; i < NPO; ++i)
#pragma unroll
                for (int j = 0; j < NPA; ++j)
                    if (i + j < (NPO > NPA ? NPO : NPA))
#pragma unroll
                        for (int m = 0; m < OT; ++m) Oown[m] = mfma(uf[i], af[m][j], Oown[m]);
#pragma unroll
            for (int m = 0; m < OT; ++m) {
                const int t = 16 * (first + m) + row16;
                IO *to = op + (t0 + t) * p.o_sl;
                if (wide) { if (t < n) store4(to, Oown[m]); }
                else if (t < n)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (c0 + 4 * g4 + r < p.dv) store_io(to + r, Oown[m][r]);
            }
        }
        if (NBUF == 1) lds_barrier();
        put(lds.buf[NBUF == 2 ? (ch + 1) & 1 : 0], st);
        lds_barrier();
    };
    auto walk = [&](int64_t ch, Stage &st, const Values &v, Values &vnext) __attribute__((always_inline)) {
        if constexpr (!LATE) {
            float whole[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) whole[r] = load_io(&v.v[0][r]) + load_io(&v.v[1][r]);
            if (__builtin_expect(__any(!__builtin_isfinite(((whole[0] + whole[1]) + (whole[2] + whole[3])) + v.gend)), 0)) return step(ch, st, v, vnext, std::true_type{});
        }
        step(ch, st, v, vnext, std::false_type{});
    };
    Stage st;
    Values va, vb;
    fetch(ch0, st, va);
    put(lds.buf[0], st);                                    // (segments have an even number of chunks)
    lds_barrier();
    if constexpr (SAVE && DS == 1)
        for (int64_t ch = ch0; ch < ch1; ++ch) walk(ch, st, va, va);
    else
        for (int64_t ch = ch0; ch < ch1;) {                 // two chunks a round, so that no register is copied while it is loaded
            walk(ch, st, va, vb);
            if (++ch >= ch1) break;
            walk(ch, st, vb, va);
            ++ch;
        }
    if constexpr (AGG) {
        if (c0 < p.dvp) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) p.entry[((head * p.nseg + un.seg + 1) * DK + 16 * m + 4 * g4 + r) * p.dvp + n0] = S[m][r];
        } else if (c0 < p.dvp + DK) store_trans<NP, DK>(S, p.trans + (head * (p.nseg - 1) + un.seg) * NP * DK * DK, n0 - p.dvp, g4);
    } else if (p.s_last && col_in && ch1 == nchunk)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = d0 + 16 * m + 4 * g4 + r;
                if (d < p.dk) p.s_last[(head * p.dk + d) * p.dv + n0] = S[m][r];
            }
}

// ---------------------------------------------------------------- chaining segments
// entry[s + 1] <- M_s entry[s] + N_s in the order of time (N_s lies in entry[s + 1]; entry[0] is s0), for the adjoint entry[s - 1] <- M_s entry[s] + N_s
// against it.  A workgroup takes 32 columns, a wavefront 16 rows of them: its rows of M and of N are under way two segments ahead, and only the state
// itself, in planes through LDS, is waited for (21 us a segment with a wavefront for all rows of 16 columns, 4 so: what a compute unit reads of M).
template <int NP, int DK, bool ADJ> __global__ __launch_bounds__(DK * 4) void k_delta_join(const DeltaParams p) {
    constexpr int KS = DK / 32;
    __shared__ __align__(16) uint16_t st[2][NP][32][DK + 8];
    const int lane = threadIdx.x & 63, m = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row16 = lane & 15, g4 = lane >> 4;
    const int n0 = blockIdx.x * 32 + row16, h = blockIdx.y, b = blockIdx.z;
    const int64_t head = (int64_t)b * p.Hv + h, plane = DK * p.dvp;
    const float *first = ADJ ? p.ds_last : p.s0;
    f32x4 S[2];
    struct Part { f32x4 N[2]; Frag M[KS][NP]; } even, odd;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = 16 * m + 4 * g4 + r, n = n0 + 16 * c;
            S[c][r] = first && n < p.dv && d < p.dk ? first[(head * p.dk + d) * p.dv + n] : 0.0f;
        }
    auto place = [&](int i) { return p.entry + (head * p.nseg + (ADJ ? p.nseg - 2 - i : i + 1)) * plane + (16 * m + 4 * g4) * p.dvp + n0; };
    auto fetch = [&](int i, Part &a) __attribute__((always_inline)) {
        if (i > p.nseg - 2) i = p.nseg - 2;                  // (past the end: the last one again, no branch around the loads)
        const uint16_t *t = p.trans + (head * (p.nseg - 1) + (ADJ ? p.nseg - 2 - i : i)) * NP * DK * DK + (16 * m + row16) * DK + 8 * g4;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int k = 0; k < NP; ++k) a.M[ks][k].v = *reinterpret_cast<const uint4 *>(t + k * DK * DK + 32 * ks);
        const float *at = place(i);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) a.N[c][r] = at[r * p.dvp + 16 * c];
    };
    auto step = [&](int i, Part &a) __attribute__((always_inline)) {
        auto &L = st[i & 1];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t lo[NP], hi[NP];
            split2<NP>(S[c][0], S[c][1], lo);
            split2<NP>(S[c][2], S[c][3], hi);
#pragma unroll
            for (int k = 0; k < NP; ++k) *reinterpret_cast<uint2 *>(&L[k][16 * c + row16][16 * m + 4 * g4]) = make_uint2(lo[k], hi[k]);
            S[c] = a.N[c];
        }
        lds_barrier();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                Frag s[NP];
#pragma unroll
                for (int k = 0; k < NP; ++k) s[k].v = *reinterpret_cast<const uint4 *>(&L[k][16 * c + row16][32 * ks + 8 * g4]);
                S[c] = mm(a.M[ks], s, S[c]);
            }
        fetch(i + 2, a);
        float *at = place(i);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) at[r * p.dvp + 16 * c] = S[c][r];
    };
    fetch(0, even);
    fetch(1, odd);
    for (int i = 0; i < p.nseg - 1;) {
        step(i, even);
        if (++i >= p.nseg - 1) break;
        step(i, odd);
        ++i;
    }
}
template <int NP, bool ADJ> static hipError_t launch_join(const DeltaParams &p, hipStream_t s) {
    const dim3 grid((unsigned)(p.dvp / 32), (unsigned)p.Hv, (unsigned)p.B);
    if (p.dk > 64) hipLaunchKernelGGL((k_delta_join<NP, 128, ADJ>), grid, dim3(512), 0, s, p);
    else hipLaunchKernelGGL((k_delta_join<NP, 64, ADJ>), grid, dim3(256), 0, s, p);
    return hipGetLastError();
}
hipError_t launch_delta_join(const DeltaParams &p, bool adjoint, hipStream_t s) {
    if (adjoint) return p.np == 3 ? launch_join<3, true>(p, s) : launch_join<2, true>(p, s);
    return p.np == 3 ? launch_join<3, false>(p, s) : launch_join<2, false>(p, s);
}

// ---------------------------------------------------------------- launches
template <int NPI, int NP, int ADJ> static hipError_t launch_prep(const DeltaParams &p, hipStream_t s) {
    const dim3 grid((unsigned)(2 * p.nslots * p.Hv)), block(64);
    if (p.dk > 64) hipLaunchKernelGGL((k_delta_prep<NPI, NP, 128, ADJ>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_delta_prep<NPI, NP, 64, ADJ>), grid, block, 0, s, p);
    return hipGetLastError();
}
hipError_t launch_delta_prep(const DeltaParams &p, hipStream_t s) {
    if (!p.io) return p.mats_adj ? launch_prep<3, 3, 3>(p, s) : launch_prep<3, 3, 0>(p, s);
    if (!p.mats_adj) return p.np == 3 ? launch_prep<1, 3, 0>(p, s) : launch_prep<1, 2, 0>(p, s);
    if (p.np_adjoint == 3) return launch_prep<1, 3, 3>(p, s);
    return p.np == 3 ? launch_prep<1, 3, 2>(p, s) : launch_prep<1, 2, 2>(p, s);
}

template <class IO, int NPI, int NP, int DK, int DS, bool SAVE, bool EXACT, bool AGG> static hipError_t launch_scan_one(DeltaParams p, hipStream_t s) {
    constexpr int NBUF = NPI == 3 && DK == 128 ? 1 : 2;
    constexpr size_t bytes = sizeof(ScanLds<NPI, NP, DK, NBUF, DS>);
    static_assert(bytes <= 160 * 1024, "LDS");
    p.groups = ((AGG ? p.dvp + DK : p.dvp) / 16 + 4 / DS - 1) / (4 / DS);
    auto k = k_delta_scan<IO, NPI, NP, DK, DS, SAVE, EXACT, AGG>;
    if (bytes > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(k, dim3(delta_blocks(p, AGG ? p.nseg - 1 : p.nseg)), dim3(256), bytes, s, p);
    return hipGetLastError();
}
template <class IO, int NPI, int NP, int DK> static hipError_t launch_scan_dk(const DeltaParams &p, hipStream_t s) {
    if (p.nseg > 1) {
        if (const hipError_t e = launch_scan_one<IO, NPI, NP, DK, 1, false, false, true>(p, s)) return e;
        if (const hipError_t e = launch_delta_join(p, false, s)) return e;
    }
    const bool split = delta_rows_split(p);
    if (!p.states) return split ? launch_scan_one<IO, NPI, NP, DK, 2, false, false, false>(p, s) : launch_scan_one<IO, NPI, NP, DK, 1, false, false, false>(p, s);
    if constexpr (NP == 3)
        if (p.exact) return split ? launch_scan_one<IO, NPI, NP, DK, 2, true, true, false>(p, s) : launch_scan_one<IO, NPI, NP, DK, 1, true, true, false>(p, s);
    if constexpr (NPI == 1)
        if (!p.exact) return split ? launch_scan_one<IO, NPI, NP, DK, 2, true, false, false>(p, s) : launch_scan_one<IO, NPI, NP, DK, 1, true, false, false>(p, s);
    return hipErrorInvalidValue;
}
hipError_t launch_delta_scan(const DeltaParams &p, hipStream_t s) {
    if (!p.io) return p.dk > 64 ? launch_scan_dk<float, 3, 3, 128>(p, s) : launch_scan_dk<float, 3, 3, 64>(p, s);
    if (p.np == 3) return p.dk > 64 ? launch_scan_dk<uint16_t, 1, 3, 128>(p, s) : launch_scan_dk<uint16_t, 1, 3, 64>(p, s);
    return p.dk > 64 ? launch_scan_dk<uint16_t, 1, 2, 128>(p, s) : launch_scan_dk<uint16_t, 1, 2, 64>(p, s);
}

}  // namespace lrnnx
