// Softmax cross entropy over a vocabulary without its logits: z = h w^T, lse = log sum exp z, loss = lse - z[target], and
//     dz = dloss (exp(z - lse) - onehot(target)),   dh = dz w,   dw = dz^T h.
// Forward: a tile of z stays in registers from its product to its largest number and sum, which is all that leaves it (8 bytes for 256 words and a row); a second
// launch joins them.  Backward: z is formed again, a piece of the vocabulary at a time, dz of the piece goes to the workspace in bfloat16 (its rounding is
// as large as the results' own) and from there into both products.  Rows without a target are left out before the products: they cost nothing and
// nothing in them, finite or not, reaches a gradient.
// Float32 inputs: every factor is the sum of three bfloat16 numbers, a product six of theirs (terms of 2^-24 and below are left out), summed in float32.
// Bound by the matrix units.  The core: tiles of 256 x 256, 64 terms at a time, eight wavefronts of 128 x 64, two stages of LDS of 64 KB filled from memory
// without registers between.
#include "vocab_loss.hpp"
#include "conv_common.hpp"

namespace lrnnx {

constexpr int kVT = kVocabTile, kVS = kVocabStep, kVocabThreads = 512;
constexpr int kOperand = kVT * kVS * 2, kStage = 2 * kOperand;           // bytes of LDS

// One factor of a tile.  ALONG: rows of the source are the tile's rows (columns: the terms of the sum); else rows of the source are the terms.
// LDS, ALONG: [256 rows][64 terms], 16-byte pieces of a row exchanged by piece ^ (row & 7), so that the 16 rows of a fragment, read at one place each, lie in
// all banks.  Else [64 terms][256], pairs of pieces (16 columns, what a transposing read takes of a row) exchanged by pair ^ (bits 3, 4 and 0, 1 of the
// row): the 16 rows that such a read touches then differ in all four bits.
template <bool ALONG> struct VocabOperand {
    const char *base;                    // of the next step
    int64_t step, left;                  // bytes from step to step; terms left
    int64_t ld, outer;                   // bytes of a row; rows (ALONG) or columns of the source from the tile's first on
    uint32_t off[4];                     // this thread's pieces
    __device__ __forceinline__ void start(const VocabFactor &f, int plane, int64_t first, int64_t outer_end, int64_t k, int64_t k_end) {
        ld = f.ld * 2;
        outer = outer_end - first;
        left = k_end - k;
        base = reinterpret_cast<const char *>(f.p + plane * f.plane) + (ALONG ? first * ld + k * 2 : k * ld + first * 2);
        step = ALONG ? kVS * 2 : kVS * ld;
    }
    __device__ __forceinline__ void place() {
        const int tid = threadIdx.x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (ALONG) {
                const int row = (tid >> 3) + 64 * j, piece = (tid & 7) ^ (row & 7);
                off[j] = (uint32_t)(row * ld) + piece * 16;
            } else {
                const int row = (tid >> 5) + 16 * j, at = tid & 31, pair = (at >> 1) ^ ((row >> 3 & 3) << 2 | (row & 3)), col = pair * 16 + (at & 1) * 8;
                off[j] = col < outer ? (uint32_t)(row * ld) + col * 2 : kOutside;
            }
        }
    }
    // the next 64 terms into LDS; terms behind the last and rows behind the last read as zeros
    __device__ __forceinline__ void load(char *lds) {
        int64_t bytes = ALONG ? (outer - 1) * ld + (left + 7) / 8 * 16 : (left - 1) * ld + (outer + 7) / 8 * 16;
        bytes = left <= 0 ? 0 : bytes > 0x7fffffff ? 0x7fffffff : bytes;
        const Buffer b = buffer_of(base, bytes);
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t o = off[j];
            if (ALONG) o = ((threadIdx.x & 7) ^ (threadIdx.x >> 3 & 7)) * 8 < left ? o : kOutside;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (__attribute__((address_space(3))) void *)(lds + (j * 512 + wave * 64) * 16), 16, o, 0, 0, 0);
        }
        base += step;
        left -= kVS;
    }
    // the fragments of N times 16 rows from `row` on, of the 32 terms from 32 kk on
    template <int N> static __device__ __forceinline__ void read(const char *lds, int row, int kk, Frag (&f)[N]) {
        const int lane = threadIdx.x & 63, g = lane >> 4;
        if (ALONG) {
            const char *at = lds + (row + (lane & 15)) * 128 + (((kk * 4 + g) ^ (lane & 7)) << 4);
#pragma unroll
            for (int i = 0; i < N; ++i) f[i].v = *reinterpret_cast<const uint4 *>(at + i * 2048);
        } else {
            typedef short half4 __attribute__((ext_vector_type(4)));
            const int r = (lane & 15) >> 2, mix = g << 2 | r;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const char *at = lds + (kk * 32 + g * 8 + r) * 512 + ((((row >> 4) + i) ^ mix) << 5) + (lane & 3) * 8;
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    f[i].h[h] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) half4 *)(at + h * 2048)));
            }
        }
    }
};

struct VocabTile { int64_t m, n; };
// Tile of a workgroup.  Workgroups go to the eight dies in turn: a die takes a stretch of the tiles, eight rows of tiles at a time, so that what its 32 workgroups
// read together is in its cache.
__device__ __forceinline__ VocabTile vocab_tile(unsigned id, unsigned mt, unsigned nt) {
    const unsigned total = mt * nt, each = total / 8, rest = total % 8, die = id % 8;
    unsigned at = die * each + (die < rest ? die : rest) + id / 8;
    const unsigned width = 8 * nt, group = at / width, first = group * 8, rows = mt - first < 8 ? mt - first : 8;
    at -= group * width;
    return {(int64_t)(first + at % rows) * kVT, (int64_t)(at / rows) * kVT};
}

// acc[i][j] += sum over terms [k, k_end) of a[16 i + ..] b[16 j + ..], for this wavefront's 128 x 64 of the tile at (m, n); acc: column (n) lane % 16, rows
// (m) 4 (lane / 16) .. + 3.
template <bool AA, bool BA> __device__ __forceinline__ void vocab_product(const VocabFactor &fa, const VocabFactor &fb, int planes, VocabTile t, int64_t m_end, int64_t n_end,
                                                                          int64_t k, int64_t k_end, char *lds, f32x4 (&acc)[8][4]) {
    const int wave = threadIdx.x >> 6, wm = (wave & 1) * 128, wn = (wave >> 1) * 64;
    VocabOperand<AA> a;
    VocabOperand<BA> b;
    const int per = (int)((k_end - k + kVS - 1) / kVS), pairs = planes == 1 ? 1 : 6, steps = per * pairs;
    if (steps <= 0) return;
    int pair = 0;
    auto begin = [&]() {                                  // of planes: (0,2) (1,1) (2,0) (0,1) (1,0) (0,0), smallest products first
        const int pa = pairs == 1 ? 0 : (0x012010 >> (20 - 4 * pair)) & 15, pb = pairs == 1 ? 0 : (0x210100 >> (20 - 4 * pair)) & 15;
        a.start(fa, pa, t.m, m_end, k, k_end);
        b.start(fb, pb, t.n, n_end, k, k_end);
    };
    begin();
    a.place();
    b.place();
    a.load(lds);
    b.load(lds + kOperand);
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    int in_pair = 1;
    for (int s = 0; s < steps; ++s) {
        const char *now = lds + (s & 1) * kStage;
        if (s + 1 < steps) {
            if (in_pair == per) { in_pair = 0; ++pair; begin(); }
            ++in_pair;
            char *next = lds + ((s + 1) & 1) * kStage;
            a.load(next);
            b.load(next + kOperand);
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            Frag x[8], y[4];
            VocabOperand<BA>::read(now + kOperand, wn, kk, y);
            VocabOperand<AA>::read(now, wm, kk, x);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma(x[i], y[j], acc[i][j]);
        }
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    }
}

// What exponents are taken relative to: the largest number, 0 where there is none but -infinity (words behind the last are -infinity too).
__device__ __forceinline__ float vocab_base(float m) { return m == -INFINITY ? 0.0f : m; }

// z of a tile, words along m, rows along n
template <bool BWD> __global__ __launch_bounds__(kVocabThreads) void k_vocab_logits(const VocabParams p) {
    __shared__ __align__(16) char lds[2 * kStage];
    const unsigned mt = (unsigned)((p.V + kVT - 1) / kVT), nt = (unsigned)((p.T + kVT - 1) / kVT);
    const VocabTile t = vocab_tile(blockIdx.x, mt, nt);
    const int64_t T = p.count ? *p.count : p.T;
    if (t.n >= T) return;
    f32x4 acc[8][4] = {};
    vocab_product<true, true>(p.w, p.h, p.planes, t, p.V, T, 0, p.K, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4;
    const int64_t v0 = t.m + (wave & 1) * 128 + 4 * g, n0 = t.n + (wave >> 1) * 64 + (lane & 15);       // this lane's first word and row
    if constexpr (!BWD) {
        float *sums = reinterpret_cast<float *>(lds);     // [2][256][2]
        const int64_t left = p.V - v0;
        float most[4], sum[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t row = n0 + j * 16;
            const int64_t hit = (row < T ? p.target[row] : -1) - p.v0 - v0;
            float m = -INFINITY, z = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (16 * i + r >= left) acc[i][j][r] = -INFINITY;
                    m = fmaxf(m, acc[i][j][r]);
                    z = hit == 16 * i + r ? acc[i][j][r] : z;
                }
            if (hit >= 0 && hit < 128 && (hit & 15) < 4 && hit < left) p.hit[row] = z;
            m = fmaxf(m, __shfl_xor(m, 16, 64));
            m = fmaxf(m, __shfl_xor(m, 32, 64));
            float e = 0.0f;
            const float base = vocab_base(m);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) e += __expf(acc[i][j][r] - base);
            e += __shfl_xor(e, 16, 64);
            e += __shfl_xor(e, 32, 64);
            most[j] = m;
            sum[j] = e;
        }
        if ((wave & 1) && g == 0)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = (wave >> 1) * 64 + j * 16 + lane;
                sums[2 * at] = most[j]; sums[2 * at + 1] = sum[j];
            }
        __syncthreads();
        if (!(wave & 1) && g == 0)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = (wave >> 1) * 64 + j * 16 + lane;
                const float m2 = sums[2 * at], e2 = sums[2 * at + 1], m = fmaxf(most[j], m2), base = vocab_base(m);
                const float e = sum[j] * __expf(most[j] - base) + e2 * __expf(m2 - base);
                if (t.n + at < T) {
                    float *to = p.part + ((t.n + at) * p.parts + (p.v0 + t.m) / kVT) * 2;
                    to[0] = m; to[1] = e;
                }
            }
    } else {
        const int64_t left = p.V - v0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t row = n0 + j * 16;
            if (row >= T) continue;
            const float lse = p.row_lse[row], scale = p.row_scale[row];
            const int64_t hit = (int64_t)p.row_target[row] - p.v0 - v0;
            uint16_t *to = const_cast<uint16_t *>(p.dz.p) + row * p.ldz + v0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float d[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    d[r] = __expf(acc[i][j][r] - lse) - (hit == 16 * i + r ? 1.0f : 0.0f);
                    d[r] = 16 * i + r < left ? d[r] * scale : 0.0f;
                }
                if (p.planes == 1) *reinterpret_cast<uint2 *>(to + 16 * i) = make_uint2(pack_rne(d[0], d[1]), pack_rne(d[2], d[3]));
                else {
                    uint32_t a[3], b[3];
                    split2<3>(d[0], d[1], a);
                    split2<3>(d[2], d[3], b);
#pragma unroll
                    for (int q = 0; q < 3; ++q) *reinterpret_cast<uint2 *>(to + q * p.dz.plane + 16 * i) = make_uint2(a[q], b[q]);
                }
            }
        }
    }
}

// dh: columns of h along m, rows along n, words summed; a workgroup takes one of `splits` stretches of the words
__global__ __launch_bounds__(kVocabThreads) void k_vocab_dh(const VocabParams p) {
    __shared__ __align__(16) char lds[2 * kStage];
    const unsigned mt = (unsigned)((p.K + kVT - 1) / kVT), nt = (unsigned)((p.T + kVT - 1) / kVT), split = blockIdx.x / (mt * nt);
    const VocabTile t = vocab_tile(blockIdx.x - split * mt * nt, mt, nt);
    const int64_t T = p.count ? *p.count : p.T;
    if (t.n >= T) return;
    const int64_t each = ((p.V + kVS - 1) / kVS + p.splits - 1) / p.splits * kVS, k = split * each, end = k + each < p.V ? k + each : p.V;
    f32x4 acc[8][4] = {};
    vocab_product<false, true>(p.w, p.dz, p.planes, t, p.K, T, k, end, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c0 = t.m + (wave & 1) * 128 + 4 * (lane >> 4), n0 = t.n + (wave >> 1) * 64 + (lane & 15);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t row = n0 + j * 16;
        if (row >= T) continue;
        float *to = p.dh_part + (split * p.T + row) * p.K + c0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (c0 + 16 * i + r < p.K) to[16 * i + r] = p.first ? acc[i][j][r] : to[16 * i + r] + acc[i][j][r];
        }
    }
}

// dw: columns of h along m, words along n, rows summed
__global__ __launch_bounds__(kVocabThreads) void k_vocab_dw(const VocabParams p) {
    __shared__ __align__(16) char lds[2 * kStage];
    const unsigned mt = (unsigned)((p.K + kVT - 1) / kVT), nt = (unsigned)((p.V + kVT - 1) / kVT);
    const VocabTile t = vocab_tile(blockIdx.x, mt, nt);
    const int64_t T = p.count ? *p.count : p.T;
    f32x4 acc[8][4] = {};
    vocab_product<false, false>(p.h, p.dz, p.planes, t, p.K, p.V, 0, T, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c0 = t.m + (wave & 1) * 128 + 4 * (lane >> 4), n0 = t.n + (wave >> 1) * 64 + (lane & 15);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t word = n0 + j * 16;
        if (word >= p.V) continue;
        const int64_t at = (p.v0 + word) * p.K + c0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (c0 + 16 * i + 4 <= p.K) {
                if (p.io) Few<uint16_t, 4>::store(reinterpret_cast<uint16_t *>(p.dw) + at + 16 * i, d);
                else Few<float, 4>::store(reinterpret_cast<float *>(p.dw) + at + 16 * i, d);
            } else
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (c0 + 16 * i + r < p.K) {
                        if (p.io) store_io(reinterpret_cast<uint16_t *>(p.dw) + at + 16 * i + r, d[r]);
                        else store_io(reinterpret_cast<float *>(p.dw) + at + 16 * i + r, d[r]);
                    }
        }
    }
}

hipError_t launch_vocab_logits(const VocabParams &p, bool backward, hipStream_t s) {
    const dim3 grid((unsigned)((p.V + kVT - 1) / kVT * ((p.T + kVT - 1) / kVT))), block(kVocabThreads);
    if (backward) hipLaunchKernelGGL(k_vocab_logits<true>, grid, block, 0, s, p);
    else hipLaunchKernelGGL(k_vocab_logits<false>, grid, block, 0, s, p);
    return hipGetLastError();
}
hipError_t launch_vocab_dh(const VocabParams &p, hipStream_t s) {
    hipLaunchKernelGGL(k_vocab_dh, dim3((unsigned)((p.K + kVT - 1) / kVT * ((p.T + kVT - 1) / kVT) * p.splits)), dim3(kVocabThreads), 0, s, p);
    return hipGetLastError();
}
hipError_t launch_vocab_dw(const VocabParams &p, hipStream_t s) {
    hipLaunchKernelGGL(k_vocab_dw, dim3((unsigned)((p.K + kVT - 1) / kVT * ((p.V + kVT - 1) / kVT))), dim3(kVocabThreads), 0, s, p);
    return hipGetLastError();
}

// ---------------------------------------------------------------- copies, rows, ends
template <class IO, int NP> __global__ __launch_bounds__(256) void k_vocab_pack(const VocabPack p) {
    const int64_t rows = p.count ? *p.count : p.rows, pieces = p.Kp / 8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / pieces;
        const int c = (int)(i - row * pieces) * 8;
        const IO *from = reinterpret_cast<const IO *>(p.src) + (p.index ? p.index[row] : row) * p.ld + c;
        float x[8] = {};
        if (c + 8 <= p.K) {
            Few<IO, 4> a, b;
            a.load(from); b.load(from + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = a.get(e); x[4 + e] = b.get(e); }
        } else
#pragma unroll
            for (int e = 0; e < 8; ++e) if (c + e < p.K) x[e] = load_io(from + e);
        uint32_t w[4][NP];
#pragma unroll
        for (int e = 0; e < 4; ++e) split2<NP>(x[2 * e], x[2 * e + 1], w[e]);
#pragma unroll
        for (int q = 0; q < NP; ++q) *reinterpret_cast<uint4 *>(p.dst + q * p.plane + row * p.Kp + c) = make_uint4(w[0][q], w[1][q], w[2][q], w[3][q]);
    }
}
hipError_t launch_vocab_pack(const VocabPack &p, hipStream_t s) {
    const int64_t blocks = (p.rows * (p.Kp / 8) + 255) / 256;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536)), block(256);
    if (p.io) hipLaunchKernelGGL((k_vocab_pack<uint16_t, 1>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_vocab_pack<float, 3>), grid, block, 0, s, p);
    return hipGetLastError();
}

// The rows with a target, in their order (one workgroup: 1024 rows at a time).  A target beyond the vocabulary makes its row's gradients NaN.
__global__ __launch_bounds__(1024) void k_vocab_rows(const VocabRows p) {
    __shared__ int part[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base = 0;
    for (int64_t first = 0; first < p.T; first += 1024) {
        const int64_t t = first + threadIdx.x;
        const int64_t target = t < p.T ? p.target[t] : -1;
        const uint64_t have = __ballot(target >= 0);
        if (lane == 0) part[wave] = __popcll(have);
        __syncthreads();
        int at = base + __popcll(have & ((1ull << lane) - 1)), all = 0;
        for (int w = 0; w < 16; ++w) { if (w < wave) at += part[w]; all += part[w]; }
        base += all;
        if (t < p.T) p.place[t] = target >= 0 ? at : -1;
        if (target >= 0) {
            p.index[at] = (int)t;
            p.row_lse[at] = p.lse[t];
            p.row_scale[at] = target < p.V ? p.dloss[t * p.dloss_stride] : __builtin_nanf("");
            p.row_target[at] = target < p.V ? (int)target : -1;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) *p.count = base;
}
hipError_t launch_vocab_rows(const VocabRows &p, hipStream_t s) {
    hipLaunchKernelGGL(k_vocab_rows, dim3(1), dim3(1024), 0, s, p);
    return hipGetLastError();
}

// lse and loss of a row from its tiles' largest numbers and sums, a wavefront a row
__global__ __launch_bounds__(256) void k_vocab_loss(const VocabLoss p) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= p.T) return;
    const float2 *part = reinterpret_cast<const float2 *>(p.part) + row * p.parts;
    float m = -INFINITY;
    for (int64_t i = lane; i < p.parts; i += 64) m = fmaxf(m, part[i].x);
#pragma unroll
    for (int x = 32; x; x >>= 1) m = fmaxf(m, __shfl_xor(m, x, 64));
    float e = 0.0f;
    const float base = vocab_base(m);
    for (int64_t i = lane; i < p.parts; i += 64) e += part[i].y * expf(part[i].x - base);
#pragma unroll
    for (int x = 32; x; x >>= 1) e += __shfl_xor(e, x, 64);
    if (lane == 0) {
        const float lse = base + logf(e);
        const int64_t t = p.target[row];
        p.lse[row] = lse;
        p.loss[row] = t < 0 ? 0.0f : t < p.V ? lse - p.hit[row] : __builtin_nanf("");
    }
}
hipError_t launch_vocab_loss(const VocabLoss &p, hipStream_t s) {
    hipLaunchKernelGGL(k_vocab_loss, dim3((unsigned)((p.T + 3) / 4)), dim3(256), 0, s, p);
    return hipGetLastError();
}

// dh of all rows from the parts: zeros for rows without a target
__global__ __launch_bounds__(256) void k_vocab_dh_out(const VocabDh p) {
    const int64_t n = p.T * p.K;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / p.K;
        const int at = p.place[row];
        float s = 0.0f;
        if (at >= 0)
            for (int q = 0; q < p.splits; ++q) s += p.part[((int64_t)q * p.T + at) * p.K + (i - row * p.K)];
        if (p.io) store_io(reinterpret_cast<uint16_t *>(p.dh) + i, s);
        else store_io(reinterpret_cast<float *>(p.dh) + i, s);
    }
}
hipError_t launch_vocab_dh_out(const VocabDh &p, hipStream_t s) {
    const int64_t blocks = (p.T * p.K + 255) / 256;
    hipLaunchKernelGGL(k_vocab_dh_out, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace lrnnx
