// Softmax cross entropy over a vocabulary, logits formed a tile at a time: z = h w^T, lse = log sum exp z, loss = lse - z[target], and
//     dz = dloss (exp(z - lse) - onehot(target)),   dh = dz w,   dw = dz^T h.
// Forward: a tile of z stays in registers from its product to its largest number and sum, which is all that leaves it (8 bytes for 256 words and a row); a second
// launch joins them.  Backward: z is formed again, a piece of the vocabulary at a time, dz of the piece goes to the workspace in bfloat16 and from there into both products.  What
// that rounding takes from the target's element, and from another word's whose p is over 1/8 (eight of a row at most), is kept in float32 and added to both, and in dh a row's p are
// taken relative to what they add up to as stored: the gradients are then as exact as their own rounding to bfloat16, 1.66e-3 (all elements rounded: 2.4e-3; all but the target's, of rows that
// give another word 0.95, 2.0e-3, and 3.8e-3 or 1.1e-2 where all words have a component in common of 3 or 10 times their own norm, which has to cancel in dh).  Rows without a target are left
// out before the gradients' products: they cost nothing there and nothing in them, finite or not, reaches a gradient.
// Float32 inputs: every factor is the sum of three bfloat16 numbers, a product six of theirs (terms of 2^-24 and below are left out), summed in float32.
// Bound by the matrix units; with few rows, by the bytes of w.  8192 rows, 32768 words, 2048 elements in bfloat16: z 805 to 850 us (1290 to 1365 TFLOP/s), dz 875 to 930, dh 795 to 820, dw 970 to 1000 with half
// of the rows' targets in one tile of words, else 860 to 890; a library's products of these sizes 1295 to 1540 TFLOP/s, nothing but the product.
#include "vocab_loss.hpp"
#include "conv_common.hpp"
#include "lds_load.hpp"

namespace lrnnx {

// The tile of a product and its wavefronts: M x N, WM wavefronts along m, each 16 NI x 64 of it; STEP terms a stage, STAGES of them in LDS.
// Large: 256 x 256, eight wavefronts of 128 x 64 (128 KB of LDS). Small: 128 x 128, four of 64 x 64, two workgroups a compute unit.
// Of three planes: 256 x 128, eight of 64 x 64; all planes of a stage lie in LDS together (72 KB), so that each is loaded and read once for its six products
// (z of 997 x 5003, 771 terms: 62 us; before loads that nothing waits for 73, as six sums of a product each, tiles of 128 x 128, then 100; tiles of 128 x 128, four wavefronts with all planes, three stages, 85);
// the small one 128 x 64, four of 32 x 64, two a compute unit.
// WIDE, the first factor in float32 and split as it is read: 128 x 64, four of 32 x 64, and 64 x 64, four of 16 x 64, two a compute unit (20 rows, 151790 words, 768 terms: z 150 us,
// dh 91: 3.1 and 5.1 TB/s; all in tiles of 64 x 64, before loads that nothing waits for, 186 and 128 where this did 160 and 95; four stages of LDS, one workgroup a compute unit: 190 and 145).
template <int M_, int N_, int WM_, int PLANES_, int WIDE_ = 0> struct VocabSize {
    static constexpr bool WIDE = WIDE_ > 0, ANY = WIDE_ > 1;
    static constexpr int M = M_, N = N_, WM = WM_, PLANES = PLANES_, STEP = PLANES == 1 ? 64 : 32;
    static constexpr int NI = M / WM / 16, NJ = 4, WAVES = WM * (N / 64), THREADS = WAVES * 64;
    static constexpr int PLANE_A = M * STEP * 2, PLANE_B = N * STEP * 2, OPERAND_A = WIDE ? M * STEP * 4 : PLANES * PLANE_A, STAGE = OPERAND_A + PLANES * PLANE_B;        // bytes of LDS
    static constexpr int LOADS = STAGE / (THREADS * 16) + (ANY ? 3 * OPERAND_A / (THREADS * 16) : 0);        // of a thread and a stage
    static constexpr int PER_UNIT = M == 256 ? 1 : 2;                                 // workgroups a compute unit
};

// One factor of a tile.  ALONG: rows of the source are the tile's rows (columns: the terms of the sum); else rows of the source are the terms.
// LDS, ALONG: [ROWS rows][STEP terms], 16-byte pieces of a row exchanged by piece ^ (row & 7), or of rows of four ^ (row / 4 & 3), so that the 16 rows of a fragment,
// read at one place each, lie in all banks.  Else [STEP terms][ROWS], pairs of pieces (16 columns, what a transposing read takes of a row) exchanged by pair ^ (bits 3, 4 and 0, 1 of the
// row): the 16 rows that such a read touches then lie in different banks, too.
// WIDE: float32 elements, split as they are read; rows of 128 bytes ALONG, else groups of 16 columns exchanged by group ^ (bits 3, 4 of the row).  ANY: the same in LDS by loads of
// an element, from rows that are no 16-byte pieces at 16-byte steps (forward calls of 11 rows, 50706 words, 2801 terms 160 us; from a copy 357; of 512, 20000, 2049 282 and 320).
template <class S, int ROWS, bool ALONG, bool WIDE = false> struct VocabOperand {
    static constexpr int BYTES = WIDE ? 4 : 2, EACH = 16 / BYTES;             // bytes of an element, elements of a piece
    static constexpr bool ANY = WIDE && S::ANY;
    static constexpr int PLANE = ROWS * S::STEP * BYTES, LOADS = PLANE / (S::THREADS * (ANY ? 4 : 16));
    const char *base;                    // of the next stage
    int64_t step, left;                  // bytes from stage to stage; terms left
    int64_t ld, outer;                   // bytes of a row; rows (ALONG) or columns of the source from the tile's first on
    int64_t plane;                       // bytes from plane to plane
    uint32_t off[ANY ? 4 : LOADS];       // this thread's pieces; ANY: of load j the one at ALONG 0, else (j's row >> 3) & 3, and so many rows on
    static constexpr int PIECES = S::STEP / EACH;         // of a row, ALONG
    static __device__ __forceinline__ int turned(int row) { return PIECES == 8 ? row & 7 : row >> 2 & 3; }
    static __device__ __forceinline__ int mixed(int row) {
        if (WIDE) return row >> 3 & 3;
        if (ROWS == 64) return (row >> 3 & 1) << 1 | (row >> 1 & 1);         // (two rows side by side in the banks)
        return ((row >> 3 & 3) << 2 | (row & 3)) & (ROWS / 16 - 1);
    }
    __device__ __forceinline__ void start(const VocabFactor &f, int64_t first, int64_t outer_end, int64_t k, int64_t k_end) {
        ld = f.ld * BYTES;
        plane = f.plane * 2;
        outer = outer_end - first;
        left = k_end - k;
        base = reinterpret_cast<const char *>(f.p) + (ALONG ? first * ld + k * BYTES : k * ld + first * BYTES);
        step = ALONG ? S::STEP * BYTES : S::STEP * ld;
        const int tid = threadIdx.x;
        if constexpr (ANY) {
            constexpr int ROW = ALONG ? S::STEP : ROWS, EVERY = S::THREADS / ROW;             // elements of a row, rows of a load
            static_assert(ALONG ? EVERY == 8 && PIECES == 8 : EVERY <= 8, "");              // (of which the exchange is the same for all loads, or for all rows)
            const int row = tid / ROW, at = tid % ROW;
#pragma unroll
            for (int m = 0; m < (ALONG ? 1 : 4); ++m) {
                const int e = ALONG ? ((at >> 2) ^ turned(row)) * 4 + (at & 3) : ((at >> 4) ^ m) * 16 + (at & 15);
                off[m] = ALONG || e < outer ? (uint32_t)(row * ld) + e * 4 : kOutside;
            }
        } else
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            if (ALONG) {
                const int row = tid / PIECES + S::THREADS / PIECES * j, piece = (tid % PIECES) ^ turned(row);
                off[j] = (uint32_t)(row * ld) + piece * 16;
            } else {
                constexpr int ROW = ROWS / EACH, GROUP = 16 / EACH;          // pieces of a row, of 16 columns
                const int row = tid / ROW + S::THREADS / ROW * j, at = tid % ROW, col = ((at / GROUP) ^ mixed(row)) * 16 + at % GROUP * EACH;
                off[j] = col < outer ? (uint32_t)(row * ld) + col * BYTES : kOutside;
            }
        }
    }
    // the next 64 terms into LDS; terms behind the last and rows behind the last read as zeros
    __device__ __forceinline__ void load(char *lds) {
        constexpr int WHOLE = ANY ? 1 : EACH;
        int64_t bytes = ALONG ? (outer - 1) * ld + (left + WHOLE - 1) / WHOLE * WHOLE * BYTES : (left - 1) * ld + (outer + WHOLE - 1) / WHOLE * WHOLE * BYTES;
        bytes = left <= 0 ? 0 : bytes > 0x7fffffff ? 0x7fffffff : bytes;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int q = 0; q < (WIDE ? 1 : S::PLANES); ++q) {
            const char *at = base + q * plane;
            const u32x4 b = {(uint32_t)(uintptr_t)at, (uint32_t)((uintptr_t)at >> 32) & 0xffff, (uint32_t)bytes, 0x00020000};       // as of buffer_of
            const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)(lds + q * PLANE + wave * (ANY ? 256 : 1024));
            if constexpr (ANY) {
                constexpr int EVERY = S::THREADS / (ALONG ? S::STEP : ROWS);
                const bool there = !ALONG || ((threadIdx.x % S::STEP >> 2) ^ turned(threadIdx.x / S::STEP)) * 4 + (threadIdx.x & 3) < left;
#pragma unroll
                for (int j = 0; j < LOADS; j += 4) {
                    uint32_t o[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = there ? off[ALONG ? 0 : EVERY * (j + i) >> 3 & 3] + (uint32_t)(EVERY * (j + i) * ld) : kOutside;
                    load_lds<4, S::THREADS * 4, 4>(to + j * S::THREADS * 4, b, o);
                }
            } else {
                uint32_t o[LOADS];
#pragma unroll
                for (int j = 0; j < LOADS; ++j) {
                    o[j] = off[j];
                    if (ALONG) o[j] = ((threadIdx.x % PIECES) ^ turned(threadIdx.x / PIECES)) * EACH < left ? o[j] : kOutside;
                }
                load_lds<LOADS, S::THREADS * 16>(to, b, o);
            }
        }
        base += step;
        left -= S::STEP;
    }
    // the fragments of N times 16 rows from `row` on, of the 32 terms from 32 kk on
    template <int N> static __device__ __forceinline__ void read(const char *lds, int row, int kk, Frag (&f)[N]) {
        static_assert(!WIDE, "");
        const int lane = threadIdx.x & 63, g = lane >> 4;
        if (ALONG) {
            constexpr int ROW = S::STEP * 2;
            const char *at = lds + (row + (lane & 15)) * ROW + (((kk * 4 + g) ^ turned(lane & 15)) << 4);
#pragma unroll
            for (int i = 0; i < N; ++i) f[i].v = *reinterpret_cast<const uint4 *>(at + i * 16 * ROW);
        } else {
            typedef short half4 __attribute__((ext_vector_type(4)));
            constexpr int ROW = ROWS * 2;
            const int r = (lane & 15) >> 2, mix = mixed(g << 3 | r);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const char *at = lds + (kk * 32 + g * 8 + r) * ROW + ((((row >> 4) + i) ^ mix) << 5) + (lane & 3) * 8;
#pragma unroll
                for (int h = 0; h < 2; ++h)       // four lanes a row of four terms: a lane gets its column's
                    f[i].h[h] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) half4 *)(at + h * 4 * ROW)));
            }
        }
    }
    // the same of a stage of float32 elements, not yet split
    template <int N> static __device__ __forceinline__ void read_wide(const char *lds, int row, float (&x)[N][8]) {
        static_assert(WIDE, "");
        const int lane = threadIdx.x & 63, g = lane >> 4;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (ALONG) {
                const char *at = lds + (row + i * 16 + (lane & 15)) * (S::STEP * 4);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4 v = *reinterpret_cast<const f32x4 *>(at + (((2 * g + h) ^ turned(lane & 15)) << 4));
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i][4 * h + e] = v[e];
                }
            } else {
                const char *at = lds + g * 8 * (ROWS * 4) + ((((row >> 4) + i) ^ mixed(g << 3)) << 6) + (lane & 15) * 4;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] = *reinterpret_cast<const float *>(at + e * (ROWS * 4));
            }
    }
};

struct VocabTile { int64_t m, n; };
// The tiles of a product in the order in which they are taken.  Workgroups go to the eight dies in turn: a die takes a stretch of the tiles, four rows of tiles at
// a time, so that what its 32 compute units read together (4 x 8 tiles) is in its cache: 32768 x 8192 with 2048 terms 1172 TFLOP/s, eight rows 1007 (of an earlier kernel,
// now 1330).
template <class S> struct VocabTiles {
    unsigned mt, nt, total;
    __device__ __forceinline__ VocabTiles(int64_t m, int64_t n) : mt((unsigned)((m + S::M - 1) / S::M)), nt((unsigned)((n + S::N - 1) / S::N)), total(mt * nt) {}
    // first tile and number of tiles of a die
    __device__ __forceinline__ unsigned first(unsigned die) const { const unsigned rest = total % 8; return die * (total / 8) + (die < rest ? die : rest); }
    __device__ __forceinline__ unsigned count(unsigned die) const { return total / 8 + (die < total % 8 ? 1 : 0); }
    __device__ __forceinline__ VocabTile tile(unsigned at) const {
        const unsigned width = 4 * nt, group = at / width, row = group * 4, rows = mt - row < 4 ? mt - row : 4;
        at -= group * width;
        return {(int64_t)(row + at % rows) * S::M, (int64_t)(at / rows) * S::N};
    }
};

// The factors of a workgroup's tiles, a stage after the other: of one tile, then of the next; behind the last, zeros.
template <class S, bool AA, bool BA> struct VocabFeed {
    VocabFactor fa, fb;
    int64_t m_end, n_end, k, k_end;
    int stages, coming;                  // of a tile; the next stage
    VocabTile t;
    VocabOperand<S, S::M, AA, S::WIDE> a;
    VocabOperand<S, S::N, BA> b;
    __device__ __forceinline__ VocabFeed(const VocabFactor &fa, const VocabFactor &fb, int64_t m_end, int64_t n_end, int64_t k, int64_t k_end)
        : fa(fa), fb(fb), m_end(m_end), n_end(n_end), k(k), k_end(k_end), stages((int)((k_end - k + S::STEP - 1) / S::STEP)) {}
    __device__ __forceinline__ void start() {
        a.start(fa, t.m, m_end, k, k_end);
        b.start(fb, t.n, n_end, k, k_end);
        coming = 0;
    }
    // `next`: sets t to the next tile, false if there is none
    template <class F> __device__ __forceinline__ void fetch(char *lds, int halves, F next) {
        if (halves & 1) {
            if (coming == stages && next()) start();
            ++coming;
            a.load(lds);
        }
        if (halves & 2) b.load(lds + S::OPERAND_A);
    }
};

// acc[i][j] += sum over the terms of a[16 i + ..] b[16 j + ..], for this wavefront's part of the tile; acc: column (n) lane % 16, rows (m) 4 (lane / 16) .. + 3.
// Two stages of LDS; fragments are read half a stage ahead of the instructions that use them, and a stage's memory is filled again as soon as its second half
// is in registers, two halves before it is read: one barrier a stage.  z of 8192 x 32768, 2048 terms: 1290 to 1365 TFLOP/s, dh 1340 to 1385.  Before other changes here: reads at the end of a half, where the compiler puts them if
// left to itself: z 50 us of 980 slower; four stages of 32 terms, a barrier each: z 987 for 903, dh 863 for 828 (half as long rows a load); and so that half of the wavefronts
// read while the others multiply, two barriers each: 1070 and 900.  With four wavefronts of 128 x 128 a third fewer reads, but 256 sums and two sets of fragments do not fit the registers.
template <class S, bool AA, bool BA, int KIND = S::WIDE ? 0 : S::PLANES> struct VocabPipe {
    // matrix instructions that go before the loads of a stage's first and second factor, four each, so that the matrix unit has work while they are issued.  (Transposing reads are twice as
    // many, and need the others beside them.)  z of 8192 x 32768, 2048 terms: none before 906 us, so 845; dh 828 and 818, with loads later 866.
    static constexpr int FIRST = AA && BA ? S::NI / 4 : 1, NEXT = AA && BA ? S::NI / 2 : 1;
    char *lds;
    int wm, wn, now;                     // rows and columns of this wavefront; the stage whose first half is in x0, y0
    Frag x0[S::NI], y0[S::NJ];
    __device__ __forceinline__ VocabPipe(char *lds) : lds(lds), now(0) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wm = wave % S::WM * (S::M / S::WM);
        wn = wave / S::WM * 64;
    }
    __device__ __forceinline__ void read(int stage, int kk, Frag (&x)[S::NI], Frag (&y)[S::NJ]) {
        const char *at = lds + stage * S::STAGE;
        VocabOperand<S, S::N, BA>::read(at + S::OPERAND_A, wn, kk, y);
        VocabOperand<S, S::M, AA>::read(at, wm, kk, x);
    }
    template <int FROM = 0, int TO = S::NI> static __device__ __forceinline__ void sums(const Frag (&x)[S::NI], const Frag (&y)[S::NJ], f32x4 (&acc)[S::NI][S::NJ]) {
#pragma unroll
        for (int i = FROM; i < TO; ++i)
#pragma unroll
            for (int j = 0; j < S::NJ; ++j) acc[i][j] = mfma(x[i], y[j], acc[i][j]);
    }
    // reads spread evenly between the matrix instructions
    template <int FROM = 0> static __device__ __forceinline__ void spread() {
        constexpr int MATRIX = (S::NI - FROM) * S::NJ, READS = (AA ? S::NI : 2 * S::NI) + (BA ? S::NJ : 2 * S::NJ), PER = MATRIX / READS;
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, MATRIX - PER * READS, 0);
        __builtin_amdgcn_sched_barrier(0);
    }
    template <class Fetch> __device__ __forceinline__ void prime(Fetch fetch) {
        fetch(lds);
        __builtin_amdgcn_sched_barrier(0);        // (the wait counts the second stage's loads)
        fetch(lds + S::STAGE);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(S::LOADS) : "memory");
        read(0, 0, x0, y0);
    }
    template <class Fetch> __device__ __forceinline__ void run(int stages, f32x4 (&acc)[S::NI][S::NJ], Fetch fetch) {
        for (int s = 0; s < stages; ++s) {
            Frag x1[S::NI], y1[S::NJ];
            read(now, 1, x1, y1);
            sums(x0, y0, acc);
            spread();
            // the other stage has come, and this one is in everyone's registers
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            sums<0, FIRST>(x1, y1, acc);
            __builtin_amdgcn_sched_barrier(0);
            fetch(lds + now * S::STAGE, 1);
            __builtin_amdgcn_sched_barrier(0);
            sums<FIRST, NEXT>(x1, y1, acc);
            __builtin_amdgcn_sched_barrier(0);
            fetch(lds + now * S::STAGE, 2);
            __builtin_amdgcn_sched_barrier(0);
            read(now ^ 1, 0, x0, y0);
            sums<NEXT>(x1, y1, acc);
            spread<NEXT>();
            now ^= 1;
        }
    }
    // nothing on its way, and LDS free for the whole workgroup
    __device__ __forceinline__ void end() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
};

// Of three planes: a stage is one set of fragments, six products of 16 matrix instructions each, smallest first.  The next stage's fragments are read as this one's are
// used up, so that both fit the registers but for one plane of each factor; a stage's memory is filled again when it is in everyone's registers.
template <class S, bool AA, bool BA> struct VocabPipe<S, AA, BA, 3> {
    struct Set { Frag x[3][S::NI], y[3][S::NJ]; };
    char *lds;
    int wm, wn, now;                     // the stage that is in `f`
    Set f;
    using A = VocabOperand<S, S::M, AA>;
    using B = VocabOperand<S, S::N, BA>;
    __device__ __forceinline__ VocabPipe(char *lds) : lds(lds), now(0) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wm = wave % S::WM * (S::M / S::WM);
        wn = wave / S::WM * 64;
    }
    template <class Fetch> __device__ __forceinline__ void prime(Fetch fetch) {
        fetch(lds);
        __builtin_amdgcn_sched_barrier(0);        // (the wait counts the second stage's loads)
        fetch(lds + S::STAGE);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(S::LOADS) : "memory");
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            B::read(lds + S::OPERAND_A + q * S::PLANE_B, wn, 0, f.y[q]);
            A::read(lds + q * S::PLANE_A, wm, 0, f.x[q]);
        }
    }
    template <int FROM = 0, int TO = S::NI> static __device__ __forceinline__ void product(const Set &s, int pa, int pb, f32x4 (&acc)[S::NI][S::NJ]) {
#pragma unroll
        for (int i = FROM; i < TO; ++i)
#pragma unroll
            for (int j = 0; j < S::NJ; ++j) acc[i][j] = mfma(s.x[pa][i], s.y[pb][j], acc[i][j]);
    }
    template <class Fetch> __device__ __forceinline__ void stage(const Set &s, Set &to, f32x4 (&acc)[S::NI][S::NJ], Fetch fetch) {
        product(s, 0, 2, acc);
        __builtin_amdgcn_sched_barrier(0);
        // the other stage has come, and this one is in everyone's registers
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const char *a = lds + (now ^ 1) * S::STAGE, *b = a + S::OPERAND_A;
        product<0, 1>(s, 1, 1, acc);
        __builtin_amdgcn_sched_barrier(0);
        fetch(lds + now * S::STAGE);
        B::read(b + 2 * S::PLANE_B, wn, 0, to.y[2]);
        product<1>(s, 1, 1, acc);
        __builtin_amdgcn_sched_barrier(0);
        A::read(a, wm, 0, to.x[0]);
        product(s, 2, 0, acc);
        __builtin_amdgcn_sched_barrier(0);
        A::read(a + 2 * S::PLANE_A, wm, 0, to.x[2]);
        product(s, 0, 1, acc);
        __builtin_amdgcn_sched_barrier(0);
        B::read(b + S::PLANE_B, wn, 0, to.y[1]);
        product(s, 1, 0, acc);
        __builtin_amdgcn_sched_barrier(0);
        A::read(a + S::PLANE_A, wm, 0, to.x[1]);
        B::read(b, wn, 0, to.y[0]);
        product(s, 0, 0, acc);
        __builtin_amdgcn_sched_barrier(0);
        now ^= 1;
    }
    template <class Fetch> __device__ __forceinline__ void run(int stages, f32x4 (&acc)[S::NI][S::NJ], Fetch fetch) {
        Set g;
        for (; stages > 1; stages -= 2) {         // (a copy of a register that is on its way would wait for it: z of 2000 x 15179, 768 terms 272 us so, 257)
            stage(f, g, acc, fetch);
            stage(g, f, acc, fetch);
        }
        if (stages > 0) {
            stage(f, g, acc, fetch);
            f = g;
        }
    }
    __device__ __forceinline__ void end() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
};

// Of a float32 factor as it lies and three planes of the other: a wavefront splits what it has read of a stage, while the next two are on their way.  For few rows: every
// element of the first factor is split once, and its bytes are what a product costs.
template <class S, bool AA, bool BA> struct VocabPipe<S, AA, BA, 0> {
    char *lds;
    int wm, wn, now;
    using A = VocabOperand<S, S::M, AA, true>;
    using B = VocabOperand<S, S::N, BA>;
    __device__ __forceinline__ VocabPipe(char *lds) : lds(lds), now(0) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wm = wave % S::WM * (S::M / S::WM);
        wn = wave / S::WM * 64;
    }
    template <class Fetch> __device__ __forceinline__ void prime(Fetch fetch) {
        fetch(lds);
        __builtin_amdgcn_sched_barrier(0);        // (the waits count the second stage's loads)
        fetch(lds + S::STAGE);
        __builtin_amdgcn_sched_barrier(0);
    }
    template <class Fetch> __device__ __forceinline__ void run(int stages, f32x4 (&acc)[S::NI][S::NJ], Fetch fetch) {
        for (int s = 0; s < stages; ++s) {
            float raw[S::NI][8];
            Frag x[3][S::NI], y[3][S::NJ];
            const char *at = lds + now * S::STAGE;
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(S::LOADS) : "memory");
            A::read_wide(at, wm, raw);
#pragma unroll
            for (int q = 0; q < 3; ++q) B::read(at + S::OPERAND_A + q * S::PLANE_B, wn, 0, y[q]);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");        // (in everyone's registers)
            fetch(lds + now * S::STAGE);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < S::NI; ++i) {
                uint32_t w[4][3];
#pragma unroll
                for (int e = 0; e < 4; ++e) split2<3>(raw[i][2 * e], raw[i][2 * e + 1], w[e]);
#pragma unroll
                for (int q = 0; q < 3; ++q) x[q][i].v = make_uint4(w[0][q], w[1][q], w[2][q], w[3][q]);
            }
            constexpr int order[6][2] = {{0, 2}, {1, 1}, {2, 0}, {0, 1}, {1, 0}, {0, 0}};         // smallest first
#pragma unroll
            for (int o = 0; o < 6; ++o)
#pragma unroll
                for (int i = 0; i < S::NI; ++i)
#pragma unroll
                    for (int j = 0; j < S::NJ; ++j) acc[i][j] = mfma(x[order[o][0]][i], y[order[o][1]][j], acc[i][j]);
            now ^= 1;
        }
    }
    __device__ __forceinline__ void end() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
};

// One tile's product.
template <class S, bool AA, bool BA> __device__ __forceinline__ void vocab_product(const VocabFactor &fa, const VocabFactor &fb, VocabTile t, int64_t m_end, int64_t n_end, int64_t k, int64_t k_end, char *lds, f32x4 (&acc)[S::NI][S::NJ]) {
    VocabFeed<S, AA, BA> feed(fa, fb, m_end, n_end, k, k_end);
    if (feed.stages <= 0) return;
    feed.t = t;
    feed.start();
    VocabPipe<S, AA, BA> pipe(lds);
    auto fetch = [&](char *to, int halves = 3) __attribute__((always_inline)) { feed.fetch(to, halves, [] { return false; }); };
    pipe.prime(fetch);
    pipe.run(feed.stages, acc, fetch);
    pipe.end();
}

// What exponents are taken relative to: the largest number, 0 where there is none but -infinity (words behind the last are -infinity too).
__device__ __forceinline__ float vocab_base(float m) { return m == -INFINITY ? 0.0f : m; }
// e^x: of float32 inputs to 1 ulp; else by the hardware's power of two, off by |x| 2^-23.5 where x's product with log2(e) is rounded: nothing beside the results' bfloat16
template <int PLANES> __device__ __forceinline__ float vocab_exp(float x) { return PLANES == 3 ? expf(x) : __expf(x); }

// four elements, or as many of them as are left
template <class IO> __device__ __forceinline__ void store_part(IO *to, const float (&x)[4], int64_t left) {
    if (left >= 4) Few<IO, 4>::store(to, x);
    else
#pragma unroll
        for (int r = 0; r < 4; ++r) if (r < left) store_io(to + r, x[r]);
}
// The place of this wavefront in a tile, and this lane's first row and column of it
template <class S> struct VocabPlace {
    int wave, m, n;
    __device__ __forceinline__ VocabPlace() {
        const int lane = threadIdx.x & 63;
        wave = threadIdx.x >> 6;
        m = wave % S::WM * (S::M / S::WM) + 4 * (lane >> 4);
        n = wave / S::WM * 64 + (lane & 15);
    }
};
// e^(x - base)
template <int PLANES> struct VocabExp {
    float base;                          // (times log2(e), but for float32 inputs)
    __device__ __forceinline__ VocabExp(float b) : base(PLANES == 3 ? b : b * -1.44269504f) {}
    __device__ __forceinline__ float operator()(float x) const { return PLANES == 3 ? expf(x - base) : __builtin_amdgcn_exp2f(__builtin_fmaf(x, 1.44269504f, base)); }
};
// What comes of a tile of z, words along m, rows along n: forward, the largest number and the sum of exponentials of every row.  (Its 128 numbers a lane are an eighth of a tile's time: what
// only the last tile of the vocabulary and what only a target's tile needs is apart.)
template <class S> __device__ __forceinline__ void vocab_sums(const VocabParams &p, VocabTile t, int64_t T, float2 *sums, f32x4 (&acc)[S::NI][S::NJ]) {
    const VocabPlace<S> at;
    const int64_t v0 = t.m + at.m, n0 = t.n + at.n, left = p.V - v0;
    if (t.m + S::M > p.V)
#pragma unroll
        for (int i = 0; i < S::NI; ++i)
#pragma unroll
            for (int j = 0; j < S::NJ; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) if (16 * i + r >= left) acc[i][j][r] = -INFINITY;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
        const int64_t row = n0 + j * 16;
        const int64_t hit = (row < T ? p.target[row] : -1) - p.v0 - v0;
        const bool here = hit >= 0 && hit < S::M / S::WM && (hit & 15) < 4 && hit < left;
        if (__any(here)) {
            float z = 0.0f;
#pragma unroll
            for (int i = 0; i < S::NI; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) z = hit == 16 * i + r ? acc[i][j][r] : z;
            if (here) p.hit[row] = z;
        }
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < S::NI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) m = fmaxf(m, acc[i][j][r]);
        m = fmaxf(m, __shfl_xor(m, 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        float e = 0.0f;
        const VocabExp<S::PLANES> exponential(vocab_base(m));
#pragma unroll
        for (int i = 0; i < S::NI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) e += exponential(acc[i][j][r]);
        e += __shfl_xor(e, 16, 64);
        e += __shfl_xor(e, 32, 64);
        if ((threadIdx.x & 48) == 0) sums[at.wave % S::WM * S::N + at.n + j * 16] = make_float2(m, e);
    }
    lds_barrier();
    const int n = threadIdx.x;
    if (n < S::N && t.n + n < T) {
        float m = sums[n].x, e = 0.0f;
#pragma unroll
        for (int w = 1; w < S::WM; ++w) m = fmaxf(m, sums[w * S::N + n].x);
        const float base = vocab_base(m);
#pragma unroll
        for (int w = 0; w < S::WM; ++w) e += sums[w * S::N + n].y * vocab_exp<S::PLANES>(sums[w * S::N + n].x - base);
        reinterpret_cast<float2 *>(p.part)[(t.n + n) * p.parts + (p.v0 + t.m) / S::M] = make_float2(m, e);
    }
}
// and backward, dz
template <int PLANES> __device__ __forceinline__ void store_dz(uint16_t *to, int64_t plane, const float (&d)[4]) {
    uint32_t a[PLANES], b[PLANES];
    split2<PLANES>(d[0], d[1], a);
    split2<PLANES>(d[2], d[3], b);
#pragma unroll
    for (int q = 0; q < PLANES; ++q) *reinterpret_cast<uint2 *>(to + q * plane) = make_uint2(a[q], b[q]);
}
// what rounding to bfloat16 leaves of a number
__device__ __forceinline__ float vocab_rest(float d) {
    const float there = __uint_as_float(pack_rne(d, 0.0f) << 16);
    return fabsf(there) < INFINITY ? d - there : 0.0f;
}
// The rest of a word that is likely without being the target.  Several wavefronts add to a row's, in any order: they are sorted before they are used.
__device__ __forceinline__ void vocab_other(const VocabParams &p, int64_t row, int64_t word, float d) {
    const int at = atomicAdd(p.row_others + row, 1) + 1;
    if (at < kVocabRests) p.rests[row * kVocabRests + at] = {(int)word, vocab_rest(d)};
}
// The rests that a column of a tile has: its lanes' targets' and those of likely words.  (Few tiles have any: small code counts for more here than few instructions.)
template <class S> __device__ __forceinline__ void vocab_column_rests(const VocabParams &p, int64_t row, int64_t v0, const f32x4 (&acc)[S::NI][S::NJ], int j) {
    const float lse = p.row_lse[row], scale = p.row_scale[row], likely = lse + __logf(kVocabLikely);
    const int hit = p.row_target[row] - (int)(p.v0 + v0), left = (int)(p.V - v0);
    const VocabExp<S::PLANES> exponential(lse);
    uint32_t found = hit >= 0 && hit < S::M / S::WM && (hit & 15) < 4 ? 1u << ((hit >> 4) * 4 + (hit & 3)) : 0;
#pragma unroll
    for (int i = 0; i < S::NI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            found |= acc[i][j][r] > likely ? 1u << (4 * i + r) : 0;
            asm volatile("" : "+v"(found));                // (one after the other: 32 masks at once are 64 registers)
        }
    for (; found; found &= found - 1) {
        const int at = __builtin_ctz(found), word = (at >> 2) * 16 + (at & 3);
        float z = 0.0f;
#pragma unroll
        for (int i = 0; i < S::NI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                z = at == 4 * i + r ? acc[i][j][r] : z;
                asm volatile("" : "+v"(z));
            }
        const float x = exponential(z);
        if (word >= left) break;                           // (words beyond the last)
        if (word == hit) p.rests[row * kVocabRests].rest = vocab_rest((x - 1.0f) * scale);
        else vocab_other(p, row, p.v0 + v0 + word, x * scale);
    }
}
// Whether there may be rests in the column.
template <class S, bool APART> __device__ __forceinline__ bool vocab_dz_column(const VocabParams &p, bool there, int64_t row, int64_t v0, int64_t left, int64_t hit, const VocabExp<S::PLANES> &exponential,
                                                                               float scale, f32x4 (&acc)[S::NI][S::NJ], int j) {
#pragma clang fp contract(off)           // (a product fused into its own split would differ between the two forms, and so with the targets of other rows)
    const int g = threadIdx.x >> 4 & 3;
    uint16_t *to = const_cast<uint16_t *>(p.dz.p) + row * p.dz.ld + v0 - 4 * g;
    uint2 part[S::PLANES][S::NI];
#pragma unroll
    for (int i = 0; i < S::NI; ++i) {
        float d[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            d[r] = exponential(acc[i][j][r]);
            if (APART && hit == 16 * i + r) d[r] -= 1.0f;
            d[r] *= scale;
            if (APART && 16 * i + r >= left) d[r] = 0.0f;
        }
        uint32_t a[S::PLANES], b[S::PLANES];
        split2<S::PLANES>(d[0], d[1], a);
        split2<S::PLANES>(d[2], d[3], b);
#pragma unroll
        for (int q = 0; q < S::PLANES; ++q) part[q][i] = make_uint2(a[q], b[q]);
    }
    bool rests = false;
    if constexpr (S::PLANES == 1) {
        // the sum over this wavefront's words of what is stored, as a product with ones: (which terms a lane holds is the same to a sum)
        Frag ones;
        ones.v = make_uint4(0x3f803f80, 0x3f803f80, 0x3f803f80, 0x3f803f80);
        f32x4 sum = {};
#pragma unroll
        for (int i = 0; i < S::NI; i += 2) {
            Frag f;
            f.h[0] = part[0][i];
            f.h[1] = part[0][i + 1];
            sum = mfma(ones, f, sum);
        }
        if (there && g == 0) p.sum_part[(v0 >> (S::M / S::WM == 128 ? 7 : 6)) * p.T + row] = sum[0];
        rests = there && (APART || fabsf(sum[0]) > 0.96f * kVocabLikely * fabsf(scale));     // (without a likely word they add up to less, rounded as they are)
    }
    if (!there) return false;
#pragma unroll
    for (int q = 0; q < S::PLANES; ++q) {
        if constexpr (S::NI % 2 == 0) {
            // of two times 16 words a lane has four each; eight of one of them, for one access, by an exchange with the lane 16 further on or back
#pragma unroll
            for (int i = 0; i < S::NI; i += 2) {
                const auto x = __builtin_amdgcn_permlane16_swap(part[q][i].x, part[q][i + 1].x, false, false), y = __builtin_amdgcn_permlane16_swap(part[q][i].y, part[q][i + 1].y, false, false);
                *reinterpret_cast<uint4 *>(to + q * p.dz.plane + 16 * (i + (g & 1)) + 8 * (g >> 1)) = make_uint4(x[0], y[0], x[1], y[1]);
            }
        } else
#pragma unroll
            for (int i = 0; i < S::NI; ++i) *reinterpret_cast<uint2 *>(to + q * p.dz.plane + 16 * i + 4 * g) = part[q][i];
    }
    return rests;
}
template <class S> __device__ __forceinline__ void vocab_dz(const VocabParams &p, VocabTile t, int64_t T, f32x4 (&acc)[S::NI][S::NJ]) {
    const VocabPlace<S> at;
    const int64_t v0 = t.m + at.m, n0 = t.n + at.n, left = p.V - v0;
    uint32_t rests = 0;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
        const int64_t row = n0 + j * 16;
        const bool there = row < T;
        const float lse = there ? p.row_lse[row] : 0.0f, scale = there ? p.row_scale[row] : 0.0f;
        const int64_t hit = (there ? (int64_t)p.row_target[row] : -1) - p.v0 - v0;
        const bool apart = t.m + S::M > p.V || __any(hit >= 0 && hit < S::M / S::WM && (hit & 15) < 4);
        const VocabExp<S::PLANES> exponential(lse);
        bool some;
        if (apart) some = vocab_dz_column<S, true>(p, there, row, v0, left, hit, exponential, scale, acc, j);
        else some = vocab_dz_column<S, false>(p, there, row, v0, left, hit, exponential, scale, acc, j);
        rests |= some ? 1u << j : 0;
    }
    if constexpr (S::PLANES == 1)
        if (__any(rests != 0))
#pragma unroll
            for (int j = 0; j < S::NJ; ++j)
                if (rests >> j & 1) vocab_column_rests<S>(p, n0 + j * 16, v0, acc, j);
}
// A workgroup stays and takes a tile after the other; the next one's factors are on their way while it works on what comes of the one before.
template <class S, bool BWD> __global__ __launch_bounds__(S::THREADS) void k_vocab_logits(const VocabParams p) {
    __shared__ __align__(16) char lds[2 * S::STAGE];
    __shared__ float2 sums[S::WM * S::N];
    const int64_t T = p.count ? *p.count : p.T;
    const VocabTiles<S> tiles(p.V, T);
    const unsigned die = blockIdx.x & 7, first = tiles.first(die), count = tiles.count(die), turn = gridDim.x / 8;
    unsigned at = blockIdx.x >> 3, coming = at;
    if (at >= count) return;
    VocabFeed<S, true, true> feed(p.w, p.h, p.V, T, 0, p.K);
    feed.t = tiles.tile(first + at);
    feed.start();
    VocabPipe<S, true, true> pipe(lds);
    auto next = [&]() __attribute__((always_inline)) {
        coming += turn;
        if (coming >= count) return false;
        feed.t = tiles.tile(first + coming);
        return true;
    };
    auto fetch = [&](char *to, int halves = 3) __attribute__((always_inline)) { feed.fetch(to, halves, next); };
    pipe.prime(fetch);
    for (; at < count; at += turn) {
        f32x4 acc[S::NI][S::NJ] = {};
        pipe.run(feed.stages, acc, fetch);
        const VocabTile t = tiles.tile(first + at);
        if constexpr (BWD) vocab_dz<S>(p, t, T, acc);
        else vocab_sums<S>(p, t, T, sums, acc);
    }
    pipe.end();
}

// A sum over stretches of its terms side by side: which tile and stretch a workgroup takes.  The tiles of a stretch read the same rows and so stay on few dies.
template <class S> struct VocabUnit {
    VocabTile t;
    int64_t split, k, end;
    bool there;
    __device__ __forceinline__ VocabUnit(int64_t m, int64_t n, int splits, int64_t terms) {
        VocabTiles<S> units(m, n);
        const unsigned tiles = units.total;
        units.total = tiles * splits;
        const unsigned die = blockIdx.x & 7, at = blockIdx.x >> 3;
        there = at < units.count(die);
        if (!there) return;
        const unsigned unit = units.first(die) + at;
        split = unit / tiles;
        t = units.tile(unit % tiles);
        const int64_t each = ((terms + S::STEP - 1) / S::STEP + splits - 1) / splits * S::STEP;
        k = split * each;
        end = k + each < terms ? k + each : terms;
    }
};

// z in stretches of its terms side by side, where there are few tiles: words along m, rows along n (1 row, 2594 words, 3712 terms in float32: 13 us and 7 for what comes of it;
// in one stretch 90)
template <class S> __global__ __launch_bounds__(S::THREADS) void k_vocab_part(const VocabParams p) {
    __shared__ __align__(16) char lds[2 * S::STAGE];
    const int64_t T = p.count ? *p.count : p.T;
    const VocabUnit<S> u(p.V, T, p.splits_z, p.K);
    if (!u.there) return;
    f32x4 acc[S::NI][S::NJ] = {};
    vocab_product<S, true, true>(p.w, p.h, u.t, p.V, T, u.k, u.end, lds, acc);
    const VocabPlace<S> place;
    const int64_t v0 = u.t.m + place.m, n0 = u.t.n + place.n;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
        const int64_t row = n0 + j * 16;
        if (row >= T) continue;
        float *to = p.z_part + (u.split * p.T + row) * p.ldz + v0;
#pragma unroll
        for (int i = 0; i < S::NI; ++i)
            if (v0 + 16 * i < p.ldz) *reinterpret_cast<f32x4 *>(to + 16 * i) = acc[i][j];
    }
}
// What comes of it, as of a tile of z: forward a workgroup or (few words) a wavefront a row, backward eight words a thread
__device__ __forceinline__ f32x4 vocab_z(const VocabParams &p, int64_t row, int64_t word) {
    const float *from = p.z_part + row * p.ldz + word;
    f32x4 z = {};
#pragma unroll 8
    for (int q = 0; q < p.splits_z; ++q) z += *reinterpret_cast<const f32x4 *>(from + q * p.T * p.ldz);
    return z;
}
template <int PLANES, int WAVES> __global__ __launch_bounds__(512) void k_vocab_part_sums(const VocabParams p) {
    __shared__ float2 lds[8];
    const int wave = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * (8 / WAVES) + wave / WAVES;
    if (row >= p.T) return;
    const int64_t hit = p.target[row] - p.v0;
    float m = -INFINITY, e = 0.0f;
    for (int64_t v = (threadIdx.x & (WAVES * 64 - 1)) * 4; v < p.V; v += WAVES * 64 * 4) {
        f32x4 z = vocab_z(p, row, v);
        float most = m;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (v + r >= p.V) z[r] = -INFINITY;
            else if (v + r == hit) p.hit[row] = z[r];
            most = fmaxf(most, z[r]);
        }
        const float base = vocab_base(most);
        e *= vocab_exp<PLANES>(m - base);
#pragma unroll
        for (int r = 0; r < 4; ++r) e += vocab_exp<PLANES>(z[r] - base);
        m = most;
    }
    float most = m;
#pragma unroll
    for (int x = 32; x; x >>= 1) most = fmaxf(most, __shfl_xor(most, x, 64));
    e *= vocab_exp<PLANES>(m - vocab_base(most));
#pragma unroll
    for (int x = 32; x; x >>= 1) e += __shfl_xor(e, x, 64);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) lds[wave] = make_float2(most, e);
        __syncthreads();
        for (int w = 0; w < WAVES; ++w) most = fmaxf(most, lds[w].x);
        e = 0.0f;
        for (int w = 0; w < WAVES; ++w) e += lds[w].y * vocab_exp<PLANES>(lds[w].x - vocab_base(most));
    }
    if ((threadIdx.x & (WAVES * 64 - 1)) == 0) reinterpret_cast<float2 *>(p.part)[row * p.parts + p.v0 / p.each] = make_float2(most, e);
}
template <int PLANES> hipError_t run_part_sums(const VocabParams &p, hipStream_t s) {
    if (p.V <= 1024) hipLaunchKernelGGL((k_vocab_part_sums<PLANES, 1>), dim3((unsigned)((p.T + 7) / 8)), dim3(512), 0, s, p);
    else hipLaunchKernelGGL((k_vocab_part_sums<PLANES, 8>), dim3((unsigned)p.T), dim3(512), 0, s, p);
    return hipGetLastError();
}
template <int PLANES> __global__ __launch_bounds__(256) void k_vocab_part_dz(const VocabParams p) {
    const int64_t T = *p.count, pieces = (p.V + 7) / 8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < T * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / pieces, v0 = (i - row * pieces) * 8, hit = (int64_t)p.row_target[row] - p.v0 - v0;
        const float lse = p.row_lse[row], scale = p.row_scale[row];
        float sum = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 z = vocab_z(p, row, v0 + 4 * h);
            float d[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool target = hit == 4 * h + r, word = v0 + 4 * h + r < p.V;
                const float x = vocab_exp<PLANES>(z[r] - lse);
                d[r] = word ? (x - (target ? 1.0f : 0.0f)) * scale : 0.0f;
                if constexpr (PLANES == 1) {
                    sum += __uint_as_float(pack_rne(d[r], 0.0f) << 16);
                    if (word && target) p.rests[row * kVocabRests].rest = vocab_rest(d[r]);
                    else if (word && x > kVocabLikely) vocab_other(p, row, p.v0 + v0 + 4 * h + r, d[r]);
                }
            }
            store_dz<PLANES>(const_cast<uint16_t *>(p.dz.p) + row * p.dz.ld + v0 + 4 * h, p.dz.plane, d);
        }
        if (PLANES == 1) p.sum_part[row * p.sum_blocks + (v0 >> 3)] = sum;
    }
}

// dh: columns of h along m, rows along n, words summed
template <class S> __global__ __launch_bounds__(S::THREADS) void k_vocab_dh(const VocabParams p) {
    __shared__ __align__(16) char lds[2 * S::STAGE];
    const int64_t T = p.count[0];
    const VocabUnit<S> u(p.K, T, p.count[1], p.V);
    if (!u.there) return;
    f32x4 acc[S::NI][S::NJ] = {};
    vocab_product<S, false, true>(p.w, p.dz, u.t, p.K, T, u.k, u.end, lds, acc);
    const VocabPlace<S> place;
    const int64_t c0 = u.t.m + place.m, n0 = u.t.n + place.n;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
        const int64_t row = n0 + j * 16;
        if (row >= T) continue;
        float *to = p.dh_part + (u.split * T + row) * p.Kp + c0;       // rows of whole 32-byte pieces: four columns are there or not
#pragma unroll
        for (int i = 0; i < S::NI; ++i)
            if (c0 + 16 * i < p.Kp) {
                f32x4 *q = reinterpret_cast<f32x4 *>(to + 16 * i);
                *q = p.first ? acc[i][j] : *q + acc[i][j];
            }
    }
}

// A row's other rests by word, its target and their number in one, and what is missing to its sum: 64 rows a workgroup, their blocks' sums in 16 stretches.  With the sum off by x, what
// all words have in common does not cancel in dh, which it does of the exact dz.  The p as they are stored add up to 1 - x / dloss: they are taken relative to that, the sum (dh + dloss w[target]) / dloss
// of their words and all.  (x given to the target instead adds its own row's error where words have nothing in common: dh of 512 rows, 4000 words in double precision 5.0e-5 so, 3.6e-5, with none 3.7e-5; with a
// component in common of 10 times a word's own 5.2e-5, 3.6e-5, 3.6e-4.)
__global__ __launch_bounds__(1024) void k_vocab_rests(const VocabParams p) {
    __shared__ float lds[16][64];
    const int lane = threadIdx.x & 63, stretch = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * 64 + lane;
    const bool there = row < *p.count;
    float s = 0.0f;
    const int64_t first = p.splits_z > 1 ? row * p.sum_blocks : row, step = p.splits_z > 1 ? 1 : p.T;
    if (there)
#pragma unroll 8
        for (int i = stretch; i < p.sum_blocks; i += 16) s += p.sum_part[first + i * step];
    lds[stretch][lane] = s;
    __syncthreads();
    if (stretch || !there) return;
    s = p.first ? 0.0f : p.row_sum[row];
#pragma unroll
    for (int i = 0; i < 16; ++i) s += lds[i][lane];
    p.row_sum[row] = s;
    VocabRest *const rest = p.rests + row * kVocabRests;
    int n = p.row_others[row];
    if (n >= kVocabRests) n = 0;                           // (no probabilities: lse is not the row's)
    for (int i = 2; i <= n; ++i) {
        const VocabRest x = rest[i];
        int at = i;
        for (; at > 1 && rest[at - 1].word > x.word; --at) rest[at] = rest[at - 1];
        rest[at] = x;
    }
    for (int i = 0; i <= n; ++i) s += rest[i].rest;
    const float scale = p.row_scale[row], grow = -s / scale;
    p.row_left[row] = fabsf(grow) < 0.1f ? make_float2(-s, grow) : make_float2(0.0f, 0.0f);        // (else, dloss 0 or next to it among others, there is no such thing)
    p.row_key[row] = p.row_target[row] < 0 ? -1 : p.row_target[row] | n << kVocabWordBits;
}
hipError_t launch_vocab_rests(const VocabParams &p, hipStream_t s) {
    hipLaunchKernelGGL(k_vocab_rests, dim3((unsigned)((p.T + 63) / 64)), dim3(1024), 0, s, p);
    return hipGetLastError();
}

// dw: what rounding took from dz.  The rows of a stretch that have a rest of a word of the tile, 64 at a time, are terms of one more stage: their rows of h and, in their word's
// column, the rest.  First those of the rows' targets, then those of other words that are likely, one of each row at a time.
template <class S> __device__ __forceinline__ void vocab_rests(const VocabParams &p, const VocabUnit<S> &u, char *lds, f32x4 (&acc)[S::NI][S::NJ]) {
    using A = VocabOperand<S, S::M, false>;
    using B = VocabOperand<S, S::N, false>;
    constexpr int R = 4, WAVES = S::WAVES;
    char *const la = lds, *const lb = lds + S::PLANE_A;
    int *const rows = reinterpret_cast<int *>(lds + S::STAGE), *const words = rows + 64 + R * S::THREADS, *const found = words + 64 + R * S::THREADS;
    static_assert(((64 + R * S::THREADS) * 2 + WAVES) * 4 <= S::STAGE, "");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % S::WM * (S::M / S::WM), wn = wave / S::WM * 64;
    const int first = (int)(p.v0 + u.t.n), some = p.V - u.t.n < S::N ? (int)(p.V - u.t.n) : S::N;
    for (int j = 0; j < B::LOADS; ++j) *reinterpret_cast<uint4 *>(lb + (j * S::THREADS + tid) * 16) = make_uint4(0, 0, 0, 0);
    uint4 h[A::LOADS];                                     // of the next 64 rows
    float rest = 0.0f;
    auto fetch = [&](int from, int n) {
        if (tid < n && tid < 64) rest = p.rests[(int64_t)rows[from + tid] * kVocabRests + (words[from + tid] >> 8)].rest;
#pragma unroll
        for (int j = 0; j < A::LOADS; ++j) {
            constexpr int ROW = S::M / 8;
            const int row = tid / ROW + S::THREADS / ROW * j, at = tid % ROW;
            const int64_t col = u.t.m + ((at >> 1) ^ A::mixed(row)) * 16 + (at & 1) * 8;
            h[j] = make_uint4(0, 0, 0, 0);
            if (row < n && col < p.Kp) h[j] = *reinterpret_cast<const uint4 *>(p.h.p + rows[from + row] * p.h.ld + col);
        }
    };
    int held = 0;                                          // rests in the queue
    int which = 0, most = 0;                               // which of the rows' rests, and the last that one of these rows has
    int key[R];
    for (int64_t t0 = u.k; t0 < u.end;) {
        int word[R];
        uint64_t have[R];
        int mine = 0, others = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t t = t0 + r * S::THREADS + tid;
            if (which == 0) key[r] = t < u.end ? p.row_key[t] : -1;
            word[r] = -1;
            if (which == 0 && key[r] >= 0) word[r] = (key[r] & ((1 << kVocabWordBits) - 1)) - first;
            if (which > 0 && key[r] >> kVocabWordBits >= which) word[r] = p.rests[t * kVocabRests + which].word - first;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            have[r] = __ballot((unsigned)word[r] < (unsigned)some);
            mine += __popcll(have[r]);
            const int n = key[r] >> kVocabWordBits;
            for (int i = which; i < kVocabRests - 1 && __any(n > i); ++i) others = others > i + 1 ? others : i + 1;
        }
        if (lane == 0) found[wave] = mine | others << 16;
        __syncthreads();
        int at = held;
        most = 0;
        for (int w = 0; w < WAVES; ++w) {
            const int f = __builtin_amdgcn_readfirstlane(found[w]), here = f & 0xffff;
            if (w < wave) at += here;
            held += here;
            most = most > f >> 16 ? most : f >> 16;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (have[r] >> lane & 1) {
                const int to = at + __popcll(have[r] & ((1ull << lane) - 1));
                rows[to] = (int)(t0 + r * S::THREADS + tid);
                words[to] = word[r] | which << 8;
            }
            at += __popcll(have[r]);
        }
        __syncthreads();
        int from = 0;
        const bool last = which >= most && t0 + R * S::THREADS >= u.end;
        const int least = last ? 1 : 64;
        if (held >= least) fetch(0, held);
#pragma unroll 1
        for (; held - from >= least; from += 64) {
            const int n = held - from < 64 ? held - from : 64;
            uint16_t *at = nullptr;                        // of the rest in its word's column
            if (tid < n) {
                const int word = words[from + tid] & 0xff;
                at = reinterpret_cast<uint16_t *>(lb + tid * (S::N * 2) + (((word >> 4) ^ B::mixed(tid)) << 5) + (word & 15) * 2);
                *at = (uint16_t)pack_rne(rest, 0.0f);
            }
#pragma unroll
            for (int j = 0; j < A::LOADS; ++j) *reinterpret_cast<uint4 *>(la + (j * S::THREADS + tid) * 16) = h[j];
            __syncthreads();
            if (held - from - 64 >= least) fetch(from + 64, held - from - 64);
#pragma unroll 1
            for (int kk = 0; kk < 2; ++kk) {
                Frag x[S::NI], y[S::NJ];
                B::read(lb, wn, kk, y);
                A::read(la, wm, kk, x);
#pragma unroll
                for (int i = 0; i < S::NI; ++i)
#pragma unroll
                    for (int j = 0; j < S::NJ; ++j) acc[i][j] = mfma(x[i], y[j], acc[i][j]);
            }
            __syncthreads();
            if (at) *at = 0;
        }
        if (last) break;
        if (from) {                                        // what is left moves to the front
            const bool moves = tid < held - from;
            const int row = moves ? rows[from + tid] : 0, w = moves ? words[from + tid] : 0;
            __syncthreads();
            if (moves) { rows[tid] = row; words[tid] = w; }
            __syncthreads();
            held -= from;
        }
        if (which < most) ++which;
        else { which = 0; t0 += R * S::THREADS; }
    }
}

// dw: columns of h along m, words along n, rows summed; of one stretch as results, of several as parts
template <class S> __global__ __launch_bounds__(S::THREADS) void k_vocab_dw(const VocabParams p) {
    __shared__ __align__(16) char lds[2 * S::STAGE];
    const int64_t T = p.count ? *p.count : p.T;
    const VocabUnit<S> u(p.K, p.V, p.splits_w, T);
    if (!u.there) return;
    f32x4 acc[S::NI][S::NJ] = {};
    vocab_product<S, false, false>(p.h, p.dz, u.t, p.K, p.V, u.k, u.end, lds, acc);
    if constexpr (S::PLANES == 1) vocab_rests<S>(p, u, lds, acc);
    const VocabPlace<S> place;
    const int64_t c0 = u.t.m + place.m, n0 = u.t.n + place.n;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
        const int64_t word = n0 + j * 16;
        if (word >= p.V) continue;
        if (p.splits_w > 1) {
            float *to = p.dw_part + (u.split * p.V + word) * p.Kp + c0;
#pragma unroll
            for (int i = 0; i < S::NI; ++i)
                if (c0 + 16 * i < p.Kp) *reinterpret_cast<f32x4 *>(to + 16 * i) = acc[i][j];
            continue;
        }
        const int64_t at = (p.v0 + word) * p.K + c0;
#pragma unroll
        for (int i = 0; i < S::NI; ++i) {
            const float d[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (p.io) store_part(reinterpret_cast<uint16_t *>(p.dw) + at + 16 * i, d, p.K - c0 - 16 * i);
            else store_part(reinterpret_cast<float *>(p.dw) + at + 16 * i, d, p.K - c0 - 16 * i);
        }
    }
}

using VocabLarge = VocabSize<256, 256, 2, 1>;
using VocabSmall = VocabSize<128, 128, 2, 1>;
using VocabPlanes = VocabSize<256, 128, 4, 3>;
using VocabPlanesSmall = VocabSize<128, 64, 4, 3>;
template <bool ANY> using VocabWide = VocabSize<128, 64, 4, 3, ANY ? 2 : 1>;
template <bool ANY> using VocabWideSmall = VocabSize<64, 64, 4, 3, ANY ? 2 : 1>;
template <class S> int64_t vocab_tiles(int64_t m, int64_t n) { return ((m + S::M - 1) / S::M) * ((n + S::N - 1) / S::N); }
inline unsigned whole_dies(int64_t n) { return (unsigned)((n + 7) / 8 * 8); }

struct RunLogits {
    static constexpr bool WIDE = true;
    const VocabParams &p;
    bool backward;
    hipStream_t s;
    template <class S> void run() const {
        const int64_t tiles = vocab_tiles<S>(p.V, p.T), most = 256 * S::PER_UNIT;
        const dim3 grid(whole_dies(tiles < most ? tiles : most)), block(S::THREADS);
        if (backward) hipLaunchKernelGGL((k_vocab_logits<S, true>), grid, block, 0, s, p);
        else hipLaunchKernelGGL((k_vocab_logits<S, false>), grid, block, 0, s, p);
    }
};
struct RunPart {
    static constexpr bool WIDE = true;
    const VocabParams &p;
    hipStream_t s;
    template <class S> void run() const { hipLaunchKernelGGL(k_vocab_part<S>, dim3(whole_dies(vocab_tiles<S>(p.V, p.T) * p.splits_z)), dim3(S::THREADS), 0, s, p); }
};
struct RunDh {
    static constexpr bool WIDE = true;
    const VocabParams &p;
    hipStream_t s;
    template <class S> void run() const { hipLaunchKernelGGL(k_vocab_dh<S>, dim3(whole_dies(vocab_tiles<S>(p.K, p.T) * p.splits)), dim3(S::THREADS), 0, s, p); }
};
struct RunDw {
    static constexpr bool WIDE = false;
    const VocabParams &p;
    hipStream_t s;
    template <class S> void run() const { hipLaunchKernelGGL(k_vocab_dw<S>, dim3(whole_dies(vocab_tiles<S>(p.K, p.V) * p.splits_w)), dim3(S::THREADS), 0, s, p); }
};
template <bool ANY, class F> hipError_t sized_wide(const F &f, int side) {
    if (side == VocabWide<ANY>::M) f.template run<VocabWide<ANY>>(); else f.template run<VocabWideSmall<ANY>>();
    return hipGetLastError();
}
template <class F> hipError_t sized(const F &f, int planes, int side, bool wide = false) {
    if constexpr (F::WIDE) if (wide) return f.p.any ? sized_wide<true>(f, side) : sized_wide<false>(f, side);
    if (planes == 3) { if (side == VocabPlanes::M) f.template run<VocabPlanes>(); else f.template run<VocabPlanesSmall>(); }
    else { if (side == VocabLarge::M) f.template run<VocabLarge>(); else f.template run<VocabSmall>(); }
    return hipGetLastError();
}
hipError_t launch_vocab_logits(const VocabParams &p, bool backward, hipStream_t s) {
    if (p.splits_z == 1) return sized(RunLogits{p, backward, s}, p.planes, p.side_z, p.wide);
    if (const hipError_t e = sized(RunPart{p, s}, p.planes, p.side_z, p.wide); e != hipSuccess) return e;
    if (backward) {
        const int64_t blocks = (p.T * ((p.V + 7) / 8) + 255) / 256;
        const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096)), block(256);
        if (p.planes == 1) hipLaunchKernelGGL(k_vocab_part_dz<1>, grid, block, 0, s, p);
        else hipLaunchKernelGGL(k_vocab_part_dz<3>, grid, block, 0, s, p);
        return hipGetLastError();
    }
    return p.planes == 1 ? run_part_sums<1>(p, s) : run_part_sums<3>(p, s);
}
hipError_t launch_vocab_dh(const VocabParams &p, hipStream_t s) {
    const RunDh f{p, s};
    return sized(f, p.planes, p.side_h, p.wide);
}
hipError_t launch_vocab_dw(const VocabParams &p, hipStream_t s) { return sized(RunDw{p, s}, p.planes, p.side_w); }

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
        if constexpr (NP == 0) {
            Few<float, 8>::store(reinterpret_cast<float *>(p.dst) + row * p.ldd + c, x);
            continue;
        }
        uint32_t w[4][NP > 0 ? NP : 1];
#pragma unroll
        for (int e = 0; e < 4; ++e) split2<(NP > 0 ? NP : 1)>(x[2 * e], x[2 * e + 1], w[e]);
#pragma unroll
        for (int q = 0; q < NP; ++q) *reinterpret_cast<uint4 *>(p.dst + q * p.plane + row * p.ldd + c) = make_uint4(w[0][q], w[1][q], w[2][q], w[3][q]);
    }
}
hipError_t launch_vocab_pack(const VocabPack &p, hipStream_t s) {
    const int64_t blocks = (p.rows * (p.Kp / 8) + 255) / 256;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536)), block(256);
    if (p.io) hipLaunchKernelGGL((k_vocab_pack<uint16_t, 1>), grid, block, 0, s, p);
    else if (p.planes) hipLaunchKernelGGL((k_vocab_pack<float, 3>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_vocab_pack<float, 0>), grid, block, 0, s, p);
    return hipGetLastError();
}

// The rows with a target, in their order (one workgroup: 4096 rows at a time).  A target beyond the vocabulary makes its row's gradients NaN.
__global__ __launch_bounds__(1024) void k_vocab_rows(const VocabRows p) {
    constexpr int R = 4;
    __shared__ int part[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base = 0;
    for (int64_t first = 0; first < p.T; first += 1024 * R) {
        int64_t target[R];
        float lse[R], scale[R];
        uint64_t have[R];
        int mine = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t t = first + (wave * R + r) * 64 + lane;
            target[r] = t < p.T ? p.target[t] : -1;
            lse[r] = t < p.T ? p.lse[t] : 0.0f;
            scale[r] = t < p.T ? p.dloss[t * p.dloss_stride] : 0.0f;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) { have[r] = __ballot(target[r] >= 0); mine += __popcll(have[r]); }
        if (lane == 0) part[wave] = mine;
        __syncthreads();
        int at = base;
        for (int w = 0; w < 16; ++w) { if (w < wave) at += part[w]; base += part[w]; }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t t = first + (wave * R + r) * 64 + lane;
            const int to = at + __popcll(have[r] & ((1ull << lane) - 1));
            if (t < p.T) p.place[t] = target[r] >= 0 ? to : -1;
            if (target[r] >= 0) {
                p.index[to] = (int)t;
                p.row_lse[to] = lse[r];
                p.row_scale[to] = target[r] < p.V ? scale[r] : __builtin_nanf("");
                p.row_target[to] = target[r] < p.V ? (int)target[r] : -1;
                if (p.row_others) p.row_others[to] = 0;
            }
            at += __popcll(have[r]);
        }
        __syncthreads();
    }
    // the stretches of dh's words that suit so many rows, within the room and the workgroups that there are
    __shared__ float least[1024];
    const int s = threadIdx.x + 1;
    const int64_t tiles = (int64_t)p.across * ((base + p.side - 1) / p.side);
    const bool fits = s == 1 || ((int64_t)s * base <= p.splits * p.T && tiles * s <= p.units && (int64_t)s * 512 <= p.each);
    const float mine = fits ? vocab_time(tiles, s, p.at_once, p.each) : INFINITY;
    least[threadIdx.x] = mine;
    __syncthreads();
    for (int half = 512; half; half >>= 1) {
        if ((int)threadIdx.x < half) least[threadIdx.x] = fminf(least[threadIdx.x], least[threadIdx.x + half]);
        __syncthreads();
    }
    const uint64_t best = __ballot(fits && mine == least[0]);
    if (lane == 0) part[wave] = best ? wave * 64 + __ffsll((unsigned long long)best) : 1 << 30;
    __syncthreads();
    if (threadIdx.x) return;
    int splits = part[0];
    for (int w = 1; w < 16; ++w) splits = part[w] < splits ? part[w] : splits;
    p.count[0] = base;
    p.count[1] = splits;
}
hipError_t launch_vocab_rows(const VocabRows &p, hipStream_t s) {
    hipLaunchKernelGGL(k_vocab_rows, dim3(1), dim3(1024), 0, s, p);
    return hipGetLastError();
}

// lse and loss of a row from its tiles' largest numbers and sums, a wavefront a row
__global__ __launch_bounds__(256) void k_vocab_loss(const VocabLoss p) {
    const int lane = threadIdx.x & 63;
    for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < p.T; row += (int64_t)gridDim.x * 4) {
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
}
hipError_t launch_vocab_loss(const VocabLoss &p, hipStream_t s) {
    hipLaunchKernelGGL(k_vocab_loss, dim3((unsigned)(p.T < 1 << 22 ? (p.T + 3) / 4 : 1 << 20)), dim3(256), 0, s, p);
    return hipGetLastError();
}

// Rows of a result from the parts of its sum, four columns a thread; PARTS threads take a stretch of the parts each where there are many.  `place`: where a row's lie, -1:
// nowhere, and the row is zero.  `key`: to a row of dh the rests are added as so much of their words' rows of w, and its p brought to the sum that they have.
template <class IO, int PARTS> __global__ __launch_bounds__(256) void k_vocab_add(const VocabAdd p) {
    constexpr int ITEMS = 256 / PARTS;
    __shared__ f32x4 lds[PARTS > 1 ? 256 : 1];
    const int64_t pieces = p.Kp / 4, n = p.rows * pieces, step = (int64_t)gridDim.x * ITEMS, plane = p.count ? p.count[0] * (int64_t)p.Kp : p.plane;
    const int splits = p.count ? p.count[1] : p.splits;
    const int mine = threadIdx.x % ITEMS, q0 = threadIdx.x / ITEMS;
    for (int64_t first = (int64_t)blockIdx.x * ITEMS; first < n; first += step) {
        const int64_t i = first + mine, row = i / pieces;
        const int c = (int)(i - row * pieces) * 4;
        const int64_t at = i < n ? p.place ? p.place[row] : row : -1;
        f32x4 s = {};
        if (at >= 0) {
            const float *from = p.part + at * p.Kp + c;
#pragma unroll 4
            for (int q = q0; q < splits; q += PARTS) s += *reinterpret_cast<const f32x4 *>(from + q * plane);
        }
        if constexpr (PARTS > 1) {
            lds[threadIdx.x] = s;
            __syncthreads();
            if (q0 == 0)
#pragma unroll
                for (int q = 1; q < PARTS; ++q) s += lds[q * ITEMS + mine];
            __syncthreads();
        }
        if (q0 == 0 && i < n) {
            const int key = p.key && at >= 0 ? p.key[at] : -1;
            if (key >= 0) {
                auto words = [&](int64_t word) {
                    const IO *w = reinterpret_cast<const IO *>(p.w) + word * p.w_ld + c;
                    f32x4 x = {};
                    if (c + 4 <= p.K) {
                        Few<IO, 4> v;
                        v.load(w);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = v.get(e);
                    } else
#pragma unroll
                        for (int e = 0; e < 4; ++e) if (c + e < p.K) x[e] = load_io(w + e);
                    return x;
                };
                const f32x4 target = words(key & ((1 << kVocabWordBits) - 1));
                const float2 left = p.left[at];
                s += target * p.rests[at * kVocabRests].rest;
                for (int q = 1; q <= key >> kVocabWordBits; ++q) s += words(p.rests[at * kVocabRests + q].word) * p.rests[at * kVocabRests + q].rest;
                s += s * left.y + target * left.x;
            }
            const float x[4] = {s[0], s[1], s[2], s[3]};
            store_part(reinterpret_cast<IO *>(p.out) + row * p.K + c, x, p.K - c);
        }
    }
}
template <class IO> hipError_t run_add(const VocabAdd &p, hipStream_t s) {
    const bool many = p.splits >= 16;
    const int64_t blocks = (p.rows * (p.Kp / 4) + (many ? 32 : 256) - 1) / (many ? 32 : 256);
    const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384)), block(256);
    if (many) hipLaunchKernelGGL((k_vocab_add<IO, 8>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_vocab_add<IO, 1>), grid, block, 0, s, p);
    return hipGetLastError();
}
hipError_t launch_vocab_add(const VocabAdd &p, hipStream_t s) { return p.io ? run_add<uint16_t>(p, s) : run_add<float>(p, s); }

}  // namespace lrnnx
