// Device helpers of the gated delta rule: bfloat16 planes, matrix instructions, sequences and slots.
//
// Precision.  Matrix instructions take bfloat16 factors and add in float32.  A float32 number is the sum of three bfloat16 numbers (8 bits
// of its mantissa each, split by truncation without loss), so a float32 product is six instructions (those of weight 2^-24 and below are left
// out), and three where one factor is bfloat16 from the start.  At 16 cycles for 16 x 16 x 32 six of them take 96 cycles, the float32 matrix
// instruction 256.  Where every result is rounded to bfloat16 two planes do (16 bits, relative error 2^-17): with bfloat16 inputs and gates and no first or
// last state.  A gradient of the first state that is asked for without one is the exception: float32, from two planes (5e-6 of its norm, 2e-7 from three).
#pragma once
#include "delta.hpp"
#include "scan_common.hpp"

namespace lrnnx {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Operand of a 16 x 16 x 32 matrix product: lane l holds row (or column) l % 16 and eight of the 32 terms of the sum.  Which eight is free as long
// as both operands agree: operands from memory take them in order (8 (l / 16) ..), operands made from a result take 4 (l / 16) .. + 3 of either
// half of 16, which is what the lane holds of two result tiles.
union Frag {
    uint32_t u[4];
    uint2 h[2];
    uint4 v;
    bf16x8 b;
    f16x8 h16;
    f16x2 p16[4];
};

__device__ __forceinline__ f32x4 mfma(const Frag &a, const Frag &b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.b, b.b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(const Frag &a, const Frag &b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h16, b.h16, c, 0, 0, 0);
}
// product of operands in planes: terms below the smallest plane's weight are left out
template <int NA, int NB> __device__ __forceinline__ f32x4 mm(const Frag (&a)[NA], const Frag (&b)[NB], f32x4 c) {
    constexpr int M = NA > NB ? NA : NB;
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            if (i + j < M) c = mfma(a[i], b[j], c);
    return c;
}

// the same for several results with one operand in common, product by product: neighbours do not wait for each other's sums
template <int N, int NA, int NB> __device__ __forceinline__ void mm_each(const Frag (&a)[N][NA], const Frag (&b)[NB], f32x4 (&c)[N]) {
    constexpr int M = NA > NB ? NA : NB;
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            if (i + j < M)
#pragma unroll
                for (int m = 0; m < N; ++m) c[m] = mfma(a[m][i], b[j], c[m]);
}

__device__ __forceinline__ float hi_part(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_hi(float a, float b) {        // the upper halves of two numbers
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ uint32_t pack_rne(float a, float b) {
    f32x2 x = {a, b};
    union { bf16x2 b; uint32_t u; } r;
    r.b = __builtin_convertvector(x, bf16x2);
    return r.u;
}
// two numbers as NP planes: by truncation (exact with three), the last of fewer planes rounded to nearest
template <int NP> __device__ __forceinline__ void split2(float a, float b, uint32_t (&out)[NP]) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        if (i == NP - 1 && NP < 3) { out[i] = pack_rne(a, b); break; }
        out[i] = pack_hi(a, b);
        if (i < NP - 1) { a -= hi_part(a); b -= hi_part(b); }
    }
}
// What the backward pass is left of states, errors and their gradients: float32 where a result is float32, which is that of the gates with float32 gates.
// Where inputs and gates are bfloat16, and so all results but the states' gradients (which come from none of it): 16-bit floating point with a common
// power of two a block, 11 bits of mantissa (the results keep 8) for numbers down to 2^-29 of the block's largest, which the power brings to 2^14 .. 2^15.
// 4 x 4096 steps of 16 heads of 128 x 128, training: 800 us so, 1190 in float32 (with three planes in both walks too).
// What is not finite stays so and has no part in it.  The power's inverse, from the largest magnitude:
__device__ __forceinline__ float block_unit(float largest) {
    const uint32_t e = __float_as_uint(largest) >> 23;
    return __uint_as_float(((e > 15 ? e : 15) - 14) << 23);
}
__device__ __forceinline__ float inverse_unit(float unit) { return __uint_as_float((254u << 23) - __float_as_uint(unit)); }
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    f32x2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
}
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
// The larger magnitudes of bfloat16 pairs, as bits plus 0x80, by which what is not finite comes out smallest.
__device__ __forceinline__ uint32_t max_finite(uint32_t most, uint32_t pair) {
    const uint32_t x = ((pair & 0x7fff7fffu) + 0x00800080u) & 0x7fff7fffu;
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, most), __builtin_bit_cast(u16x2, x)));
}
template <int N, bool FINITE = false> __device__ __forceinline__ float largest_of(const f32x4 (&x)[N]) {
    float m[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float v = fabsf(x[i][r]);
            m[i & 1] = fmaxf(m[i & 1], FINITE && v == INFINITY ? 0.0f : v);
        }
    return fmaxf(m[0], m[1]);
}
template <int CTRL, int ROW_MASK = 0xF> __device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
    const uint32_t y = __builtin_amdgcn_update_dpp(0, x, CTRL, ROW_MASK, 0xF, false);
    return x > y ? x : y;
}
__device__ __forceinline__ float wave_max(float m) {          // of numbers that are not negative: they compare as their bits do
    uint32_t x = __float_as_uint(m);
    x = dpp_max<0x111>(x);                                    // row_shr 1, 2, 4, 8
    x = dpp_max<0x112>(x);
    x = dpp_max<0x114>(x);
    x = dpp_max<0x118>(x);
    x = dpp_max<0x142, 0xA>(x);                               // lane 15 of a row to the next row, lane 31 to the upper half
    x = dpp_max<0x143, 0xC>(x);
    return __uint_as_float(__builtin_amdgcn_readlane(x, 63));
}
// the unit of a wavefront's numbers, by the largest that is finite
template <int N> __device__ __forceinline__ float unit_of(const f32x4 (&x)[N]) {
    float m = wave_max(largest_of(x));
    if (m == INFINITY) m = wave_max(largest_of<N, true>(x));
    return block_unit(m);
}
// MT tiles of a state's 16 columns as they are saved, a column to a row of DK (this lane's part starts at element `at`): float32, or 16 bits with
// their unit (a unit each half of the rows)
template <bool EXACT, int DK, int MT> __device__ __forceinline__ void save_state(const f32x4 (&S)[MT], void *states, int64_t at, float *unit, int G) {
    if constexpr (EXACT) {
#pragma unroll
        for (int m = 0; m < MT; ++m) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(states) + at + 16 * m) = S[m];
    } else {
        const float u = unit_of(S), inv = inverse_unit(u);
        if ((threadIdx.x & 63) == 0) {
            *unit = u;
            if (MT == DK / 16) unit[G] = u;
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
            *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(states) + at + 16 * m) =
                make_uint2(pack_f16(S[m][0] * inv, S[m][1] * inv), pack_f16(S[m][2] * inv, S[m][3] * inv));
    }
}
// 16 columns of N tiles of 16 steps of E or Z, a step to a lane (`at`: this lane's element of the first, the next ones' rows16 on; n: steps there
// are from the first tile on; a unit a tile, G apart)
template <bool EXACT, int N> __device__ __forceinline__ void save_rows(const f32x4 (&X)[N], void *rows, int64_t at, int64_t rows16, int n, float *unit, int G) {
    const int row16 = threadIdx.x & 15;
    float inv = 0.0f;
    if constexpr (!EXACT) {
        const float u = unit_of(X);
        inv = inverse_unit(u);
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int m = 0; m < N; ++m) unit[m * G] = u;
    }
#pragma unroll
    for (int m = 0; m < N; ++m)
        if (16 * m + row16 < n) {
            if constexpr (EXACT) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(rows) + at + m * rows16) = X[m];
            else *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(rows) + at + m * rows16) =
                     make_uint2(pack_f16(X[m][0] * inv, X[m][1] * inv), pack_f16(X[m][2] * inv, X[m][3] * inv));
        }
}

// two result tiles as the operand of the next product
template <int NP> __device__ __forceinline__ void split_tiles(const f32x4 &lo, const f32x4 &hi, Frag (&f)[NP]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t w[NP];
        if (e < 2) split2<NP>(lo[2 * e], lo[2 * e + 1], w);
        else split2<NP>(hi[2 * e - 4], hi[2 * e - 3], w);
#pragma unroll
        for (int i = 0; i < NP; ++i) f[i].u[e] = w[i];
    }
}
// The same with the matrix unit taking off what a plane holds: x - plane as (-I) plane + x, exact like the subtraction, one instruction for a tile
// where two vector instructions an element are eight.  (A wavefront alone on its SIMD is bound by the instructions it issues.)
struct NegId { Frag lo, hi; };                               // -I for the terms of the lower and of the upper tile of an operand
__device__ __forceinline__ NegId neg_id() {
    NegId n;
    const int lane = threadIdx.x & 63, at = (lane & 15) - 4 * (lane >> 4);          // this row's own term, if it is one of the lane's four
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t w = at == 2 * i ? 0xbf80u : at == 2 * i + 1 ? 0xbf800000u : 0u;
        n.lo.u[i] = w; n.lo.u[i + 2] = 0;
        n.hi.u[i] = 0; n.hi.u[i + 2] = w;
    }
    return n;
}
template <int NP> __device__ __forceinline__ void split_tiles(f32x4 lo, f32x4 hi, Frag (&f)[NP], const NegId &neg) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            f[i].u[e] = i == NP - 1 && NP < 3 ? pack_rne(lo[2 * e], lo[2 * e + 1]) : pack_hi(lo[2 * e], lo[2 * e + 1]);
            f[i].u[e + 2] = i == NP - 1 && NP < 3 ? pack_rne(hi[2 * e], hi[2 * e + 1]) : pack_hi(hi[2 * e], hi[2 * e + 1]);
        }
        if (i < NP - 1) { lo = mfma(neg.lo, f[i], lo); hi = mfma(neg.hi, f[i], hi); }
    }
}
// Tiles of a chunk's triangular matrices as they lie in memory and LDS: UP: of T^T and A^T, whose second tile of rows has no first block; else of T and
// A, whose first has no second.  `half`: that tile.
template <bool UP> __device__ __forceinline__ void triangle_tile(bool half, const uint16_t *halves, const uint16_t *wholes, int lane, Frag &f) {
    const uint16_t *p = half ? halves + 4 * lane : wholes + 8 * lane;
    const uint2 a = *reinterpret_cast<const uint2 *>(p), b = *reinterpret_cast<const uint2 *>(p + (UP && half ? 0 : 4));
    f.h[0] = UP && half ? make_uint2(0, 0) : a;
    f.h[1] = !UP && half ? make_uint2(0, 0) : b;
}
template <bool UP> __device__ __forceinline__ Frag half_tile(const uint16_t *halves, int lane) {
    Frag f;
    f.h[UP] = *reinterpret_cast<const uint2 *>(halves + 4 * lane);
    f.h[!UP] = make_uint2(0, 0);
    return f;
}
__device__ __forceinline__ Frag whole_tile(const uint16_t *wholes, int lane) {
    Frag f;
    f.v = *reinterpret_cast<const uint4 *>(wholes + 8 * lane);
    return f;
}
// LDS reads before this stay before it (they are wanted early, registers or not)
__device__ __forceinline__ void reads_first() { asm volatile("" ::: "memory"); }

template <int NP> __device__ __forceinline__ void zero_frags(Frag (&f)[NP]) {
#pragma unroll
    for (int i = 0; i < NP; ++i) f[i].v = make_uint4(0, 0, 0, 0);
}

// Rows of a chunk through a buffer descriptor: steps past the end of a sequence lie past the descriptor's end and read as zero, so nothing is
// compared, cleared or branched around on the way, and offsets are 32 bits that stay the same from chunk to chunk.  The host sees to it that
// rows do not overlap and that 32 of them span less than 2 GB.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const void *p, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00020000);
}
constexpr uint32_t kOutside = 0x80000000u;                    // an offset past every descriptor's end
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint2 buffer_load8(Buffer b, uint32_t off) {
    const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(b, off, 0, 0));
    return make_uint2(v.x, v.y);
}
__device__ __forceinline__ uint4 buffer_load16(Buffer b, uint32_t off) {
    const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, off, 0, 0));
    return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ void buffer_load(Buffer b, uint32_t off, uint16_t &x) { x = __builtin_amdgcn_raw_buffer_load_b16(b, off, 0, 0); }
__device__ __forceinline__ void buffer_load(Buffer b, uint32_t off, float &x) { x = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b, off, 0, 0)); }

__device__ __forceinline__ float load_io(const float *p) { return *p; }
__device__ __forceinline__ float load_io(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store_io(float *p, float x) { *p = x; }
__device__ __forceinline__ void store_io(uint16_t *p, float x) { *p = (uint16_t)pack_rne(x, x); }
// four elements; `vec`: the address takes one access
__device__ __forceinline__ void store4(float *p, const f32x4 &x) { *reinterpret_cast<f32x4 *>(p) = x; }
__device__ __forceinline__ void store4(uint16_t *p, const f32x4 &x) {
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack_rne(x[0], x[1]), pack_rne(x[2], x[3]));
}

// g or beta of a step, in float32 or in the I/O type
__device__ __forceinline__ float load_gate(const void *p, int64_t i, int io, int gate_io) {
    return gate_io && io ? load_io(reinterpret_cast<const uint16_t *>(p) + i) : load_io(reinterpret_cast<const float *>(p) + i);
}

// Position of terms 4 q .. 4 q + 3 of a block of 32 in a row of LDS: what lane group g reads lies together (4 g .. and 16 + 4 g ..).
__device__ __forceinline__ int quad_place(int q) { return ((q & 3) * 2 + (q >> 2)) * 4; }
// Where a turned operand's 16-byte piece of a row lies: pieces of every 16 rows change places, so that a wavefront that writes a piece of every
// fourth row reaches all banks.  (The pieces of a tile of 16 rows move together: a constant for who reads it.)
__device__ __forceinline__ int turned(int row, int place) { return place ^ (((row >> 4) & 3) << 3); }
// four rows of four neighbouring elements -> four columns of four
__device__ __forceinline__ void transpose_quad(const uint2 (&w)[4], uint2 (&c)[4]) {
    c[0] = make_uint2(__builtin_amdgcn_perm(w[1].x, w[0].x, 0x05040100u), __builtin_amdgcn_perm(w[3].x, w[2].x, 0x05040100u));
    c[1] = make_uint2(__builtin_amdgcn_perm(w[1].x, w[0].x, 0x07060302u), __builtin_amdgcn_perm(w[3].x, w[2].x, 0x07060302u));
    c[2] = make_uint2(__builtin_amdgcn_perm(w[1].y, w[0].y, 0x05040100u), __builtin_amdgcn_perm(w[3].y, w[2].y, 0x05040100u));
    c[3] = make_uint2(__builtin_amdgcn_perm(w[1].y, w[0].y, 0x07060302u), __builtin_amdgcn_perm(w[3].y, w[2].y, 0x07060302u));
}

// Barrier of a workgroup whose wavefronts exchange through LDS alone: accesses to global memory stay under way (__syncthreads would wait for
// every store of results, about a microsecond each time).
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Which workgroup does what: a unit is a segment of a head of a batch entry; the workgroups of its groups of columns, which read the same rows, are
// 8 apart and so on one die.  False: none (the launch rounds up to whole eights).
struct DeltaUnit { int group, h, b, seg; };
__device__ __forceinline__ bool delta_unit(const DeltaParams &p, unsigned segs, DeltaUnit &u) {
    const unsigned id = blockIdx.x, per = 8u * p.groups, heads = (unsigned)p.B * p.Hv;
    const unsigned unit = id / per * 8 + (id & 7);
    u.group = (int)(id % per >> 3);
    if (unit >= heads * segs) return false;
    u.seg = (int)(unit / heads);
    const unsigned bh = unit - u.seg * heads;
    u.b = (int)(bh / (unsigned)p.Hv);
    u.h = (int)(bh - (unsigned)u.b * p.Hv);
    return true;
}

inline unsigned delta_blocks(const DeltaParams &p, int segs) { return (unsigned)(((int64_t)p.B * p.Hv * segs + 7) / 8 * 8 * p.groups); }
// Two wavefronts to 16 columns: where one each would leave half of the compute units without a workgroup, or half of a workgroup without columns; more come
// in two rounds.  1024 steps of 128 x 128, whole calls, one wavefront / two: 64 heads (128 workgroups of one) 85 / 76 us for a prompt, 245 / 208 in training,
// in float32 195 / 165 and 680 / 604; 65 heads 86 / 131, 258 / 260; 64 x 64 of 128 heads 69 / 67 and 209 / 199, of 160 heads 71 / 82 and 238 / 255.
inline bool delta_rows_split(const DeltaParams &p) { return p.dvp <= 32 || (int64_t)p.B * p.Hv * p.nseg * ((p.dvp + 63) / 64) <= 128; }
// A wavefront's 16 columns (this lane's: j) of a segment's transition, as planes [dk][dk].
template <int NP, int DK> __device__ __forceinline__ void store_trans(const f32x4 (&S)[DK / 16], uint16_t *to, int j, int g4) {
#pragma unroll
    for (int m = 0; m < DK / 16; ++m)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
            uint32_t w[NP];
            split2<NP>(S[m][r], S[m][r + 1], w);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                uint16_t *q = to + (i * DK + 16 * m + 4 * g4 + r) * DK + j;
                q[0] = (uint16_t)w[i];
                q[DK] = (uint16_t)(w[i] >> 16);
            }
        }
}

struct DeltaSeq {
    int64_t at, len;                     // first step on its time axis, steps
    int64_t slot, row;                   // first slot; first row of the arrays [row, head, column] that the library lays out
    int64_t ib;                          // batch entry of the caller's tensors
};
__device__ __forceinline__ int64_t delta_clamp(int64_t x, int64_t L) { return x < 0 ? 0 : x > L ? L : x; }
__device__ __forceinline__ DeltaSeq delta_seq(const DeltaParams &p, int b) {
    DeltaSeq s;
    if (p.cu) {
        const int64_t lo = delta_clamp(p.cu[b], p.L), hi = delta_clamp(p.cu[b + 1], p.L);
        s.at = lo; s.len = hi > lo ? hi - lo : 0; s.slot = lo / kDeltaSlot + b; s.row = lo; s.ib = 0;
    } else {
        s.at = 0; s.len = p.L; s.slot = (int64_t)b * p.slots_each; s.row = (int64_t)b * p.L; s.ib = b;
    }
    return s;
}
// The sequence that a slot of a packed batch belongs to, by a 64-way search of ascending boundaries (whole wavefronts call it).
__device__ __forceinline__ int delta_find(const DeltaParams &p, int64_t slot) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = p.B;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, i = lo + lane * step;
        const bool before = i < hi && (lane == 0 || delta_clamp(p.cu[i], p.L) / kDeltaSlot + i <= slot);
        const int n = __popcll(__ballot(before));
        lo = lo + (n - 1) * step;
        hi = hi < lo + step ? hi : lo + step;
    }
    return lo;
}
// Steps of a slot: its sequence, its first step within it and how many of the 64 there are (0: none).
__device__ __forceinline__ int delta_slot(const DeltaParams &p, int64_t slot, DeltaSeq &s, int64_t &t0, int &b) {
    b = p.cu ? delta_find(p, slot) : (int)(slot / p.slots_each);
    s = delta_seq(p, b);
    t0 = (slot - s.slot) * kDeltaSlot;
    const int64_t n = t0 < 0 ? 0 : s.len - t0;
    return n <= 0 ? 0 : n > kDeltaSlot ? kDeltaSlot : (int)n;
}

// Logarithm of a decay: -inf (forget everything) as a number whose sums stay finite; exp of it is 0 all the same.  Decays are taken by the hardware's
// power of two: off by 1e-7 (1 + |x|) of e^x, so by 3e-8 of 1 at most beyond rounding.
__device__ __forceinline__ double gate_log(float g) { return g < -1e5f ? -1e5 : (double)g; }

}  // namespace lrnnx
