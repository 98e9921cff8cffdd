// Device helpers of the short causal convolution: pieces of the contiguous axis, the activation, the sequences of a packed batch.
#pragma once
#include "conv.hpp"
#include "delta_common.hpp"

namespace lrnnx {

// Vector accesses at element alignment.
template <int BYTES> struct OnElement;
template <> struct OnElement<2> {
    typedef uint32_t one __attribute__((aligned(2)));
    typedef u32x2 two __attribute__((aligned(2)));
    typedef u32x4 four __attribute__((aligned(2)));
};
template <> struct OnElement<4> {
    typedef uint32_t one __attribute__((aligned(4)));
    typedef u32x2 two __attribute__((aligned(4)));
    typedef u32x4 four __attribute__((aligned(4)));
};
// VEC neighbouring elements as one access at element alignment (rows of odd length, views and packed sequences start anywhere).
template <class T, int VEC> struct Few {
    static constexpr int W = VEC * (int)sizeof(T) / 4;            // words
    uint32_t w[W > 0 ? W : 1];
    using At = OnElement<sizeof(T)>;
    using one = typename At::one;
    using two = typename At::two;
    using four = typename At::four;
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (VEC == 1) w[0] = sizeof(T) == 4 ? *reinterpret_cast<const uint32_t *>(p) : *reinterpret_cast<const uint16_t *>(p);
        else if constexpr (W == 1) w[0] = *reinterpret_cast<const one *>(p);
        else if constexpr (W == 2) { const u32x2 v = *reinterpret_cast<const two *>(p); w[0] = v.x; w[1] = v.y; }
        else
#pragma unroll
            for (int i = 0; i < W; i += 4) {
                const u32x4 v = *reinterpret_cast<const four *>(p + i * 4 / (int)sizeof(T));
                w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
            }
    }
    // the first n elements, zeros behind them; all loads at once (where each is branched around, each is waited for)
    __device__ __forceinline__ void load_some(const T *p, int n) {
#pragma unroll
        for (int i = 0; i < (W > 0 ? W : 1); ++i) w[i] = 0;
        if (n <= 0) return;
        uint32_t v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const T *at = p + (e < n ? e : n - 1);
            if constexpr (sizeof(T) == 4) v[e] = *reinterpret_cast<const uint32_t *>(at);
            else v[e] = *reinterpret_cast<const uint16_t *>(at);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            v[e] = e < n ? v[e] : 0;
            if constexpr (sizeof(T) == 4) w[e] = v[e];
            else w[e >> 1] |= v[e] << (e & 1) * 16;
        }
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[VEC]) {
        static_assert(sizeof(T) == 4 ? VEC <= 2 || VEC % 4 == 0 : VEC == 1 || VEC == 4 || VEC % 8 == 0, "whole accesses");
        if constexpr (VEC == 1) store_io(p, x[0]);
        else if constexpr (sizeof(T) == 4 && VEC == 2) *reinterpret_cast<two *>(p) = u32x2{__float_as_uint(x[0]), __float_as_uint(x[1])};
        else if constexpr (sizeof(T) == 4)
#pragma unroll
            for (int i = 0; i < VEC; i += 4) *reinterpret_cast<four *>(p + i) = u32x4{__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]), __float_as_uint(x[i + 3])};
        else if constexpr (VEC == 4 && sizeof(T) == 2) *reinterpret_cast<two *>(p) = u32x2{pack_rne(x[0], x[1]), pack_rne(x[2], x[3])};
        else
#pragma unroll
            for (int i = 0; i < VEC; i += 8) *reinterpret_cast<four *>(p + i) = u32x4{pack_rne(x[i], x[i + 1]), pack_rne(x[i + 2], x[i + 3]), pack_rne(x[i + 4], x[i + 5]), pack_rne(x[i + 6], x[i + 7])};
    }
};
template <class IO> constexpr int kFew = 16 / (int)sizeof(IO);    // elements of a 16-byte access

// silu(z) = z s, s = 1 / (1 + e^-z), and its derivative s (1 + z (1 - s)).  With float32 results e^-z is the exact function's, with bfloat16 ones the
// hardware's power of two (1e-7 (1 + |z|) of e^-z); the reciprocal is off by 1 ulp.
template <class IO> __device__ __forceinline__ float conv_sigmoid(float z) {
    return __builtin_amdgcn_rcpf(1.0f + (sizeof(IO) == 4 ? expf(-z) : __expf(-z)));
}
template <class IO, bool SILU> __device__ __forceinline__ float conv_act(float z) { return SILU ? z * conv_sigmoid<IO>(z) : z; }
template <class IO, bool SILU> __device__ __forceinline__ float conv_dact(float z) {
    if constexpr (!SILU) return 1.0f;
    const float s = conv_sigmoid<IO>(z);
    return s * __builtin_fmaf(z, 1.0f - s, 1.0f);
}

// The sequence that step l lies in: lo <= l < hi; or none, and then `hi` is where the next one may start (past l, so that a walk always ends,
// whatever the boundaries hold).  Boundaries ascend and are clamped to the axis.
struct ConvSpan { int64_t lo, hi; int seq; bool in; };
// `after`: the sequences before that one start at l or before (0: not known).
__device__ __forceinline__ ConvSpan conv_span(const ConvParams &p, int b, int64_t l, int after = 0) {
    if (!p.cu) return {0, p.L, b, true};
    int lo = -1, hi = p.seqs;                              // the last sequence that starts at l or before
    if (after) {                                           // (a walk's next: a few further on)
        lo = after - 1;
        while (lo + 1 < hi && delta_clamp(p.cu[lo + 1], p.L) <= l) ++lo;
        hi = lo + 1;
    }
    while (hi - lo > 1) {                                  // eight boundaries at a time: a wait for memory for three steps of a search by halves
        const int step = (hi - lo - 1 + 7) / 8;
        int64_t at[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) { const int k = lo + (i + 1) * step; at[i] = p.cu[k < hi ? k : hi - 1]; }
        int found = lo, next = hi;
#pragma unroll
        for (int i = 7; i >= 0; --i) {
            const int k = lo + (i + 1) * step;
            if (k < hi && found == lo) { if (delta_clamp(at[i], p.L) <= l) found = k; else next = k; }
        }
        lo = found;
        hi = next;
    }
    if (lo >= 0) {
        const int64_t s = delta_clamp(p.cu[lo], p.L), e = delta_clamp(p.cu[lo + 1], p.L);
        if (s <= l && l < e) return {s, e, lo, true};
    }
    int64_t next = hi < p.seqs ? delta_clamp(p.cu[hi], p.L) : p.L;
    if (next <= l) next = l + 1;
    return {l, next, lo, false};
}

// Input at step l of channel d of the sequence `s`; before its first step what was carried, or 0.
template <class IO, int W> __device__ __forceinline__ float conv_input(const ConvParams &p, const ConvSpan &s, int b, int64_t l, int d) {
    if (l >= s.lo) return load_io(reinterpret_cast<const IO *>(p.x) + b * p.x_b + l * p.x_l + d * p.x_d);
    if (!p.x0) return 0.0f;
    return load_io(reinterpret_cast<const IO *>(p.x0) + ((int64_t)s.seq * (W - 1) + (W - 1) + (l - s.lo)) * p.D + d);
}
template <class IO, int W> __device__ __forceinline__ float conv_pre(const ConvParams &p, const ConvSpan &s, int b, int64_t l, int d) {
    float z = p.bias ? p.bias[d] : 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) z = __builtin_fmaf(p.w[(int64_t)d * W + j], conv_input<IO, W>(p, s, b, l - (W - 1) + j, d), z);
    return z;
}
__device__ __forceinline__ ConvSpan conv_sequence(const ConvParams &p, int seq) {
    if (!p.cu) return {0, p.L, seq, true};
    const int64_t lo = delta_clamp(p.cu[seq], p.L), hi = delta_clamp(p.cu[seq + 1], p.L);
    return {lo, hi > lo ? hi : lo, seq, true};
}

// The last W - 1 inputs of every sequence, an element a thread.  (Workgroups behind those of the sequences, in the same launch.)
template <class IO, int W> __device__ __forceinline__ void conv_last(const ConvParams &p, int64_t first, int64_t stride) {
    const int64_t n = (int64_t)p.seqs * (W - 1) * p.D;
    for (int64_t i = first; i < n; i += stride) {
        const int d = (int)(i % p.D);
        const int64_t r = i / p.D;
        const int seq = (int)(r / (W - 1)), slot = (int)(r % (W - 1));
        const ConvSpan s = conv_sequence(p, seq);
        const int64_t l = s.hi - (W - 1) + slot;
        IO *to = reinterpret_cast<IO *>(p.x_last) + i;
        if (l >= s.lo) *to = reinterpret_cast<const IO *>(p.x)[(p.cu ? 0 : seq) * p.x_b + l * p.x_l + d * p.x_d];
        else *to = p.x0 ? reinterpret_cast<const IO *>(p.x0)[((int64_t)seq * (W - 1) + (W - 1) + (l - s.lo)) * p.D + d] : IO(0);
    }
}
// Gradients of the carried inputs: dx0[i] = sum_{j <= i} w[i-j] g[j] over the sequence's first steps, and of a sequence of fewer than W - 1 steps what dx_last
// says of those that are still there.
template <class IO, int W, bool SILU> __device__ __forceinline__ void conv_dx0(const ConvParams &p, int64_t first, int64_t stride) {
    const int64_t n = (int64_t)p.seqs * p.D;
    for (int64_t i = first; i < n; i += stride) {
        const int d = (int)(i % p.D), seq = (int)(i / p.D), b = p.cu ? 0 : seq;
        const ConvSpan s = conv_sequence(p, seq);
        const int64_t steps = s.hi - s.lo;
        float out[W - 1] = {};
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            if (j < steps) {
                const float g = load_io(reinterpret_cast<const IO *>(p.dy) + b * p.dy_b + (s.lo + j) * p.dy_l + d * p.dy_d) *
                                conv_dact<IO, SILU>(conv_pre<IO, W>(p, s, b, s.lo + j, d));
#pragma unroll
                for (int k = j; k < W - 1; ++k) out[k] = __builtin_fmaf(p.w[(int64_t)d * W + k - j], g, out[k]);
            }
#pragma unroll
        for (int k = 0; k < W - 1; ++k) {
            const int64_t at = ((int64_t)seq * (W - 1) + k) * p.D + d;
            if (p.dx_last && k >= steps) out[k] += load_io(reinterpret_cast<const IO *>(p.dx_last) + at - steps * p.D);
            store_io(reinterpret_cast<IO *>(p.dx0) + at, out[k]);
        }
    }
}

inline unsigned conv_blocks(int64_t items) { return (unsigned)(items < 1 ? 0 : items > 256 * 256 ? 256 : (items + 255) / 256); }

}  // namespace lrnnx
