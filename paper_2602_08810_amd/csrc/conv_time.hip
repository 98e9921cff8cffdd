// Short causal convolution with an activation, time axis contiguous ([B,D,L]): the formulas of the other layout's kernels.
// The lanes of a row take a 16-byte piece of the time axis each, side by side; forward, the W - 1 inputs before a piece come from a second, narrower access that the
// first level of cache has.  Bound by memory.
// A piece that a sequence of a packed batch starts or ends in goes step by step.
#include "conv_common.hpp"

namespace lrnnx {

// inputs xs[i] at steps l - (W - 1) + i, i < W - 1, of a piece that starts at l (s.lo <= l)
template <class IO, int W> __device__ __forceinline__ void time_before(const ConvParams &p, const ConvSpan &s, const IO *x, int b, int64_t l, int d, float *xs) {
    if (l - s.lo >= 4) {
        Few<IO, 4> v;
        v.load(x + l - 4);
#pragma unroll
        for (int i = 0; i < W - 1; ++i) xs[i] = v.get(4 - (W - 1) + i);
    } else {
#pragma unroll
        for (int i = 0; i < W - 1; ++i) xs[i] = conv_input<IO, W>(p, s, b, l - (W - 1) + i, d);
    }
}
template <class IO, int W, int VEC, bool SILU> __global__ __launch_bounds__(256) void k_conv_time_fwd(const ConvParams p) {
    const int tid = threadIdx.x, lane = tid & ((1 << p.shift) - 1), d = blockIdx.y * (256 >> p.shift) + (tid >> p.shift);
    if ((int)blockIdx.x >= p.blocks) {
        conv_last<IO, W>(p, ((int64_t)(blockIdx.x - p.blocks) * gridDim.y + blockIdx.y) * 256 + tid, (int64_t)(gridDim.x - p.blocks) * gridDim.y * 256);
        return;
    }
    if (d >= p.D) return;
    const int b = p.cu ? 0 : (int)(blockIdx.x / (unsigned)p.tiles_each);
    const int64_t t0 = (int64_t)(blockIdx.x - (unsigned)b * (unsigned)p.tiles_each) * p.tile, t1 = t0 + p.tile < p.L ? t0 + p.tile : p.L;
    const IO *x = reinterpret_cast<const IO *>(p.x) + b * p.x_b + d * p.x_d;
    IO *y = reinterpret_cast<IO *>(p.y) + b * p.y_b + d * p.y_d;
    float w[W];
    const float bias = p.bias ? p.bias[d] : 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) w[j] = p.w[(int64_t)d * W + j];
    for (int64_t piece = t0 + lane * VEC; piece < t1; piece += VEC << p.shift) {
        const int64_t l = piece + VEC <= p.L ? piece : p.L - VEC;        // the last piece overlaps the one before
        const ConvSpan s = conv_span(p, b, l);
        if (s.in && l + VEC <= s.hi) {
            Few<IO, VEC> in;
            in.load(x + l);
            float xs[VEC + W - 1], out[VEC];
            time_before<IO, W>(p, s, x, b, l, d, xs);
#pragma unroll
            for (int e = 0; e < VEC; ++e) xs[W - 1 + e] = in.get(e);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float z = bias;
#pragma unroll
                for (int j = 0; j < W; ++j) z = __builtin_fmaf(w[j], xs[e + j], z);
                out[e] = conv_act<IO, SILU>(z);
            }
            Few<IO, VEC>::store(y + l, out);
        } else {
            for (int64_t t = l; t < l + VEC; ++t) {
                const ConvSpan q = conv_span(p, b, t);
                if (q.in) store_io(y + t, conv_act<IO, SILU>(conv_pre<IO, W>(p, q, b, t, d)));
            }
        }
    }
}

// Backward a row is walked from its end, so that the g that a piece needs of the W - 1 steps behind it are the next lane's, or what the first lane had the visit
// before; the inputs before it are the lane's before.  (With every piece forming them again: 45 us where this takes ?, 8 x 1536 x 2048 in bfloat16.)
// A packed batch goes step by step.
template <class IO, int W, int VEC, bool SILU> __global__ __launch_bounds__(256, 3) void k_conv_time_bwd(const ConvParams p) {
    const int tid = threadIdx.x, side = 1 << p.shift, lane = tid & (side - 1), d0 = blockIdx.y * (256 >> p.shift) + (tid >> p.shift);
    if ((int)blockIdx.x >= p.blocks) {
        conv_dx0<IO, W, SILU>(p, ((int64_t)(blockIdx.x - p.blocks) * gridDim.y + blockIdx.y) * 256 + tid, (int64_t)(gridDim.x - p.blocks) * gridDim.y * 256);
        return;
    }
    const int d = d0 < p.D ? d0 : p.D - 1;                 // (lanes without a row go along)
    float dw[W + 1] = {}, w[W];
    const float bias = p.bias ? p.bias[d] : 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) w[j] = p.w[(int64_t)d * W + j];
    const int visit = VEC << p.shift;
    // tile after tile, and each from its last visit to its first; the next is on its way while a visit is worked on
    struct At {
        unsigned slot;
        int b, first, len, rest;                           // first step of the visit, steps of the tile, steps to the end of the row (all from the tile's first step on)
        int64_t t0;
        const IO *x, *dy;
    };
    struct Loads { Few<IO, VEC> x, dy; Few<IO, 4> before; };
    auto tile = [&](unsigned slot) {
        At a;
        a.slot = slot;
        a.b = p.cu ? 0 : (int)(slot / (unsigned)p.tiles_each);
        a.t0 = (int64_t)(slot - (unsigned)a.b * (unsigned)p.tiles_each) * p.tile;
        const int64_t rest = p.L - a.t0;
        a.rest = rest < 1 << 30 ? (int)rest : 1 << 30;
        a.len = a.rest < p.tile ? a.rest : p.tile;
        a.first = (a.len - 1) / visit * visit;
        a.x = reinterpret_cast<const IO *>(p.x) + a.b * p.x_b + d * p.x_d + a.t0;
        a.dy = reinterpret_cast<const IO *>(p.dy) + a.b * p.dy_b + d * p.dy_d + a.t0;
        return a;
    };
    auto fetch = [&](const At &a, Loads &v) {
        const int l = a.first + lane * VEC;
        if (l + VEC <= a.len) { v.x.load(a.x + l); v.dy.load(a.dy + l); }
        else if (!p.cu) { v.x.load_some(a.x + l, a.len - l); v.dy.load_some(a.dy + l, a.len - l); }      // (zeros behind the tile: no part of any sum)
        if (lane == 0 && a.t0 + l >= 4) v.before.load(a.x + l - 4);
    };
    if (blockIdx.x < (unsigned)p.tiles) {
        // the next visit; false behind the last
        auto advance = [&](At &a) {
            if (a.first > 0) { a.first -= visit; return true; }
            if (a.slot + p.blocks >= (unsigned)p.tiles) return false;
            a = tile(a.slot + p.blocks);
            return true;
        };
        At now = tile(blockIdx.x), ahead = now;
        Loads in{}, in1{};
        float after[W - 1];                                // g of the steps behind the visit
        fetch(ahead, in);
        bool fresh = true, more = true;
        for (; more; now = ahead, in = in1) {
            more = advance(ahead);
            if (more) fetch(ahead, in1);
            const int b = now.b, first = now.first, l = first + lane * VEC;
            const int64_t t0 = now.t0;
            IO *dx = reinterpret_cast<IO *>(p.dx) + b * p.y_b + d * p.y_d + t0;
            const ConvSpan own{0, p.L, b, true};
            auto from_last = [&](const ConvSpan &s, int64_t t) {         // what the last inputs' gradient brings to step t
                if (!p.dx_last || t < s.hi - (W - 1)) return 0.0f;
                return load_io(reinterpret_cast<const IO *>(p.dx_last) + ((int64_t)s.seq * (W - 1) + (t - (s.hi - (W - 1)))) * p.D + d);
            };
            auto g_at = [&](const ConvSpan &s, int64_t t) { return t < s.hi ? load_io(now.dy + (t - t0)) * conv_dact<IO, SILU>(conv_pre<IO, W>(p, s, b, t, d)) : 0.0f; };
            if (fresh)
#pragma unroll
                for (int i = 0; i < W - 1; ++i) after[i] = !p.cu && now.len < now.rest ? g_at(own, t0 + now.len + i) : 0.0f;
            fresh = first == 0;
            if (!p.cu) {
                float xs[VEC + W - 1], g[VEC + W - 1], out[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) xs[W - 1 + e] = in.x.get(e);
                if constexpr (VEC >= W - 1) {
#pragma unroll
                    for (int i = 0; i < W - 1; ++i) {
                        const float before = dpp<DPP_WAVE_SHR1>(0.0f, xs[VEC + i]);
                        xs[i] = lane == 0 ? in.before.get(4 - (W - 1) + i) : before;
                    }
                }
                if (VEC < W - 1 || t0 + first == 0) {      // (else the first lane starts at step 4 at least)
                    if (VEC < W - 1 ? l < now.len : lane == 0)         // (the row's first piece)
#pragma unroll
                        for (int i = 0; i < W - 1; ++i) xs[i] = conv_input<IO, W>(p, own, b, t0 + l + i - (W - 1), d);
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float z = bias;
#pragma unroll
                    for (int j = 0; j < W; ++j) z = __builtin_fmaf(w[j], xs[e + j], z);
                    g[e] = in.dy.get(e) * conv_dact<IO, SILU>(z);
#pragma unroll
                    for (int j = 0; j < W; ++j) dw[j] = __builtin_fmaf(g[e], xs[e + j], dw[j]);
                    dw[W] += g[e];
                }
                if constexpr (VEC >= W - 1) {
#pragma unroll
                    for (int i = 0; i < W - 1; ++i) {
                        const float next = dpp<DPP_WAVE_SHL1>(0.0f, g[i]);
                        g[VEC + i] = lane == side - 1 ? after[i] : next;
                        after[i] = __shfl(g[i], tid & 63 & ~(side - 1), 64);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < W - 1; ++i) g[VEC + i] = l < now.len ? g_at(own, t0 + l + VEC + i) : 0.0f;
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float a = 0.0f;
#pragma unroll
                    for (int j = 0; j < W; ++j) a = __builtin_fmaf(w[j], g[e + W - 1 - j], a);
                    out[e] = a;
                }
                if (p.dx_last && l + VEC > now.rest - (W - 1))
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (l + e < now.len) out[e] += from_last(own, t0 + l + e);
                if (d0 < p.D) {
                    if (l + VEC <= now.len) Few<IO, VEC>::store(dx + l, out);
                    else if (l < now.len)
#pragma unroll
                        for (int e = 0; e < VEC; ++e)
                            if (l + e < now.len) store_io(dx + l + e, out[e]);
                }
                continue;
            }
            if (d0 < p.D)
                for (int i = l; i < l + VEC && i < now.len; ++i) {
                    const ConvSpan q = conv_span(p, b, t0 + i);
                    float a = 0.0f;
                    if (q.in) {
#pragma unroll 1
                        for (int j = 0; j < W; ++j) {                    // g of step i + (W - 1) - j
                            const float h = g_at(q, t0 + i + (W - 1) - j);
                            a = __builtin_fmaf(p.w[(int64_t)d * W + j], h, a);
                            if (j == W - 1) {
#pragma unroll
                                for (int u = 0; u < W; ++u) dw[u] = __builtin_fmaf(h, conv_input<IO, W>(p, q, b, t0 + i - (W - 1) + u, d), dw[u]);
                                dw[W] += h;
                            }
                        }
                        a += from_last(q, t0 + i);
                    }
                    store_io(dx + i, a);
                }
        }
    }
#pragma unroll
    for (int j = 0; j <= W; ++j) {
        for (int m = 1; m < side; m <<= 1) dw[j] += __shfl_xor(dw[j], m, 64);
        if (lane == 0 && d0 < p.D) p.sums[((int64_t)blockIdx.x * (W + 1) + j) * p.D + d0] = dw[j];
    }
}

template <class IO, int W, int VEC, bool SILU, bool BWD> hipError_t run_time(const ConvParams &p, hipStream_t s) {
    const int rows = 256 >> p.shift;
    const unsigned y = (unsigned)((p.D + rows - 1) / rows);
    const unsigned more = BWD ? (p.dx0 ? conv_blocks((int64_t)p.seqs * p.D) : 0) : (p.x_last ? conv_blocks((int64_t)p.seqs * (W - 1) * p.D) : 0);
    const dim3 grid((unsigned)p.blocks + (more + y - 1) / y, y);
    if constexpr (BWD) hipLaunchKernelGGL((k_conv_time_bwd<IO, W, VEC, SILU>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((k_conv_time_fwd<IO, W, VEC, SILU>), grid, dim3(256), 0, s, p);
    return hipGetLastError();
}
template <class IO, int V, bool SILU, bool BWD> hipError_t time_of(const ConvParams &p, hipStream_t s) {
    switch (p.W) {
    case 2: return run_time<IO, 2, V, SILU, BWD>(p, s);
    case 3: return run_time<IO, 3, V, SILU, BWD>(p, s);
    default: return run_time<IO, 4, V, SILU, BWD>(p, s);
    }
}
template <class IO, bool SILU> hipError_t time_axis(const ConvParams &p, bool bwd, hipStream_t s) {
    constexpr int V = kFew<IO>;
    if (p.L < V) return bwd ? time_of<IO, 1, SILU, true>(p, s) : time_of<IO, 1, SILU, false>(p, s);
    return bwd ? time_of<IO, 2 * V, SILU, true>(p, s) : time_of<IO, V, SILU, false>(p, s);
}
hipError_t launch_conv_time(const ConvParams &p, bool bwd, hipStream_t s) {
    if (p.act) return p.io ? time_axis<uint16_t, false>(p, bwd, s) : time_axis<float, false>(p, bwd, s);
    return p.io ? time_axis<uint16_t, true>(p, bwd, s) : time_axis<float, true>(p, bwd, s);
}

static int log2_up(int64_t n, int most) {
    int s = 0;
    while (s < most && ((int64_t)1 << s) < n) ++s;
    return s;
}
void plan_conv(ConvParams &p, bool backward) {
    const int64_t along = p.time_last ? p.L : p.D, wide = p.io ? 8 : 4, each = along < wide ? 1 : !backward ? wide : p.time_last ? 2 * wide : wide / 2, pieces = (along + each - 1) / each;
    p.shift = log2_up(pieces, 6);
    const int side = 256 >> p.shift;
    int64_t groups;                                        // workgroups of a tile
    if (p.time_last) {
        const int64_t visit = each << p.shift, rows = (int64_t)p.B * p.D;
        int64_t n = rows * ((p.L + visit - 1) / visit) * (1 << p.shift) / 64 / (backward ? 4096 : 8192);      // wavefronts' visits over the chip
        n = n < 1 ? 1 : n > 8 ? 8 : n;
        p.tile = (int)(visit * n);
        groups = ((int64_t)p.D + side - 1) / side;
    } else {
        // as many steps to a thread as leave every compute unit three (backward; their registers' number) or four workgroups, in as few equal turns as 128 or 64 steps allow
        groups = (pieces + (1 << p.shift) - 1) >> p.shift;
        const int64_t at_once = (backward ? 768 : 1024) / groups, slots = (at_once < 1 ? 1 : at_once) * side, most = backward ? 128 : 64;
        int64_t n = ((int64_t)p.B * p.L + slots - 1) / slots;
        n = n <= most ? n : (n + (n + most - 1) / most - 1) / ((n + most - 1) / most);
        p.tile = (int)(n < 8 ? 8 : (n + 3) / 4 * 4);
    }
    p.tiles_each = (p.L + p.tile - 1) / p.tile;
    p.tiles = p.B * p.tiles_each;
    const int64_t blocks = p.time_last ? p.tiles : (p.tiles + side - 1) / side;
    int64_t most = 768 / groups;
    if (most < 1) most = 1;
    p.blocks = (int)(backward && blocks > most ? most : blocks);
}

}  // namespace lrnnx
