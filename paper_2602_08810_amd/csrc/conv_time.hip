// Short causal convolution with an activation, time axis contiguous ([B,D,L]): the formulas of the other layout's kernels.
// The lanes of a row take a 16-byte piece of the time axis each, side by side; the W - 1 inputs before a piece, and backward the W - 1 steps after it (whose g
// each piece forms again), come from a second, narrower access that the first level of cache has.  Bound by memory.
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
// elements at steps l .. l + W - 2 of a row, zero from `end` on
template <class IO, int W> __device__ __forceinline__ void time_after(const IO *row, int64_t l, int64_t end, float *xs) {
    if (l + 4 <= end) {
        Few<IO, 4> v;
        v.load(row + l);
#pragma unroll
        for (int i = 0; i < W - 1; ++i) xs[i] = v.get(i);
    } else {
#pragma unroll
        for (int i = 0; i < W - 1; ++i) xs[i] = l + i < end ? load_io(row + l + i) : 0.0f;
    }
}

template <class IO, int W, int VEC> __global__ __launch_bounds__(256) void k_conv_time_fwd(const ConvParams p) {
    const int tid = threadIdx.x, lane = tid & ((1 << p.shift) - 1), d = blockIdx.y * (256 >> p.shift) + (tid >> p.shift);
    if ((int)blockIdx.x >= p.blocks) {
        conv_last<IO, W>(p, ((int64_t)(blockIdx.x - p.blocks) * gridDim.y + blockIdx.y) * 256 + tid, (int64_t)(gridDim.x - p.blocks) * gridDim.y * 256);
        return;
    }
    if (d >= p.D) return;
    const int b = p.cu ? 0 : (int)(blockIdx.x / p.tiles_each);
    const int64_t t0 = (blockIdx.x - (int64_t)b * p.tiles_each) * p.tile, t1 = t0 + p.tile < p.L ? t0 + p.tile : p.L;
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
                out[e] = conv_act<IO>(z, p.act);
            }
            Few<IO, VEC>::store(y + l, out);
        } else {
            for (int64_t t = l; t < l + VEC; ++t) {
                const ConvSpan q = conv_span(p, b, t);
                if (q.in) store_io(y + t, conv_act<IO>(conv_pre<IO, W>(p, q, b, t, d), p.act));
            }
        }
    }
}

template <class IO, int W, int VEC> __global__ __launch_bounds__(256) void k_conv_time_bwd(const ConvParams p) {
    const int tid = threadIdx.x, lane = tid & ((1 << p.shift) - 1), d = blockIdx.y * (256 >> p.shift) + (tid >> p.shift);
    if ((int)blockIdx.x >= p.blocks) {
        conv_dx0<IO, W>(p, ((int64_t)(blockIdx.x - p.blocks) * gridDim.y + blockIdx.y) * 256 + tid, (int64_t)(gridDim.x - p.blocks) * gridDim.y * 256);
        return;
    }
    float dw[W + 1] = {};
    if (d < p.D) {
        float w[W];
        const float bias = p.bias ? p.bias[d] : 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] = p.w[(int64_t)d * W + j];
        for (int64_t slot = blockIdx.x; slot < p.tiles; slot += p.blocks) {
            const int b = p.cu ? 0 : (int)(slot / p.tiles_each);
            const int64_t t0 = (slot - (int64_t)b * p.tiles_each) * p.tile, t1 = t0 + p.tile < p.L ? t0 + p.tile : p.L;
            const IO *x = reinterpret_cast<const IO *>(p.x) + b * p.x_b + d * p.x_d, *dy = reinterpret_cast<const IO *>(p.dy) + b * p.dy_b + d * p.dy_d;
            IO *dx = reinterpret_cast<IO *>(p.dx) + b * p.y_b + d * p.y_d;
            auto from_last = [&](const ConvSpan &s, int64_t t) {         // what the last inputs' gradient brings to step t
                if (!p.dx_last || t < s.hi - (W - 1)) return 0.0f;
                return load_io(reinterpret_cast<const IO *>(p.dx_last) + ((int64_t)s.seq * (W - 1) + (t - (s.hi - (W - 1)))) * p.D + d);
            };
            for (int64_t piece = t0 + lane * VEC; piece < t1; piece += VEC << p.shift) {
                const int64_t l = piece + VEC <= p.L ? piece : p.L - VEC;
                const ConvSpan s = conv_span(p, b, l);
                if (s.in && l + VEC <= s.hi) {
                    Few<IO, VEC> in, up;
                    in.load(x + l);
                    up.load(dy + l);
                    float xs[VEC + 2 * (W - 1)], g[VEC + W - 1], out[VEC];
                    time_before<IO, W>(p, s, x, b, l, d, xs);
                    time_after<IO, W>(x, l + VEC, s.hi, xs + VEC + W - 1);
                    time_after<IO, W>(dy, l + VEC, s.hi, g + VEC);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) { xs[W - 1 + e] = in.get(e); g[e] = up.get(e); }
#pragma unroll
                    for (int e = 0; e < VEC + W - 1; ++e) {
                        float z = bias;
#pragma unroll
                        for (int j = 0; j < W; ++j) z = __builtin_fmaf(w[j], xs[e + j], z);
                        g[e] = e < VEC || l + e < s.hi ? g[e] * conv_dact<IO>(z, p.act) : 0.0f;
                    }
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        if (l + e >= piece) {
#pragma unroll
                            for (int j = 0; j < W; ++j) dw[j] = __builtin_fmaf(g[e], xs[e + j], dw[j]);
                            dw[W] += g[e];
                        }
                        float a = 0.0f;
#pragma unroll
                        for (int j = 0; j < W; ++j) a = __builtin_fmaf(w[j], g[e + W - 1 - j], a);
                        out[e] = a;
                    }
                    if (l + VEC > s.hi - (W - 1))
#pragma unroll
                        for (int e = 0; e < VEC; ++e) out[e] += from_last(s, l + e);
                    Few<IO, VEC>::store(dx + l, out);
                } else {
                    for (int64_t t = l; t < l + VEC; ++t) {
                        const ConvSpan q = conv_span(p, b, t);
                        float a = 0.0f;
                        if (q.in) {
#pragma unroll 1
                            for (int j = 0; j < W; ++j) {                // g of step t + (W - 1) - j
                                const int64_t at = t + (W - 1) - j;
                                if (at >= q.hi) continue;
                                const float h = load_io(dy + at) * conv_dact<IO>(conv_pre<IO, W>(p, q, b, at, d), p.act);
                                a = __builtin_fmaf(p.w[(int64_t)d * W + j], h, a);
                                if (at == t && t >= piece) {
#pragma unroll
                                    for (int i = 0; i < W; ++i) dw[i] = __builtin_fmaf(h, conv_input<IO, W>(p, q, b, t - (W - 1) + i, d), dw[i]);
                                    dw[W] += h;
                                }
                            }
                            a += from_last(q, t);
                        }
                        store_io(dx + t, a);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j <= W; ++j) {
        for (int m = 1; m < 1 << p.shift; m <<= 1) dw[j] += __shfl_xor(dw[j], m, 64);
        if (lane == 0 && d < p.D) p.sums[((int64_t)blockIdx.x * (W + 1) + j) * p.D + d] = dw[j];
    }
}

template <class IO, int W, int VEC> hipError_t run_time(const ConvParams &p, bool bwd, hipStream_t s) {
    const int rows = 256 >> p.shift;
    const unsigned y = (unsigned)((p.D + rows - 1) / rows);
    const unsigned more = bwd ? (p.dx0 ? conv_blocks((int64_t)p.seqs * p.D) : 0) : (p.x_last ? conv_blocks((int64_t)p.seqs * (W - 1) * p.D) : 0);
    const dim3 grid((unsigned)p.blocks + (more + y - 1) / y, y);
    if (bwd) hipLaunchKernelGGL((k_conv_time_bwd<IO, W, VEC>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((k_conv_time_fwd<IO, W, VEC>), grid, dim3(256), 0, s, p);
    return hipGetLastError();
}
template <class IO> hipError_t time_axis(const ConvParams &p, bool bwd, hipStream_t s) {
    constexpr int V = kFew<IO>;
    const bool vec = p.L >= V;
    switch (p.W) {
    case 2: return vec ? run_time<IO, 2, V>(p, bwd, s) : run_time<IO, 2, 1>(p, bwd, s);
    case 3: return vec ? run_time<IO, 3, V>(p, bwd, s) : run_time<IO, 3, 1>(p, bwd, s);
    default: return vec ? run_time<IO, 4, V>(p, bwd, s) : run_time<IO, 4, 1>(p, bwd, s);
    }
}
hipError_t launch_conv_time_fwd(const ConvParams &p, hipStream_t s) { return p.io ? time_axis<uint16_t>(p, false, s) : time_axis<float>(p, false, s); }
hipError_t launch_conv_time_bwd(const ConvParams &p, hipStream_t s) { return p.io ? time_axis<uint16_t>(p, true, s) : time_axis<float>(p, true, s); }

static int log2_up(int64_t n, int most) {
    int s = 0;
    while (s < most && ((int64_t)1 << s) < n) ++s;
    return s;
}
void plan_conv(ConvParams &p, bool backward) {
    const int64_t along = p.time_last ? p.L : p.D, each = p.io ? 8 : 4, pieces = along >= each ? (along + each - 1) / each : along;
    p.shift = log2_up(pieces, 6);
    const int side = 256 >> p.shift;
    int64_t groups;                                        // workgroups of a tile
    if (p.time_last) {
        const int64_t visit = (along >= each ? each : 1) << p.shift, rows = (int64_t)p.B * p.D;
        int64_t n = rows * ((p.L + visit - 1) / visit) * (1 << p.shift) / 64 / (backward ? 4096 : 8192);      // wavefronts' visits over the chip
        n = n < 1 ? 1 : n > 8 ? 8 : n;
        p.tile = (int)(visit * n);
        groups = ((int64_t)p.D + side - 1) / side;
    } else {
        int64_t n = (int64_t)p.B * p.L * pieces / 262144;
        const int least = backward ? 8 : 4, most = backward ? 64 : 32;
        p.tile = (int)(n < least ? least : n > most ? most : n / 4 * 4);
        groups = (pieces + (1 << p.shift) - 1) >> p.shift;
    }
    p.tiles_each = (p.L + p.tile - 1) / p.tile;
    p.tiles = p.B * p.tiles_each;
    const int64_t blocks = p.time_last ? p.tiles : (p.tiles + side - 1) / side;
    int64_t most = 1024 / groups;
    if (most < 1) most = 1;
    p.blocks = (int)(backward && blocks > most ? most : blocks);
}

}  // namespace lrnnx
