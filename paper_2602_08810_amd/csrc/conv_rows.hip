// Short causal convolution with an activation, channels contiguous ([B,L,D]):
//     pre[l] = bias + sum_j w[j] x[l-(W-1)+j],   y = act(pre);   a step of generation from the last W - 1 inputs.
// Backward, with pre formed again: g = dy act'(pre), dx[l] = sum_j w[j] g[l+(W-1)-j], dw[j] = sum g[l] x[l-(W-1)+j], dbias = sum g.
// A thread walks the time axis for the channels of one 16-byte access, the last inputs (and, backward, the last g) in registers: every input is read from
// memory once but for the W - 1 steps around a tile, which the caches have.  Bound by memory.
// The weights' gradients are summed in registers over all tiles of a thread, over a workgroup through LDS, and over workgroups by a second launch, in a fixed order.
#include "conv_common.hpp"

namespace lrnnx {

constexpr int kConvAhead = 4;                             // steps loaded at a time

template <class IO, int W, int VEC> struct ConvWeights {
    float w[W][VEC], b[VEC];
    __device__ __forceinline__ void load(const ConvParams &p, int d) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            b[e] = p.bias ? p.bias[d + e] : 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][e] = p.w[(int64_t)(d + e) * W + j];
        }
    }
};
// the W - 1 inputs before step l
template <class IO, int W, int VEC> __device__ __forceinline__ void conv_before(const ConvParams &p, const ConvSpan &s, const IO *x, int64_t l, int d, float (&seen)[W - 1][VEC]) {
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
        const int64_t t = l - (W - 1) + i;
        Few<IO, VEC> v{};
        if (t >= s.lo) v.load(x + t * p.x_l);
        else if (p.x0) v.load(reinterpret_cast<const IO *>(p.x0) + ((int64_t)s.seq * (W - 1) + (W - 1) + (t - s.lo)) * p.D + d);
#pragma unroll
        for (int e = 0; e < VEC; ++e) seen[i][e] = v.get(e);
    }
}

template <class IO, int W, int VEC> __global__ __launch_bounds__(256) void k_conv_rows_fwd(const ConvParams p) {
    const int tid = threadIdx.x, c = (blockIdx.y << p.shift) + (tid & ((1 << p.shift) - 1));
    if ((int)blockIdx.x >= p.blocks) {
        conv_last<IO, W>(p, ((int64_t)(blockIdx.x - p.blocks) * gridDim.y + blockIdx.y) * 256 + tid, (int64_t)(gridDim.x - p.blocks) * gridDim.y * 256);
        return;
    }
    const int64_t slot = (int64_t)blockIdx.x * (256 >> p.shift) + (tid >> p.shift);
    if (slot >= p.tiles || (int64_t)c * VEC >= p.D) return;
    const int d = c * VEC + VEC <= p.D ? c * VEC : p.D - VEC;            // the last piece overlaps the one before
    const int b = p.cu ? 0 : (int)(slot / p.tiles_each);
    const int64_t t0 = (slot - (int64_t)b * p.tiles_each) * p.tile, t1 = t0 + p.tile < p.L ? t0 + p.tile : p.L;
    const IO *x = reinterpret_cast<const IO *>(p.x) + b * p.x_b + d;
    IO *y = reinterpret_cast<IO *>(p.y) + b * p.y_b + d;
    ConvWeights<IO, W, VEC> k;
    k.load(p, d);
    for (int64_t l = t0; l < t1;) {
        const ConvSpan s = conv_span(p, b, l);
        const int64_t end = s.hi < t1 ? s.hi : t1;
        if (!s.in) { l = end; continue; }
        float seen[W - 1][VEC];
        conv_before<IO, W, VEC>(p, s, x, l, d, seen);
        for (; l < end; l += kConvAhead) {
            Few<IO, VEC> in[kConvAhead];
#pragma unroll
            for (int u = 0; u < kConvAhead; ++u) in[u].load(x + (l + u < end ? l + u : end - 1) * p.x_l);
#pragma unroll
            for (int u = 0; u < kConvAhead; ++u) {
                float out[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float now = in[u].get(e);
                    float z = k.b[e];
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) z = __builtin_fmaf(k.w[j][e], seen[j][e], z);
                    out[e] = conv_act<IO>(__builtin_fmaf(k.w[W - 1][e], now, z), p.act);
#pragma unroll
                    for (int j = 0; j + 1 < W - 1; ++j) seen[j][e] = seen[j + 1][e];
                    seen[W - 2][e] = now;
                }
                if (l + u < end) Few<IO, VEC>::store(y + (l + u) * p.y_l, out);
            }
        }
        l = end;
    }
}

template <class IO, int W, int VEC> __global__ __launch_bounds__(256) void k_conv_rows_bwd(const ConvParams p) {
    __shared__ float lds[256 * VEC];
    const int tid = threadIdx.x, across = 1 << p.shift, c = (blockIdx.y << p.shift) + (tid & (across - 1));
    if ((int)blockIdx.x >= p.blocks) {
        conv_dx0<IO, W>(p, ((int64_t)(blockIdx.x - p.blocks) * gridDim.y + blockIdx.y) * 256 + tid, (int64_t)(gridDim.x - p.blocks) * gridDim.y * 256);
        return;
    }
    const bool there = (int64_t)c * VEC < p.D;
    const int d = c * VEC + VEC <= p.D ? c * VEC : p.D - VEC;
    float dw[W + 1][VEC] = {};
    if (there) {
        ConvWeights<IO, W, VEC> k;
        k.load(p, d);
        for (int64_t slot = (int64_t)blockIdx.x * (256 >> p.shift) + (tid >> p.shift); slot < p.tiles; slot += (int64_t)p.blocks * (256 >> p.shift)) {
            const int b = p.cu ? 0 : (int)(slot / p.tiles_each);
            const int64_t t0 = (slot - (int64_t)b * p.tiles_each) * p.tile, t1 = t0 + p.tile < p.L ? t0 + p.tile : p.L;
            const IO *x = reinterpret_cast<const IO *>(p.x) + b * p.x_b + d, *dy = reinterpret_cast<const IO *>(p.dy) + b * p.dy_b + d;
            IO *dx = reinterpret_cast<IO *>(p.dx) + b * p.y_b + d;
            for (int64_t first = t0; first < t1;) {
                const ConvSpan s = conv_span(p, b, first);
                const int64_t end = s.hi < t1 ? s.hi : t1;
                if (!s.in) {                              // steps outside every sequence
                    const float none[VEC] = {};
                    for (int64_t l = first; l < end; ++l) Few<IO, VEC>::store(dx + l * p.y_l, none);
                    first = end;
                    continue;
                }
                float seen[W - 1][VEC], g[W][VEC] = {};   // g[i]: of the step i - (W - 1) from now
                conv_before<IO, W, VEC>(p, s, x, first, d, seen);
                for (int64_t l = first; l < end + (W - 1); l += kConvAhead) {
                    Few<IO, VEC> in[kConvAhead], up[kConvAhead];
#pragma unroll
                    for (int u = 0; u < kConvAhead; ++u) {
                        const int64_t t = l + u < s.hi ? l + u : s.hi - 1;
                        in[u].load(x + t * p.x_l);
                        up[u].load(dy + t * p.dy_l);
                    }
#pragma unroll
                    for (int u = 0; u < kConvAhead; ++u) {
                        const bool within = l + u < s.hi, mine = l + u < end;
                        float out[VEC];
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            const float now = in[u].get(e);
                            float z = k.b[e];
#pragma unroll
                            for (int j = 0; j < W - 1; ++j) z = __builtin_fmaf(k.w[j][e], seen[j][e], z);
                            z = __builtin_fmaf(k.w[W - 1][e], now, z);
                            const float h = within ? up[u].get(e) * conv_dact<IO>(z, p.act) : 0.0f;
#pragma unroll
                            for (int j = 0; j + 1 < W; ++j) g[j][e] = g[j + 1][e];
                            g[W - 1][e] = h;
                            if (mine) {
#pragma unroll
                                for (int j = 0; j < W - 1; ++j) dw[j][e] = __builtin_fmaf(h, seen[j][e], dw[j][e]);
                                dw[W - 1][e] = __builtin_fmaf(h, now, dw[W - 1][e]);
                                dw[W][e] += h;
                            }
#pragma unroll
                            for (int j = 0; j + 1 < W - 1; ++j) seen[j][e] = seen[j + 1][e];
                            seen[W - 2][e] = now;
                            float a = 0.0f;
#pragma unroll
                            for (int j = 0; j < W; ++j) a = __builtin_fmaf(k.w[j][e], g[W - 1 - j][e], a);
                            out[e] = a;
                        }
                        const int64_t t = l + u - (W - 1);
                        if (t >= first && t < end) {
                            if (p.dx_last && t >= s.hi - (W - 1)) {
                                Few<IO, VEC> v;
                                v.load(reinterpret_cast<const IO *>(p.dx_last) + ((int64_t)s.seq * (W - 1) + (t - (s.hi - (W - 1)))) * p.D + d);
#pragma unroll
                                for (int e = 0; e < VEC; ++e) out[e] += v.get(e);
                            }
                            Few<IO, VEC>::store(dx + t * p.y_l, out);
                        }
                    }
                }
                first = end;
            }
        }
    }
    // over the workgroup, one weight after the other
    const int cols = across * VEC, column = tid & (across - 1);
#pragma unroll
    for (int j = 0; j <= W; ++j) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) lds[(tid >> p.shift) * cols + column * VEC + e] = dw[j][e];
        __syncthreads();
        for (int i = tid; i < cols; i += 256) {
            float sum = 0.0f;
            for (int r = 0; r < 256 >> p.shift; ++r) sum += lds[r * cols + i];
            const int64_t piece = ((int64_t)blockIdx.y << p.shift) + i / VEC, at = piece * VEC + VEC <= p.D ? piece * VEC : (int64_t)p.D - VEC, ch = at + i % VEC;
            if (piece * VEC < p.D && ch >= piece * VEC) p.sums[((int64_t)blockIdx.x * (W + 1) + j) * p.D + ch] = sum;       // (what overlaps is the piece before's)
        }
        __syncthreads();
    }
}

// dw [D,W] and dbias [D] from the parts: 64 channels a workgroup, four rows of parts side by side.
__global__ __launch_bounds__(256) void k_conv_sums(const ConvParams p) {
    __shared__ float lds[4][64];
    const int j = blockIdx.y, lane = threadIdx.x & 63, row = threadIdx.x >> 6;
    const int64_t d = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (d < p.D)
        for (int i = row; i < p.blocks; i += 4) s += p.sums[((int64_t)i * (p.W + 1) + j) * p.D + d];
    lds[row][lane] = s;
    __syncthreads();
    if (row == 0 && d < p.D) {
        s = (lds[0][lane] + lds[1][lane]) + (lds[2][lane] + lds[3][lane]);
        if (j < p.W) p.dw[d * p.W + j] = s;
        else p.db[d] = s;
    }
}
hipError_t launch_conv_sums(const ConvParams &p, hipStream_t s) {
    hipLaunchKernelGGL(k_conv_sums, dim3((unsigned)(((int64_t)p.D + 63) / 64), (unsigned)(p.W + (p.db ? 1 : 0))), dim3(256), 0, s, p);
    return hipGetLastError();
}

template <class IO, int W, int VEC> hipError_t run_rows(const ConvParams &p, bool bwd, hipStream_t s) {
    const int64_t pieces = (p.D + VEC - 1) / VEC;
    const unsigned y = (unsigned)((pieces + (1 << p.shift) - 1) >> p.shift);
    const unsigned more = bwd ? (p.dx0 ? conv_blocks((int64_t)p.seqs * p.D) : 0) : (p.x_last ? conv_blocks((int64_t)p.seqs * (W - 1) * p.D) : 0);
    const dim3 grid((unsigned)p.blocks + (more + y - 1) / y, y);
    if (bwd) hipLaunchKernelGGL((k_conv_rows_bwd<IO, W, VEC>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((k_conv_rows_fwd<IO, W, VEC>), grid, dim3(256), 0, s, p);
    return hipGetLastError();
}
template <class IO> hipError_t rows(const ConvParams &p, bool bwd, hipStream_t s) {
    constexpr int V = kFew<IO>;
    const bool vec = p.D >= V;
    switch (p.W) {
    case 2: return vec ? run_rows<IO, 2, V>(p, bwd, s) : run_rows<IO, 2, 1>(p, bwd, s);
    case 3: return vec ? run_rows<IO, 3, V>(p, bwd, s) : run_rows<IO, 3, 1>(p, bwd, s);
    default: return vec ? run_rows<IO, 4, V>(p, bwd, s) : run_rows<IO, 4, 1>(p, bwd, s);
    }
}
hipError_t launch_conv_rows_fwd(const ConvParams &p, hipStream_t s) { return p.io ? rows<uint16_t>(p, false, s) : rows<float>(p, false, s); }
hipError_t launch_conv_rows_bwd(const ConvParams &p, hipStream_t s) { return p.io ? rows<uint16_t>(p, true, s) : rows<float>(p, true, s); }

// One token: VEC channels of a batch entry a thread; the carried inputs move on by one in place.
template <class IO, int W, int VEC> __global__ __launch_bounds__(256) void k_conv_step(const ConvStepParams p) {
    const int c = blockIdx.x * 256 + threadIdx.x, b = blockIdx.y;
    if ((int64_t)c * VEC >= p.D) return;
    const int d = c * VEC;
    IO *state = reinterpret_cast<IO *>(p.state) + (int64_t)b * (W - 1) * p.D + d;
    const IO *x = reinterpret_cast<const IO *>(p.x) + b * p.x_b + d * p.x_d;
    Few<IO, VEC> in[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) in[j].load(state + (int64_t)j * p.D);
    in[W - 1].load(x);
    float out[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        float z = p.bias ? p.bias[d + e] : 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) z = __builtin_fmaf(p.w[(int64_t)(d + e) * W + j], in[j].get(e), z);
        out[e] = conv_act<IO>(z, p.act);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = in[j + 1].get(e);
        Few<IO, VEC>::store(state + (int64_t)j * p.D, v);
    }
    Few<IO, VEC>::store(reinterpret_cast<IO *>(p.y) + b * p.y_b + d * p.y_d, out);
}
template <class IO, int W> hipError_t run_step(const ConvStepParams &p, hipStream_t s) {
    constexpr int V = 4;
    const bool vec = p.D % V == 0 && p.x_d == 1 && p.y_d == 1;
    const dim3 grid((unsigned)(((int64_t)p.D / (vec ? V : 1) + 255) / 256), (unsigned)p.B);
    if (vec) hipLaunchKernelGGL((k_conv_step<IO, W, V>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((k_conv_step<IO, W, 1>), grid, dim3(256), 0, s, p);
    return hipGetLastError();
}
hipError_t launch_conv_step(const ConvStepParams &p, hipStream_t s) {
    switch (p.W) {
    case 2: return p.io ? run_step<uint16_t, 2>(p, s) : run_step<float, 2>(p, s);
    case 3: return p.io ? run_step<uint16_t, 3>(p, s) : run_step<float, 3>(p, s);
    default: return p.io ? run_step<uint16_t, 4>(p, s) : run_step<float, 4>(p, s);
    }
}

}  // namespace lrnnx
