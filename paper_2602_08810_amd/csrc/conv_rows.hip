// Short causal convolution with an activation, channels contiguous ([B,L,D]):
//     pre[l] = bias + sum_j w[j] x[l-(W-1)+j],   y = act(pre);   a step of generation from the last W - 1 inputs.
// Backward, with pre formed again: g = dy act'(pre), dx[l] = sum_j w[j] g[l+(W-1)-j], dw[j] = sum g[l] x[l-(W-1)+j], dbias = sum g.
// A thread walks the time axis for the channels of one 16-byte access, the last inputs (and, backward, the last g) in registers: every input is read from
// memory once but for the W - 1 steps around a tile, which the caches have.  Bound by memory.
// 4 x 4096 x 6144 in bfloat16: forward 92 us (4.4 TB/s), backward 141 (4.3), in float32 175 and 257 (4.6, 4.7), each in a loop of its own; in turns, as in training, 81 and 154, 162 and 268 (what
// one wrote last is still on its way to memory in the other); a copy of as much 76 and 150.  Backward a piece is 8 bytes: in
// pieces of 16 inputs, g and sums do not fit 256 registers (22 to 26 spilled in bfloat16 with four weights), and a compute unit has two workgroups, not three.
// The weights' gradients are summed in registers over all tiles of a thread, over a workgroup through LDS, and over workgroups by a second launch, in a fixed order.
#include "conv_common.hpp"

namespace lrnnx {

constexpr int kConvAhead = 4;                             // steps loaded at a time
// workgroups of a step, two a compute unit: 256 entries of 8192 channels 6.3 us, with 1024 7.1, 4096 (an entry a thread) 8.6; 1024 entries 21, 22, 24
constexpr int kStepBlocks = 512;

template <class IO, int W, int VEC> struct ConvWeights {
    float w[W][VEC], b[VEC];
    __device__ __forceinline__ void load(const float *weight, const float *bias, int d) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            b[e] = bias ? bias[d + e] : 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][e] = weight[(int64_t)(d + e) * W + j];
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

// Steps l .. l + kConvAhead - 1 of a row, the last one before `end` for those behind it
template <class IO, int VEC> struct RowsAhead {
    Few<IO, VEC> v[kConvAhead];
    __device__ __forceinline__ void load(const IO *x, int64_t stride, int64_t l) {
#pragma unroll
        for (int u = 0; u < kConvAhead; ++u) v[u].load(x + (l + u) * stride);
    }
    __device__ __forceinline__ void load(const IO *x, int64_t stride, int64_t l, int64_t end) {
#pragma unroll
        for (int u = 0; u < kConvAhead; ++u) v[u].load(x + (l + u < end ? l + u : end - 1) * stride);
    }
};
// WHOLE: all steps lie before `end`.
template <class IO, int W, int VEC, bool SILU, bool WHOLE> __device__ __forceinline__ void rows_fwd_steps(const ConvParams &p, const ConvWeights<IO, W, VEC> &k, const RowsAhead<IO, VEC> &in, IO *y, int64_t l,
                                                                                                         int64_t end, float (&seen)[W - 1][VEC]) {
#pragma unroll
    for (int u = 0; u < kConvAhead; ++u) {
        float out[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float now = in.v[u].get(e);
            float z = k.b[e];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) z = __builtin_fmaf(k.w[j][e], seen[j][e], z);
            out[e] = conv_act<IO, SILU>(__builtin_fmaf(k.w[W - 1][e], now, z));
#pragma unroll
            for (int j = 0; j + 1 < W - 1; ++j) seen[j][e] = seen[j + 1][e];
            seen[W - 2][e] = now;
        }
        if (WHOLE || l + u < end) Few<IO, VEC>::store(y + (l + u) * p.y_l, out);
    }
}
template <class IO, int W, int VEC, bool SILU> __global__ __launch_bounds__(256) void k_conv_rows_fwd(const ConvParams p) {
    const int tid = threadIdx.x, c = (blockIdx.y << p.shift) + (tid & ((1 << p.shift) - 1));
    if ((int)blockIdx.x >= p.blocks) {
        conv_last<IO, W>(p, ((int64_t)(blockIdx.x - p.blocks) * gridDim.y + blockIdx.y) * 256 + tid, (int64_t)(gridDim.x - p.blocks) * gridDim.y * 256);
        return;
    }
    const int64_t slot = (int64_t)blockIdx.x * (256 >> p.shift) + (tid >> p.shift);
    if (slot >= p.tiles || (int64_t)c * VEC >= p.D) return;
    const int d = c * VEC + VEC <= p.D ? c * VEC : p.D - VEC;            // the last piece overlaps the one before
    const int b = p.cu ? 0 : (int)((unsigned)slot / (unsigned)p.tiles_each);
    const int64_t t0 = (slot - (int64_t)b * p.tiles_each) * p.tile, t1 = t0 + p.tile < p.L ? t0 + p.tile : p.L;
    const IO *x = reinterpret_cast<const IO *>(p.x) + b * p.x_b + d;
    IO *y = reinterpret_cast<IO *>(p.y) + b * p.y_b + d;
    ConvWeights<IO, W, VEC> k;
    k.load(p.w, p.bias, d);
    int after = 0;
    for (int64_t l = t0; l < t1;) {
        const ConvSpan s = conv_span(p, b, l, after);
        after = s.seq + 1;
        const int64_t end = s.hi < t1 ? s.hi : t1;
        if (!s.in) { l = end; continue; }
        float seen[W - 1][VEC];
        conv_before<IO, W, VEC>(p, s, x, l, d, seen);
        RowsAhead<IO, VEC> in, next;                      // what comes after is on its way while this is worked on
        in.load(x, p.x_l, l, end);
        for (; l + 2 * kConvAhead <= end; l += kConvAhead) {
            next.load(x, p.x_l, l + kConvAhead);
            rows_fwd_steps<IO, W, VEC, SILU, true>(p, k, in, y, l, end, seen);
            in = next;
        }
        for (; l < end; l += kConvAhead) {
            rows_fwd_steps<IO, W, VEC, SILU, false>(p, k, in, y, l, end, seen);
            in.load(x, p.x_l, l + kConvAhead, end);
        }
        l = end;
    }
}

// What a walk back carries along: the last inputs, the last g (g[i]: of the step i - (W - 1) from now), and the weights' gradients
template <int W, int VEC> struct RowsBack {
    float seen[W - 1][VEC], g[W][VEC], dw[W + 1][VEC];
};
// Steps l .. l + kConvAhead - 1 of the steps [first, end) of sequence `s`; INSIDE: they and the steps whose dx they complete are all of these, and none of the sequence's last W - 1.
template <class IO, int W, int VEC, bool SILU, bool INSIDE> __device__ __forceinline__ void rows_bwd_steps(const ConvParams &p, const ConvWeights<IO, W, VEC> &k, const ConvSpan &s, const RowsAhead<IO, VEC> &in,
                                                                                                          const RowsAhead<IO, VEC> &up, IO *dx, int d, int64_t l, int64_t first, int64_t end, RowsBack<W, VEC> &r) {
#pragma unroll
    for (int u = 0; u < kConvAhead; ++u) {
        const bool within = INSIDE || l + u < s.hi, mine = INSIDE || l + u < end;
        float out[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float now = in.v[u].get(e);
            float z = k.b[e];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) z = __builtin_fmaf(k.w[j][e], r.seen[j][e], z);
            z = __builtin_fmaf(k.w[W - 1][e], now, z);
            float h = up.v[u].get(e) * conv_dact<IO, SILU>(z);
            h = within ? h : 0.0f;
#pragma unroll
            for (int j = 0; j + 1 < W; ++j) r.g[j][e] = r.g[j + 1][e];
            r.g[W - 1][e] = h;
            if (mine) {
#pragma unroll
                for (int j = 0; j < W - 1; ++j) r.dw[j][e] = __builtin_fmaf(h, r.seen[j][e], r.dw[j][e]);
                r.dw[W - 1][e] = __builtin_fmaf(h, now, r.dw[W - 1][e]);
                r.dw[W][e] += h;
            }
#pragma unroll
            for (int j = 0; j + 1 < W - 1; ++j) r.seen[j][e] = r.seen[j + 1][e];
            r.seen[W - 2][e] = now;
            float a = 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j) a = __builtin_fmaf(k.w[j][e], r.g[W - 1 - j][e], a);
            out[e] = a;
        }
        const int64_t t = l + u - (W - 1);
        if (INSIDE || (t >= first && t < end)) {
            if (!INSIDE && p.dx_last && t >= s.hi - (W - 1)) {
                Few<IO, VEC> v;
                v.load(reinterpret_cast<const IO *>(p.dx_last) + ((int64_t)s.seq * (W - 1) + (t - (s.hi - (W - 1)))) * p.D + d);
#pragma unroll
                for (int e = 0; e < VEC; ++e) out[e] += v.get(e);
            }
            Few<IO, VEC>::store(dx + t * p.y_l, out);
        }
    }
}
template <class IO, int W, int VEC, bool SILU> __global__ __launch_bounds__(256, 3) void k_conv_rows_bwd(const ConvParams p) {
    __shared__ float lds[256 * VEC];
    const int tid = threadIdx.x, across = 1 << p.shift, c = (blockIdx.y << p.shift) + (tid & (across - 1));
    if ((int)blockIdx.x >= p.blocks) {
        conv_dx0<IO, W, SILU>(p, ((int64_t)(blockIdx.x - p.blocks) * gridDim.y + blockIdx.y) * 256 + tid, (int64_t)(gridDim.x - p.blocks) * gridDim.y * 256);
        return;
    }
    const bool there = (int64_t)c * VEC < p.D;
    const int d = c * VEC + VEC <= p.D ? c * VEC : p.D - VEC;
    RowsBack<W, VEC> r = {};
    if (there) {
        ConvWeights<IO, W, VEC> k;
        k.load(p.w, p.bias, d);
        for (int64_t slot = (int64_t)blockIdx.x * (256 >> p.shift) + (tid >> p.shift); slot < p.tiles; slot += (int64_t)p.blocks * (256 >> p.shift)) {
            const int b = p.cu ? 0 : (int)((unsigned)slot / (unsigned)p.tiles_each);
            const int64_t t0 = (slot - (int64_t)b * p.tiles_each) * p.tile, t1 = t0 + p.tile < p.L ? t0 + p.tile : p.L;
            const IO *x = reinterpret_cast<const IO *>(p.x) + b * p.x_b + d, *dy = reinterpret_cast<const IO *>(p.dy) + b * p.dy_b + d;
            IO *dx = reinterpret_cast<IO *>(p.dx) + b * p.y_b + d;
            int after = 0;
            for (int64_t first = t0; first < t1;) {
                const ConvSpan s = conv_span(p, b, first, after);
                after = s.seq + 1;
                const int64_t end = s.hi < t1 ? s.hi : t1;
                if (!s.in) {                              // steps outside every sequence
                    const float none[VEC] = {};
                    for (int64_t l = first; l < end; ++l) Few<IO, VEC>::store(dx + l * p.y_l, none);
                    first = end;
                    continue;
                }
                conv_before<IO, W, VEC>(p, s, x, first, d, r.seen);
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) r.g[j][e] = 0.0f;
                // the first steps complete nothing, the last are another tile's or none
                RowsAhead<IO, VEC> in, up, in2, up2;
                int64_t l = first;
                in.load(x, p.x_l, l, s.hi);
                up.load(dy, p.dy_l, l, s.hi);
                auto edge = [&]() {
                    rows_bwd_steps<IO, W, VEC, SILU, false>(p, k, s, in, up, dx, d, l, first, end, r);
                    l += kConvAhead;
                    in.load(x, p.x_l, l, s.hi);
                    up.load(dy, p.dy_l, l, s.hi);
                };
                edge();
                for (; l + 2 * kConvAhead <= end; l += kConvAhead) {
                    in2.load(x, p.x_l, l + kConvAhead);
                    up2.load(dy, p.dy_l, l + kConvAhead);
                    rows_bwd_steps<IO, W, VEC, SILU, true>(p, k, s, in, up, dx, d, l, first, end, r);
                    in = in2;
                    up = up2;
                }
                while (l < end + (W - 1)) edge();
                first = end;
            }
        }
    }
    // over the workgroup, one weight after the other
    const int cols = across * VEC, column = tid & (across - 1);
#pragma unroll
    for (int j = 0; j <= W; ++j) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) lds[(tid >> p.shift) * cols + column * VEC + e] = r.dw[j][e];
        __syncthreads();
        for (int i = tid; i < cols; i += 256) {
            float sum = 0.0f;
            for (int q = 0; q < 256 >> p.shift; ++q) sum += lds[q * cols + i];
            const int64_t piece = ((int64_t)blockIdx.y << p.shift) + i / VEC, at = piece * VEC + VEC <= p.D ? piece * VEC : (int64_t)p.D - VEC, ch = at + i % VEC;
            if (piece * VEC < p.D && ch >= piece * VEC) p.sums[((int64_t)blockIdx.x * (W + 1) + j) * p.D + ch] = sum;       // (what overlaps is the piece before's)
        }
        __syncthreads();
    }
}

// dw [D,W] and dbias [D] from the parts: 64 channels a workgroup, 16 rows of parts side by side.
__global__ __launch_bounds__(1024) void k_conv_sums(const ConvParams p) {
    __shared__ float lds[16][64];
    const int j = blockIdx.y, lane = threadIdx.x & 63, row = threadIdx.x >> 6;
    const int64_t d = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (d < p.D)
#pragma unroll 4
        for (int i = row; i < p.blocks; i += 16) s += p.sums[((int64_t)i * (p.W + 1) + j) * p.D + d];
    lds[row][lane] = s;
    __syncthreads();
    if (row == 0 && d < p.D) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += lds[i][lane];
        if (j < p.W) p.dw[d * p.W + j] = s;
        else p.db[d] = s;
    }
}
hipError_t launch_conv_sums(const ConvParams &p, hipStream_t s) {
    hipLaunchKernelGGL(k_conv_sums, dim3((unsigned)(((int64_t)p.D + 63) / 64), (unsigned)(p.W + (p.db ? 1 : 0))), dim3(1024), 0, s, p);
    return hipGetLastError();
}

template <class IO, int W, int VEC, bool SILU, bool BWD> hipError_t run_rows(const ConvParams &p, hipStream_t s) {
    const int64_t pieces = (p.D + VEC - 1) / VEC;
    const unsigned y = (unsigned)((pieces + (1 << p.shift) - 1) >> p.shift);
    const unsigned more = BWD ? (p.dx0 ? conv_blocks((int64_t)p.seqs * p.D) : 0) : (p.x_last ? conv_blocks((int64_t)p.seqs * (W - 1) * p.D) : 0);
    const dim3 grid((unsigned)p.blocks + (more + y - 1) / y, y);
    if constexpr (BWD) hipLaunchKernelGGL((k_conv_rows_bwd<IO, W, VEC, SILU>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((k_conv_rows_fwd<IO, W, VEC, SILU>), grid, dim3(256), 0, s, p);
    return hipGetLastError();
}
template <class IO, int V, bool SILU, bool BWD> hipError_t rows_of(const ConvParams &p, hipStream_t s) {
    switch (p.W) {
    case 2: return run_rows<IO, 2, V, SILU, BWD>(p, s);
    case 3: return run_rows<IO, 3, V, SILU, BWD>(p, s);
    default: return run_rows<IO, 4, V, SILU, BWD>(p, s);
    }
}
template <class IO, bool SILU> hipError_t rows(const ConvParams &p, bool bwd, hipStream_t s) {
    constexpr int V = kFew<IO>;
    if (p.D < V) return bwd ? rows_of<IO, 1, SILU, true>(p, s) : rows_of<IO, 1, SILU, false>(p, s);
    return bwd ? rows_of<IO, V / 2, SILU, true>(p, s) : rows_of<IO, V, SILU, false>(p, s);
}
hipError_t launch_conv_rows(const ConvParams &p, bool bwd, hipStream_t s) {
    if (p.act) return p.io ? rows<uint16_t, false>(p, bwd, s) : rows<float, false>(p, bwd, s);
    return p.io ? rows<uint16_t, true>(p, bwd, s) : rows<float, true>(p, bwd, s);
}

// One token: VEC channels of a batch entry a thread, and of the entries gridDim.y further on, for which it has the weights already (they are more bytes than an
// entry's inputs); the carried inputs move on by one in place.
template <class IO, int W, int VEC> __global__ __launch_bounds__(256) void k_conv_step(const ConvStepParams p) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if ((int64_t)c * VEC >= p.D) return;
    const int d = c * VEC;
    ConvWeights<IO, W, VEC> k;
    k.load(p.w, p.bias, d);
    for (int b = blockIdx.y; b < p.B; b += gridDim.y) {
        IO *state = reinterpret_cast<IO *>(p.state) + (int64_t)b * (W - 1) * p.D + d;
        Few<IO, VEC> in[W];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) in[j].load(state + (int64_t)j * p.D);
        in[W - 1].load(reinterpret_cast<const IO *>(p.x) + b * p.x_b + d * p.x_d);
        float out[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            float z = k.b[e];
#pragma unroll
            for (int j = 0; j < W; ++j) z = __builtin_fmaf(k.w[j][e], in[j].get(e), z);
            out[e] = p.act ? conv_act<IO, false>(z) : conv_act<IO, true>(z);
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
}
template <class IO, int W, int V> hipError_t step_of(const ConvStepParams &p, hipStream_t s) {
    const int x = (p.D / V + 255) / 256, most = kStepBlocks / x < 1 ? 1 : kStepBlocks / x;
    hipLaunchKernelGGL((k_conv_step<IO, W, V>), dim3((unsigned)x, (unsigned)(p.B < most ? p.B : most)), dim3(256), 0, s, p);
    return hipGetLastError();
}
template <class IO, int W> hipError_t run_step(const ConvStepParams &p, hipStream_t s) {
    return p.x_d == 1 && p.y_d == 1 && p.D % 4 == 0 ? step_of<IO, W, 4>(p, s) : step_of<IO, W, 1>(p, s);
}
hipError_t launch_conv_step(const ConvStepParams &p, hipStream_t s) {
    switch (p.W) {
    case 2: return p.io ? run_step<uint16_t, 2>(p, s) : run_step<float, 2>(p, s);
    case 3: return p.io ? run_step<uint16_t, 3>(p, s) : run_step<float, 3>(p, s);
    default: return p.io ? run_step<uint16_t, 4>(p, s) : run_step<float, 4>(p, s);
    }
}

}  // namespace lrnnx
