// Short causal convolution with an activation, time axis contiguous ([B,D,L]): the formulas of the other layout's kernels.
// The lanes of a row take a 16-byte piece of the time axis each, side by side; forward, the W - 1 inputs before a piece come from a second, narrower access that the
// first level of cache has.  Bound by memory: 4 x 6144 x 4096 in bfloat16 94 us forward (4.3 TB/s), 129 backward (4.7), in float32 158 and 240 (5.1, 5.0), each in a loop of its own; in turns
// 83 and 138, 151 and 259.
// A sequence of a packed batch is a row of its own, with as many lanes as one of average length needs (16384 steps of 2048 channels in bfloat16: 24 sequences 40 us
// forward and 94 backward, 400 sequences 68 and 139; with pieces that may cross a boundary, and look for theirs, 137 and 739, 250 and 1206).
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
// What the lanes of a row take at a time: a stretch of a sequence.  The slots of a packed batch (a sequence of its own row for these kernels) are counted as if every sequence
// started in a slot of its own: sequence b has those from its first step / tile + b on.  Whole wavefronts call it.
struct ConvSlot {
    int seq, b;                                            // sequence; batch entry in memory
    int64_t lo, len, t0;                                   // its first step and steps; the slot's first step in it
};
__device__ __forceinline__ ConvSlot conv_slot(const ConvParams &p, unsigned slot) {
    ConvSlot c;
    if (!p.cu) {
        c.seq = c.b = (int)(slot / (unsigned)p.tiles_each);
        c.lo = 0;
        c.len = p.L;
        c.t0 = (int64_t)(slot - (unsigned)c.b * (unsigned)p.tiles_each) << p.tile_log2;
        return c;
    }
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = p.seqs;
    while (hi - lo > 1) {                                  // 64 boundaries at a time
        const int step = (hi - lo + 63) / 64, i = lo + lane * step;
        const bool before = i < hi && (lane == 0 || (delta_clamp(p.cu[i], p.L) >> p.tile_log2) + i <= (int64_t)slot);
        const int n = __popcll(__ballot(before));
        lo += (n - 1) * step;
        hi = hi < lo + step ? hi : lo + step;
    }
    const ConvSpan s = conv_sequence(p, lo);
    c.seq = lo;
    c.b = 0;
    c.lo = s.lo;
    c.len = s.hi - s.lo;
    c.t0 = ((int64_t)slot - ((s.lo >> p.tile_log2) + lo)) << p.tile_log2;
    if (c.t0 < 0) c.t0 = c.len;                            // (boundaries that do not ascend)
    return c;
}
// Elements x[0 .. VEC) of a row, of which `left` are there
template <class IO, int VEC> __device__ __forceinline__ void store_some(IO *to, const float (&x)[VEC], int64_t left) {
    if (left >= VEC) Few<IO, VEC>::store(to, x);
    else
#pragma unroll
        for (int e = 0; e < VEC; ++e) if (e < left) store_io(to + e, x[e]);
}

template <class IO, int W, int VEC, bool SILU> __global__ __launch_bounds__(256) void k_conv_time_fwd(const ConvParams p) {
    const int tid = threadIdx.x, lane = tid & ((1 << p.shift) - 1), d = blockIdx.y * (256 >> p.shift) + (tid >> p.shift);
    if ((int)blockIdx.x >= p.blocks) {
        conv_last<IO, W>(p, ((int64_t)(blockIdx.x - p.blocks) * gridDim.y + blockIdx.y) * 256 + tid, (int64_t)(gridDim.x - p.blocks) * gridDim.y * 256);
        return;
    }
    const ConvSlot c = conv_slot(p, blockIdx.x);
    if (d >= p.D) return;
    const ConvSpan s{c.lo, c.lo + c.len, c.seq, true};
    const int64_t t1 = c.t0 + p.tile < c.len ? c.t0 + p.tile : c.len;
    const IO *x = reinterpret_cast<const IO *>(p.x) + c.b * p.x_b + d * p.x_d;
    IO *y = reinterpret_cast<IO *>(p.y) + c.b * p.y_b + d * p.y_d;
    float w[W];
    const float bias = p.bias ? p.bias[d] : 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) w[j] = p.w[(int64_t)d * W + j];
    for (int64_t piece = c.t0 + lane * VEC; piece < t1; piece += VEC << p.shift) {
        const int64_t l = c.lo + piece, left = c.len - piece;
        Few<IO, VEC> in;
        if (left >= VEC) in.load(x + l); else in.load_some(x + l, (int)left);
        float xs[VEC + W - 1], out[VEC];
        time_before<IO, W>(p, s, x, c.b, l, d, xs);
#pragma unroll
        for (int e = 0; e < VEC; ++e) xs[W - 1 + e] = in.get(e);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            float z = bias;
#pragma unroll
            for (int j = 0; j < W; ++j) z = __builtin_fmaf(w[j], xs[e + j], z);
            out[e] = conv_act<IO, SILU>(z);
        }
        store_some<IO, VEC>(y + l, out, left);
    }
}

// dx of the steps of a packed axis before the first sequence and behind the last: zeros
template <class IO> __device__ __forceinline__ void conv_outside(const ConvParams &p, int64_t first, int64_t stride) {
    if (!p.cu) return;
    const int64_t before = delta_clamp(p.cu[0], p.L), from = delta_clamp(p.cu[p.seqs], p.L), n = before + (p.L - from);
    for (int64_t i = first; i < n * p.D; i += stride) {
        const int64_t d = i / n, t = i - d * n;
        reinterpret_cast<IO *>(p.dx)[d * p.y_d + (t < before ? t : from + (t - before))] = IO(0);
    }
}

// Backward a row is walked from its end, so that the g that a piece needs of the W - 1 steps behind it are the next lane's, or what the first lane had the visit
// before; the inputs before it are the lane's before.  (8 x 1536 x 2048 in bfloat16: 35 us; with every piece forming the g behind it again 45, with pieces half as long 40: bound by
// instructions as much as by memory.)
template <class IO, int W, int VEC, bool SILU> __global__ __launch_bounds__(256, 3) void k_conv_time_bwd(const ConvParams p) {
    const int tid = threadIdx.x, side = 1 << p.shift, lane = tid & (side - 1), d0 = blockIdx.y * (256 >> p.shift) + (tid >> p.shift);
    if ((int)blockIdx.x >= p.blocks) {
        const int64_t first = ((int64_t)(blockIdx.x - p.blocks) * gridDim.y + blockIdx.y) * 256 + tid, stride = (int64_t)(gridDim.x - p.blocks) * gridDim.y * 256;
        if (p.dx0) conv_dx0<IO, W, SILU>(p, first, stride);
        conv_outside<IO>(p, first, stride);
        return;
    }
    const int d = d0 < p.D ? d0 : p.D - 1;                 // (lanes without a row go along)
    float dw[W + 1] = {}, w[W];
    const float bias = p.bias ? p.bias[d] : 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) w[j] = p.w[(int64_t)d * W + j];
    const int visit = VEC << p.shift;
    // slot after slot, and each from its last visit to its first; the next is on its way while a visit is worked on
    struct At {
        unsigned slot;
        int seq, b, first, len, rest;                      // first step of the visit, steps of the slot, steps to the end of the sequence (all from the slot's first step on)
        int64_t lo, t0;
        const IO *x, *dy;
    };
    struct Loads { Few<IO, VEC> x, dy; Few<IO, 4> before; };
    auto open = [&](unsigned slot, At &a) {                // the first slot from this one on that has steps; false if there is none
        for (; slot < (unsigned)p.tiles; slot += p.blocks) {
            const ConvSlot c = conv_slot(p, slot);
            const int64_t rest = c.len - c.t0;
            if (rest <= 0) continue;
            a.slot = slot;
            a.seq = c.seq; a.b = c.b; a.lo = c.lo; a.t0 = c.t0;
            a.rest = rest < 1 << 30 ? (int)rest : 1 << 30;
            a.len = a.rest < p.tile ? a.rest : p.tile;
            a.first = (a.len - 1) / visit * visit;
            a.x = reinterpret_cast<const IO *>(p.x) + a.b * p.x_b + d * p.x_d + (c.lo + c.t0);
            a.dy = reinterpret_cast<const IO *>(p.dy) + a.b * p.dy_b + d * p.dy_d + (c.lo + c.t0);
            return true;
        }
        return false;
    };
    auto fetch = [&](const At &a, Loads &v) {
        const int l = a.first + lane * VEC;
        if (l + VEC <= a.len) { v.x.load(a.x + l); v.dy.load(a.dy + l); }
        else { v.x.load_some(a.x + l, a.len - l); v.dy.load_some(a.dy + l, a.len - l); }         // (zeros behind the slot: no part of any sum)
        if (lane == 0 && a.t0 + l >= 4) v.before.load(a.x + l - 4);
    };
    At now, ahead;
    if (open(blockIdx.x, ahead)) {
        now = ahead;
        Loads in{}, in1{};
        float after[W - 1];                                // g of the steps behind the visit
        fetch(now, in);
        bool fresh = true, more = true;
        for (; more; now = ahead, in = in1) {
            if (ahead.first > 0) ahead.first -= visit;
            else more = open(ahead.slot + p.blocks, ahead);
            if (more) fetch(ahead, in1);
            const int first = now.first, l = first + lane * VEC;
            const int64_t t0 = now.lo + now.t0;            // on the axis
            IO *dx = reinterpret_cast<IO *>(p.dx) + now.b * p.y_b + d * p.y_d + t0;
            const ConvSpan own{now.lo, t0 + now.rest, now.seq, true};
            auto g_at = [&](int64_t t) { return t < own.hi ? load_io(now.dy + (t - t0)) * conv_dact<IO, SILU>(conv_pre<IO, W>(p, own, now.b, t, d)) : 0.0f; };
            if (fresh)
#pragma unroll
                for (int i = 0; i < W - 1; ++i) after[i] = now.len < now.rest ? g_at(t0 + now.len + i) : 0.0f;
            fresh = first == 0;
            float xs[VEC + W - 1], g[VEC + W - 1], out[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) xs[W - 1 + e] = in.x.get(e);
            if constexpr (VEC >= W - 1) {
#pragma unroll
                for (int i = 0; i < W - 1; ++i) {
                    const float before = dpp<DPP_WAVE_SHR1>(0.0f, xs[VEC + i]);
                    xs[i] = lane == 0 ? in.before.get(4 - (W - 1) + i) : before;
                }
            } else {
#pragma unroll
                for (int i = 0; i < W - 1; ++i) xs[i] = 0.0f;
            }
            if (VEC < W - 1 || now.t0 + first == 0) {      // (else the first lane starts at step 4 at least)
                if (VEC < W - 1 ? l < now.len : lane == 0)               // (the sequence's first piece)
#pragma unroll
                    for (int i = 0; i < W - 1; ++i) xs[i] = conv_input<IO, W>(p, own, now.b, t0 + l + i - (W - 1), d);
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
                for (int i = 0; i < W - 1; ++i) g[VEC + i] = l < now.len ? g_at(t0 + l + VEC + i) : 0.0f;
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float a = 0.0f;
#pragma unroll
                for (int j = 0; j < W; ++j) a = __builtin_fmaf(w[j], g[e + W - 1 - j], a);
                out[e] = a;
            }
            if (d0 >= p.D || l >= now.len) continue;
            if (p.dx_last && l + VEC > now.rest - (W - 1))               // what the last inputs' gradient brings
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int slot = l + e - (now.rest - (W - 1));
                    if (slot >= 0 && l + e < now.len) out[e] += load_io(reinterpret_cast<const IO *>(p.dx_last) + ((int64_t)now.seq * (W - 1) + slot) * p.D + d);
                }
            store_some<IO, VEC>(dx + l, out, now.len - l);
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
    const unsigned more = BWD ? (p.dx0 || p.cu ? conv_blocks((int64_t)p.seqs * p.D) : 0) : (p.x_last ? conv_blocks((int64_t)p.seqs * (W - 1) * p.D) : 0);
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
    if (p.L < V && !p.cu) return bwd ? time_of<IO, 1, SILU, true>(p, s) : time_of<IO, 1, SILU, false>(p, s);
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
    const int64_t along = p.time_last ? p.L : p.D, wide = p.io ? 8 : 4, narrow = p.time_last && p.cu ? 0 : wide;
    const int64_t each = along < narrow ? 1 : !backward ? wide : p.time_last ? 2 * wide : wide / 2;
    // (a packed time axis: lanes for a sequence of average length)
    const int64_t pieces = ((p.time_last && p.cu ? p.L / p.seqs + 1 : along) + each - 1) / each;
    p.shift = log2_up(pieces, 6);
    const int side = 256 >> p.shift;
    int64_t groups;                                        // workgroups of a tile
    if (p.time_last) {
        // a row's lanes take up to eight pieces each, where that leaves the chip its workgroups
        const int64_t visit = each << p.shift, waves = (int64_t)p.B * p.D * ((p.L + visit - 1) / visit + (p.cu ? p.seqs : 0)) / side * 4 / (backward ? 4096 : 8192);
        p.tile_log2 = log2_up(visit, 62) + (waves >= 8 ? 3 : waves >= 4 ? 2 : waves >= 2 ? 1 : 0);
        p.tile = 1 << p.tile_log2;
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
    p.tiles = p.time_last && p.cu ? p.L / p.tile + p.seqs : p.B * p.tiles_each;
    const int64_t blocks = p.time_last ? p.tiles : (p.tiles + side - 1) / side;
    // backward: parts of the weights' gradients.  768 workgroups are all that fit at once ([B,L,D], 4 x 4096 x 6144 in bfloat16, in a loop of its own, 144 us; 1536 153, 3840 174); the sequences of a packed time
    // axis are of all lengths, and more even each other out (24 sequences of 16384 steps, 2048 channels: 768 159 us, 1536 110, 2304 94, 3840 119; 400: 166, 141, 139, 157)
    int64_t most = (p.time_last && p.cu ? 2304 : 768) / groups;
    if (most < 1) most = 1;
    p.blocks = (int)(backward && blocks > most ? most : blocks);
}

}  // namespace lrnnx
