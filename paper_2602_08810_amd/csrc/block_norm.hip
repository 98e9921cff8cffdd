// Norms around a block, with its gate and the scale of its residual:
//     n = x / rms(x), group by group;   m = post_weight n act(gate);   h = residual + res_scale m;   y = pre_weight h / rms(h)
// every part but x optional.  A row stays in the registers of a workgroup from the first load to the last store: one read of every input, one
// write of every output, which is what bounds it.  Sums of squares are taken in float32 over lanes and wavefronts.
// Backward, with everything of the forward pass formed again from its inputs (which the gradients need anyway; nothing is saved):
//     dn2 = dy pre_weight;  dh += (dn2 - n2 mean(dn2 n2)) / rms(h);   dresidual = dh;   dp = dh res_scale;   dgate = dp n post_weight act'(gate)
//     dn1 = dp act(gate) post_weight;   dx = (dn1 - n mean(dn1 n)) / rms(x)
// (of a norm over one element the difference is dn eps / (x^2 + eps), which is formed so: as a difference nothing of it would be left)
// and over all rows dpre_weight = sum dy n2, dres_scale = sum dh m, dpost_weight = sum dp act(gate) n: a workgroup adds up the rows it takes in
// registers and leaves them in the workspace, a second launch adds up the workgroups in a fixed order.
#include "block_norm.hpp"
#include "delta_common.hpp"

namespace lrnnx {

template <class T, int VEC> struct Piece;        // VEC neighbouring elements as one access
template <> struct Piece<float, 4> {
    static __device__ __forceinline__ void load(const float *p, float (&x)[4]) { const f32x4 v = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = v[e]; }
    static __device__ __forceinline__ void store(float *p, const float (&x)[4]) { *reinterpret_cast<f32x4 *>(p) = f32x4{x[0], x[1], x[2], x[3]}; }
};
template <> struct Piece<uint16_t, 4> {
    static __device__ __forceinline__ void load(const uint16_t *p, float (&x)[4]) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        x[0] = __uint_as_float(v.x << 16); x[1] = hi_part(__uint_as_float(v.x)); x[2] = __uint_as_float(v.y << 16); x[3] = hi_part(__uint_as_float(v.y));
    }
    static __device__ __forceinline__ void store(uint16_t *p, const float (&x)[4]) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack_rne(x[0], x[1]), pack_rne(x[2], x[3]));
    }
};
template <class T> struct Piece<T, 8> {
    static __device__ __forceinline__ void load(const T *p, float (&x)[8]) {
        if constexpr (sizeof(T) == 2) {
            const uint4 v = *reinterpret_cast<const uint4 *>(p);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(w[e] << 16); x[2 * e + 1] = hi_part(__uint_as_float(w[e])); }
        } else {
            float a[4], b[4];
            Piece<float, 4>::load(p, a); Piece<float, 4>::load(p + 4, b);
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
        }
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[8]) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4 *>(p) = make_uint4(pack_rne(x[0], x[1]), pack_rne(x[2], x[3]), pack_rne(x[4], x[5]), pack_rne(x[6], x[7]));
        } else {
            Piece<float, 4>::store(p, {x[0], x[1], x[2], x[3]});
            Piece<float, 4>::store(p + 4, {x[4], x[5], x[6], x[7]});
        }
    }
};
template <class T> struct Piece<T, 1> {
    static __device__ __forceinline__ void load(const T *p, float (&x)[1]) { x[0] = load_io(p); }
    static __device__ __forceinline__ void store(T *p, const float (&x)[1]) { store_io(p, x[0]); }
};

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) x += __shfl_xor(x, m, 64);
    return x;
}
// Sum over the workgroup; `part`: a float of LDS per wavefront, free again after the next barrier.
__device__ __forceinline__ float block_sum(float x, float *part) {
    x = wave_sum(x);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return x;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < waves; ++w) s += part[w];
    __syncthreads();
    return s;
}

// How the sum over a group is taken: over the workgroup (one group), over `lanes` neighbouring lanes (a power of two), or through LDS.
enum : int { GROUP_ROW = 0, GROUP_LANES = 1, GROUP_LDS = 2 };

// Sums over each thread's groups of `x[i]` (piece i of the row lies in one group), into x.
template <int NV> __device__ __forceinline__ void group_sums(float (&x)[NV], int how, int pieces, int per_group, float *lds) {
    if (how == GROUP_ROW) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) s += x[i];
        s = block_sum(s, lds);
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = s;
    } else if (how == GROUP_LANES) {
        for (int m = 1; m < per_group; m <<= 1)
#pragma unroll
            for (int i = 0; i < NV; ++i) x[i] += __shfl_xor(x[i], m, 64);
    } else {
        const int nt = blockDim.x, groups = pieces / per_group;
#pragma unroll
        for (int i = 0; i < NV; ++i) { const int v = threadIdx.x + i * nt; if (v < pieces) lds[v] = x[i]; }
        __syncthreads();
        float *out = lds + pieces;
        for (int g = threadIdx.x; g < groups; g += nt) {
            float s = 0.0f;
            for (int j = 0; j < per_group; ++j) s += lds[g * per_group + j];
            out[g] = s;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i) { const int v = threadIdx.x + i * nt; x[i] = v < pieces ? out[v / per_group] : 0.0f; }
        __syncthreads();
    }
}

template <bool FINE> __device__ __forceinline__ void gate_of(float z, int act, float &a, float &da) {
    const float s = 1.0f / (1.0f + (FINE ? expf(-z) : __expf(-z)));
    if (act) { a = s; da = s * (1.0f - s); }
    else { a = z * s; da = s * (1.0f + z * (1.0f - s)); }
}

template <class IO, class RES, int VEC, int NV, bool BWD> __global__ __launch_bounds__(512) void k_block_norm(const NormParams p, int how) {
    extern __shared__ float lds[];
    const int nt = blockDim.x, pieces = p.D / VEC, per_group = p.width / VEC;
    float *part = lds;
    float w1[BWD ? NV : 1][VEC] = {}, w2[BWD ? NV : 1][VEC] = {}, w3[BWD ? NV : 1][VEC] = {};
    const float by_width = 1.0f / (float)p.width, by_D = 1.0f / (float)p.D;
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x) {
        float x[NV][VEC], z[NV][VEC], r[NV][VEC], act[NV][VEC], r1[NV];
        float dh[BWD ? NV : 1][VEC], dy[BWD ? NV : 1][VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = threadIdx.x + i * nt;
            const bool in = v < pieces;
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[i][e] = z[i][e] = r[i][e] = 0.0f;
            if (BWD)
#pragma unroll
                for (int e = 0; e < VEC; ++e) dh[i][e] = dy[i][e] = 0.0f;
            if (in) {
                const int64_t c = (int64_t)v * VEC;
                Piece<IO, VEC>::load(reinterpret_cast<const IO *>(p.x) + row * p.x_s + c, x[i]);
                if (p.gate) Piece<IO, VEC>::load(reinterpret_cast<const IO *>(p.gate) + row * p.gate_s + c, z[i]);
                if (p.res) Piece<RES, VEC>::load(reinterpret_cast<const RES *>(p.res) + row * p.res_s + c, r[i]);
                if constexpr (BWD) {
                    if (p.dh) Piece<RES, VEC>::load(reinterpret_cast<const RES *>(p.dh) + row * p.dh_s + c, dh[i]);
                    if (p.dy) Piece<IO, VEC>::load(reinterpret_cast<const IO *>(p.dy) + row * p.dy_s + c, dy[i]);
                }
            }
        }
        // n (in x), and h
        if (p.post) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                r1[i] = 0.0f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) r1[i] = __builtin_fmaf(x[i][e], x[i][e], r1[i]);
            }
            group_sums<NV>(r1, how, pieces, per_group, part);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                r1[i] = 1.0f / sqrtf(__builtin_fmaf(r1[i], by_width, p.eps));
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[i][e] *= r1[i];
            }
        }
        float h[NV][VEC], ss = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = threadIdx.x + i * nt, c = v * VEC;
            if (v < pieces) {
                const int cp = p.post_shared ? c % p.width : c;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float m = p.post ? p.post[cp + e] * x[i][e] : x[i][e];
                    if (p.gate) { float da; gate_of<sizeof(IO) == 4>(z[i][e], p.gate_act, act[i][e], da); m *= act[i][e]; if (BWD) z[i][e] = da; }
                    if (p.scale) m *= p.scale[c + e];
                    h[i][e] = r[i][e] + m;
                    ss = __builtin_fmaf(h[i][e], h[i][e], ss);
                }
            }
        }
        float r2 = 0.0f;
        if (p.pre) r2 = 1.0f / sqrtf(__builtin_fmaf(block_sum(ss, part), by_D, p.eps));
        if constexpr (!BWD) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int v = threadIdx.x + i * nt, c = v * VEC;
                if (v < pieces) {
                    Piece<RES, VEC>::store(reinterpret_cast<RES *>(p.h) + row * p.D + c, h[i]);
                    if (p.pre) {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) h[i][e] *= r2 * p.pre[c + e];
                        Piece<IO, VEC>::store(reinterpret_cast<IO *>(p.y) + row * p.D + c, h[i]);
                    }
                }
            }
        } else {
            if (p.pre) {
                float dot = 0.0f;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int v = threadIdx.x + i * nt, c = v * VEC;
                    if (v < pieces)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            h[i][e] *= r2;                                       // n2
                            w3[i][e] = __builtin_fmaf(dy[i][e], h[i][e], w3[i][e]);
                            dy[i][e] *= p.pre[c + e];
                            dot = __builtin_fmaf(dy[i][e], h[i][e], dot);
                        }
                }
                dot = block_sum(dot, part) * by_D;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (threadIdx.x + i * nt < pieces)
#pragma unroll
                        for (int e = 0; e < VEC; ++e)
                            dh[i][e] = __builtin_fmaf(r2, p.D == 1 ? dy[i][e] * p.eps * r2 * r2 : __builtin_fmaf(-h[i][e], dot, dy[i][e]), dh[i][e]);
            }
            float dots[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int v = threadIdx.x + i * nt, c = v * VEC;
                dots[i] = 0.0f;
                if (v < pieces) {
                    if (p.dres) Piece<RES, VEC>::store(reinterpret_cast<RES *>(p.dres) + row * p.D + c, dh[i]);
                    const int cp = p.post_shared ? c % p.width : c;
                    float dz[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float w = p.post ? p.post[cp + e] : 1.0f, m = w * x[i][e], a = p.gate ? act[i][e] : 1.0f;
                        float dp = dh[i][e];
                        if (p.scale) { w2[i][e] = __builtin_fmaf(dp, m * a, w2[i][e]); dp *= p.scale[c + e]; }
                        dz[e] = p.gate ? dp * m * z[i][e] : 0.0f;
                        dp *= a;
                        if (p.post) w1[i][e] = __builtin_fmaf(dp, x[i][e], w1[i][e]);
                        dh[i][e] = dp * w;
                        dots[i] = __builtin_fmaf(dh[i][e], x[i][e], dots[i]);
                    }
                    if (p.dgate) Piece<IO, VEC>::store(reinterpret_cast<IO *>(p.dgate) + row * p.D + c, dz);
                }
            }
            if (p.post) group_sums<NV>(dots, how, pieces, per_group, part);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int v = threadIdx.x + i * nt, c = v * VEC;
                if (v < pieces) {
                    if (p.post)
#pragma unroll
                        for (int e = 0; e < VEC; ++e)
                            dh[i][e] = r1[i] * (p.width == 1 ? dh[i][e] * p.eps * r1[i] * r1[i] : __builtin_fmaf(-x[i][e], dots[i] * by_width, dh[i][e]));
                    Piece<IO, VEC>::store(reinterpret_cast<IO *>(p.dx) + row * p.D + c, dh[i]);
                }
            }
        }
    }
    if constexpr (BWD) {
        float *to = p.sums + (int64_t)blockIdx.x * 3 * p.D;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = threadIdx.x + i * nt, c = v * VEC;
            if (v < pieces) {
                if (p.dpost) Piece<float, VEC>::store(to + c, w1[i]);
                if (p.dscale) Piece<float, VEC>::store(to + p.D + c, w2[i]);
                if (p.dpre) Piece<float, VEC>::store(to + 2 * (int64_t)p.D + c, w3[i]);
            }
        }
    }
}

// Sums over workgroups (and over groups, of a shared weight): 16 columns by 16 parts of the workgroups, in a fixed order.
__global__ __launch_bounds__(256) void k_norm_sums(const NormParams p) {
    __shared__ float part[16][17];
    const int which = blockIdx.y, cl = threadIdx.x & 15, q = threadIdx.x >> 4, c = blockIdx.x * 16 + cl;
    float *to = which == 0 ? p.dpost : which == 1 ? p.dscale : p.dpre;
    if (!to) return;
    const bool shared = which == 0 && p.post_shared;
    const int n = shared ? p.width : p.D, reps = shared ? p.groups : 1;
    float s = 0.0f;
    if (c < n)
        for (int b = q; b < p.blocks; b += 16)
            for (int g = 0; g < reps; ++g) s += p.sums[((int64_t)b * 3 + which) * p.D + (int64_t)g * n + c];
    part[q][cl] = s;
    __syncthreads();
    if (q == 0 && c < n) {
        for (int i = 1; i < 16; ++i) s += part[i][cl];
        to[c] = s;
    }
}

// Shape of a launch: pieces of 16 bytes of the narrowest tensor where every row allows it, threads so that a thread has few pieces.
struct NormShape { int vec, nt, nv, how; size_t lds; };
static bool norm_rows_fit(const NormParams &p, int vec) {
    const int es = p.io ? 2 : 4, rs = p.res_io ? 2 : 4;
    auto fits = [&](const void *q, int64_t stride, int size) {
        return !q || (((reinterpret_cast<uintptr_t>(q) | (uintptr_t)(stride * size)) & (uintptr_t)(vec * size < 16 ? vec * size - 1 : 15)) == 0);
    };
    return p.D % vec == 0 && p.width % vec == 0 && fits(p.x, p.x_s, es) && fits(p.gate, p.gate_s, es) && fits(p.res, p.res_s, rs) &&
           fits(p.dh, p.dh_s, rs) && fits(p.dy, p.dy_s, es) && fits(p.h, p.D, rs) && fits(p.y, p.D, es) && fits(p.dx, p.D, es) &&
           fits(p.dgate, p.D, es) && fits(p.dres, p.D, rs) && fits(p.sums, p.D, 4);
}
static NormShape norm_shape(const NormParams &p) {
    NormShape s;
    s.vec = norm_rows_fit(p, 8) ? 8 : norm_rows_fit(p, 4) ? 4 : 1;
    const int pieces = p.D / s.vec, per_group = p.width / s.vec;
    const int most = 16 / s.vec;                     // pieces a thread: 16 elements of every tensor in its registers
    s.nt = 64;
    while (s.nt < 512 && s.nt * most < pieces) s.nt *= 2;
    const int need = (pieces + s.nt - 1) / s.nt;
    s.nv = 1;
    while (s.nv < need) s.nv *= 2;
    const bool pow2 = (per_group & (per_group - 1)) == 0;
    s.how = p.groups == 1 ? GROUP_ROW : pow2 && per_group <= 64 ? GROUP_LANES : GROUP_LDS;
    s.lds = s.how == GROUP_LDS && p.post ? sizeof(float) * (size_t)(pieces + p.groups) : 0;
    if (s.lds < 16 * sizeof(float)) s.lds = 16 * sizeof(float);
    return s;
}
template <class IO, class RES, int VEC, bool BWD> static hipError_t launch_norm_nv(const NormParams &p, const NormShape &s, unsigned blocks, hipStream_t st) {
    switch (s.nv) {
        case 1: hipLaunchKernelGGL((k_block_norm<IO, RES, VEC, 1, BWD>), dim3(blocks), dim3(s.nt), s.lds, st, p, s.how); break;
        case 2: hipLaunchKernelGGL((k_block_norm<IO, RES, VEC, 2, BWD>), dim3(blocks), dim3(s.nt), s.lds, st, p, s.how); break;
        case 4: if constexpr (VEC <= 4) { hipLaunchKernelGGL((k_block_norm<IO, RES, VEC, 4, BWD>), dim3(blocks), dim3(s.nt), s.lds, st, p, s.how); break; }
        case 8: if constexpr (VEC == 1) { hipLaunchKernelGGL((k_block_norm<IO, RES, VEC, 8, BWD>), dim3(blocks), dim3(s.nt), s.lds, st, p, s.how); break; }
        case 16: if constexpr (VEC == 1) { hipLaunchKernelGGL((k_block_norm<IO, RES, VEC, 16, BWD>), dim3(blocks), dim3(s.nt), s.lds, st, p, s.how); break; }
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}
template <class IO, class RES, bool BWD> static hipError_t launch_norm_vec(const NormParams &p, unsigned blocks, hipStream_t st) {
    const NormShape s = norm_shape(p);
    if (s.vec == 8) return launch_norm_nv<IO, RES, 8, BWD>(p, s, blocks, st);
    if (s.vec == 4) return launch_norm_nv<IO, RES, 4, BWD>(p, s, blocks, st);
    return launch_norm_nv<IO, RES, 1, BWD>(p, s, blocks, st);
}
template <bool BWD> static hipError_t launch_norm(const NormParams &p, unsigned blocks, hipStream_t st) {
    if (p.io) return p.res_io ? launch_norm_vec<uint16_t, uint16_t, BWD>(p, blocks, st) : launch_norm_vec<uint16_t, float, BWD>(p, blocks, st);
    return launch_norm_vec<float, float, BWD>(p, blocks, st);
}
hipError_t launch_norm_fwd(const NormParams &p, hipStream_t s) { return launch_norm<false>(p, (unsigned)(p.M < 65536 ? p.M : 65536), s); }

int norm_bwd_blocks(int64_t M, int) { return (int)(M < 1024 ? M : 1024); }
hipError_t launch_norm_bwd(const NormParams &p, hipStream_t s) {
    hipError_t e = launch_norm<true>(p, (unsigned)p.blocks, s);
    if (e != hipSuccess || (!p.dpost && !p.dscale && !p.dpre)) return e;
    hipLaunchKernelGGL(k_norm_sums, dim3((unsigned)((p.D + 15) / 16), 3), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace lrnnx
