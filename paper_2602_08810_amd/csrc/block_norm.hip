// Norms around a block, with its gate and the scale of its residual:
//     n = x / rms(x), group by group;   m = post_weight n act(gate);   h = residual + res_scale m;   y = pre_weight h / rms(h)
// every part but x optional.  A row stays in the registers of a workgroup from the first load to the last store: one read of every input, one
// write of every output, which is what bounds it.  Sums of squares are taken in float32 over lanes and wavefronts; roots are taken to 1 ulp, of subnormal means too.
// Lanes past the end of the row bring zeros into its sums: their groups' sum is taken as 1 (with eps = 0 their norm would be 0 / 0), their weights are
// zeros behind the row's own in LDS.
// Backward, with everything of the forward pass formed again from its inputs (which the gradients need anyway; nothing is saved):
//     dn2 = dy pre_weight;  dh += (dn2 - n2 mean(dn2 n2)) / rms(h);   dresidual = dh;   dp = dh res_scale;   dgate = dp n post_weight act'(gate)
//     dn1 = dp act(gate) post_weight;   dx = (dn1 - n mean(dn1 n)) / rms(x)
// (of a norm over one element the difference is dn eps / (x^2 + eps), which is formed so: as a difference nothing of it would be left)
// and over all rows dpre_weight = sum dy n2, dres_scale = sum dh m, dpost_weight = sum dp act(gate) n: a workgroup adds up the rows it takes in
// registers and leaves them in the workspace, a second launch adds up the workgroups in a fixed order.
// 16384 rows of 2560, bfloat16 with the residual stream in float32: forward 503 MB in 85 us (5.9 TB/s), backward 755 MB in 172 (4.4) and 7 of sums; gated
// heads, 16 of 128: 201 MB in 43 (4.7) and 335 in 74 (4.5) and 6; a copy of these sizes does 5.3 TB/s.  Few rows: latency, 5.0 us for 16.
#include "block_norm.hpp"
#include "delta_common.hpp"

namespace lrnnx {

// VEC neighbouring elements as one access, as they lie in memory (so that a row can be on its way while the one before is worked on) and in float32
template <class T, int VEC> struct Piece {
    static constexpr int W = VEC * (int)sizeof(T) / 4;            // words
    uint32_t w[W > 0 ? W : 1];
    __device__ __forceinline__ void load(Buffer b, uint32_t off) {
        if constexpr (W == 0) w[0] = __builtin_amdgcn_raw_buffer_load_b16(b, off, 0, 0);
        else if constexpr (W == 1) w[0] = __builtin_amdgcn_raw_buffer_load_b32(b, off, 0, 0);
        else if constexpr (W == 2) { const uint2 v = buffer_load8(b, off); w[0] = v.x; w[1] = v.y; }
        else
#pragma unroll
            for (int i = 0; i < W; i += 4) {
                const uint4 v = buffer_load16(b, off + 4 * i);
                w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
            }
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[VEC]) {
        if constexpr (VEC == 1) store_io(p, x[0]);
        else if constexpr (sizeof(T) == 4)
#pragma unroll
            for (int i = 0; i < VEC; i += 4) *reinterpret_cast<f32x4 *>(p + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
        else if constexpr (VEC == 4) *reinterpret_cast<uint2 *>(p) = make_uint2(pack_rne(x[0], x[1]), pack_rne(x[2], x[3]));
        else *reinterpret_cast<uint4 *>(p) = make_uint4(pack_rne(x[0], x[1]), pack_rne(x[2], x[3]), pack_rne(x[4], x[5]), pack_rne(x[6], x[7]));
    }
};

// Sum over the wavefront, the same number in every lane: moves within rows of 16 lanes and from row to row, no LDS.
__device__ __forceinline__ float wave_sum(float x) {
    x += dpp<0x111>(0.0f, x);                     // from 1, 2, 4, 8 lanes below within a row
    x += dpp<0x112>(0.0f, x);
    x += dpp<0x114>(0.0f, x);
    x += dpp<0x118>(0.0f, x);
    x += dpp<0x142, 0xA>(0.0f, x);                // the last lane of a row to the next, into rows 1 and 3
    x += dpp<0x143, 0xC>(0.0f, x);                // and of the lower half to the upper
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 63));
}
// Sum over the workgroup.  `part`: a float of LDS for each of eight wavefronts, taken in turn from a set (`Sums`) that is large enough for a
// slot not to be written again before a barrier has passed since it was read: one barrier a sum.  Wavefronts that are not there have left zeros.
__device__ __forceinline__ float block_sum(float x, float *part) {
    x = wave_sum(x);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return x;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    lds_barrier();
    const f32x4 a = *reinterpret_cast<const f32x4 *>(part), b = *reinterpret_cast<const f32x4 *>(part + 4);
    return ((a[0] + a[1]) + (a[2] + a[3])) + ((b[0] + b[1]) + (b[2] + b[3]));
}
constexpr int kSumSlots = 8;                      // four sums a row, two rows
// Floats of LDS for a weight of n elements, whole pieces of it and a piece of zeros.
__host__ __device__ constexpr int weight_room(int n) { return ((n + 3) & ~3) + 8; }

// How the sum over a group is taken: over the workgroup (one group), over `lanes` neighbouring lanes (a power of two), or through LDS.
enum : int { GROUP_ROW = 0, GROUP_LANES = 1, GROUP_LDS = 2 };

// Sums over each thread's groups of `x[i]` (piece i of the row lies in one group, `of[i]`), into x (1 past the end of the row).  Through LDS a power of two of neighbouring lanes
// takes a group, as many as the workgroup has for it (2442 rows of 32 groups of 49, gated, bfloat16: 30 us forward and 69 backward with a lane a group, 24 and 48 so).
template <int NV> __device__ __forceinline__ void group_sums(float (&x)[NV], const int (&of)[NV], int how, int pieces, int per_group, float *lds, float *part) {
    if (how == GROUP_ROW) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) s += x[i];
        s = block_sum(s, part);
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = s;
    } else if (how == GROUP_LANES) {
        for (int m = 1; m < per_group; m <<= 1)
#pragma unroll
            for (int i = 0; i < NV; ++i) x[i] += __shfl_xor(x[i], m, 64);
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = (int)(threadIdx.x + i * blockDim.x) < pieces ? x[i] : 1.0f;
    } else {
        const int nt = blockDim.x, groups = pieces / per_group;
#pragma unroll
        for (int i = 0; i < NV; ++i) { const int v = threadIdx.x + i * nt; if (v < pieces) lds[v] = x[i]; }
        lds_barrier();
        float *out = lds + pieces;
        const int room = nt / groups, lanes = room >= 64 ? 64 : room > 1 ? 1 << (31 - __builtin_clz(room)) : 1;
        const int at = threadIdx.x & (lanes - 1), g0 = threadIdx.x / lanes;                   // (a power of two: a shift)
        for (int first = 0; first < groups; first += nt / lanes) {
            const int g = first + g0;
            float s = 0.0f;
            if (g < groups)
                for (int j = at; j < per_group; j += lanes) s += lds[g * per_group + j];
            if (lanes == 64) s = wave_sum(s);
            else
                for (int m = 1; m < lanes; m <<= 1) s += __shfl_xor(s, m, 64);
            if (at == 0 && g < groups) out[g] = s;
        }
        lds_barrier();
#pragma unroll
        for (int i = 0; i < NV; ++i) { const int v = threadIdx.x + i * nt; x[i] = v < pieces ? out[of[i]] : 1.0f; }
        lds_barrier();
    }
}

// (the reciprocal is the hardware's, 1 ulp)
template <bool FINE> __device__ __forceinline__ void gate_of(float z, int act, float &a, float &da) {
    const float s = __builtin_amdgcn_rcpf(1.0f + (FINE ? expf(-z) : __expf(-z)));
    if (act) { a = s; da = s * (1.0f - s); }
    else { a = z * s; da = s * (1.0f + z * (1.0f - s)); }
}

// The row that a workgroup takes next, on its way from memory while it works on this one.  All loads go through buffer descriptors: what is past the
// row, past the last row or not given at all reads as zero, with no branch in which the loads would have to be waited for.
template <class IO, class RES, int VEC, int NV, bool BWD> struct NormRow {
    Piece<IO, VEC> x[NV], z[NV], dy[BWD ? NV : 1];
    Piece<RES, VEC> r[NV], dh[BWD ? NV : 1];
    template <class T> static __device__ __forceinline__ Buffer row_of(const NormParams &p, const void *base, int64_t stride, int64_t row) {
        return buffer_of(reinterpret_cast<const T *>(base) + row * stride, base && row < p.M ? p.D * (int)sizeof(T) : 0);
    }
    __device__ __forceinline__ void load(const NormParams &p, int64_t row) {
        const Buffer bx = row_of<IO>(p, p.x, p.x_s, row), bz = row_of<IO>(p, p.gate, p.gate_s, row), br = row_of<RES>(p, p.res, p.res_s, row);
        const Buffer bh = row_of<RES>(p, p.dh, p.dh_s, row), by = row_of<IO>(p, p.dy, p.dy_s, row);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t c = (threadIdx.x + i * blockDim.x) * VEC;
            x[i].load(bx, c * sizeof(IO));
            z[i].load(bz, c * sizeof(IO));
            r[i].load(br, c * sizeof(RES));
            if constexpr (BWD) { dh[i].load(bh, c * sizeof(RES)); dy[i].load(by, c * sizeof(IO)); }
        }
    }
};

template <class IO, class RES, int VEC, int NV, bool BWD> __global__ __launch_bounds__(512) void k_block_norm(const NormParams p, int how) {
    extern __shared__ __align__(16) float lds[];
    const int nt = blockDim.x, pieces = p.D / VEC, per_group = p.width / VEC;
    // LDS: slots of sums, the weights (a wait for them from memory would be a wait for the next row too), sums of groups
    const int n_post = p.post_shared ? p.width : p.D;
    float *const w_post = lds + kSumSlots * 8, *const w_scale = w_post + (p.post ? weight_room(n_post) : 0);
    float *const w_pre = w_scale + (p.scale ? weight_room(p.D) : 0), *const wide = w_pre + (p.pre ? weight_room(p.D) : 0);
    int turn = 0;
    auto slot = [&]() { turn = (turn + 1) % kSumSlots; return lds + turn * 8; };
    float w1[BWD ? NV : 1][VEC] = {}, w2[BWD ? NV : 1][VEC] = {}, w3[BWD ? NV : 1][VEC] = {};
    const float by_width = 1.0f / (float)p.width, by_D = 1.0f / (float)p.D;
    int of[NV], cp[NV];                                   // where a piece's part of post_weight starts
#pragma unroll
    for (int i = 0; i < NV; ++i) { const int c = (threadIdx.x + i * nt) * VEC; of[i] = how == GROUP_LDS ? c / p.width : 0; cp[i] = c >= p.D ? n_post : p.post_shared ? c % p.width : c; }
    struct Weight { float w[VEC]; __device__ __forceinline__ float get(int e) const { return w[e]; } };
    auto weight = [&](const float *w, int c) {
        Weight r;
        if (c >= p.D) c = p.D;
        if constexpr (VEC == 1) r.w[0] = w[c];
        else
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
                const f32x4 v = *reinterpret_cast<const f32x4 *>(w + c + e);
#pragma unroll
                for (int f = 0; f < 4; ++f) r.w[e + f] = v[f];
            }
        return r;
    };
    using Row = NormRow<IO, RES, VEC, NV, BWD>;
    Row even, odd;
    int64_t row = blockIdx.x;
    even.load(p, row);
    if (threadIdx.x < kSumSlots * 8) lds[threadIdx.x] = 0.0f;
    if (threadIdx.x < VEC) {
        if (p.post) w_post[n_post + threadIdx.x] = 0.0f;
        if (p.scale) w_scale[p.D + threadIdx.x] = 0.0f;
        if (p.pre) w_pre[p.D + threadIdx.x] = 0.0f;
    }
    {
        const Buffer bp = buffer_of(p.post, p.post ? n_post * 4 : 0), bs = buffer_of(p.scale, p.scale ? p.D * 4 : 0),
                     br = buffer_of(p.pre, p.pre ? p.D * 4 : 0);
        Piece<float, VEC> a[NV], b[NV], c[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t off = (threadIdx.x + i * nt) * VEC * 4;
            a[i].load(bp, off); b[i].load(bs, off); c[i].load(br, off);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (threadIdx.x + i * nt) * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if (p.post && at < n_post) w_post[at + e] = a[i].get(e);
                if (p.scale && at < p.D) w_scale[at + e] = b[i].get(e);
                if (p.pre && at < p.D) w_pre[at + e] = c[i].get(e);
            }
        }
    }
    lds_barrier();
    auto take = [&](const Row &in) __attribute__((always_inline)) {
        float x[NV][VEC], r1[NV], h[NV][VEC], ss = 0.0f;
        float act[BWD ? NV : 1][VEC], dact[BWD ? NV : 1][VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[i][e] = in.x[i].get(e);
        if (p.post) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                r1[i] = 0.0f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) r1[i] = __builtin_fmaf(x[i][e], x[i][e], r1[i]);
            }
            group_sums<NV>(r1, of, how, pieces, per_group, wide, slot());
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                r1[i] = rsqrtf(__builtin_fmaf(r1[i], by_width, p.eps));
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[i][e] *= r1[i];                  // n
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (threadIdx.x + i * nt) * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e) h[i][e] = x[i][e];
            if (p.post) {
                const auto w = weight(w_post, cp[i]);
#pragma unroll
                for (int e = 0; e < VEC; ++e) h[i][e] *= w.get(e);
            }
            if (p.gate)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float a, da;
                    gate_of<sizeof(IO) == 4>(in.z[i].get(e), p.gate_act, a, da);
                    h[i][e] *= a;
                    if constexpr (BWD) { act[i][e] = a; dact[i][e] = da; }
                }
            else if constexpr (BWD)
#pragma unroll
                for (int e = 0; e < VEC; ++e) { act[i][e] = 1.0f; dact[i][e] = 0.0f; }
            if (p.scale) {
                const auto w = weight(w_scale, c);
#pragma unroll
                for (int e = 0; e < VEC; ++e) h[i][e] *= w.get(e);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) { h[i][e] += in.r[i].get(e); ss = __builtin_fmaf(h[i][e], h[i][e], ss); }
        }
        float r2 = 0.0f;
        if (p.pre) r2 = rsqrtf(__builtin_fmaf(block_sum(ss, slot()), by_D, p.eps));
        if constexpr (!BWD) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (threadIdx.x + i * nt) * VEC;
                if (c < p.D) {
                    Piece<RES, VEC>::store(reinterpret_cast<RES *>(p.h) + row * p.D + c, h[i]);
                    if (p.pre) {
                        const auto w = weight(w_pre, c);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) h[i][e] *= r2 * w.get(e);
                        Piece<IO, VEC>::store(reinterpret_cast<IO *>(p.y) + row * p.D + c, h[i]);
                    }
                }
            }
        } else {
            float g[NV][VEC];                         // the gradient on its way down: of y, h, m, n
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) g[i][e] = in.dh[i].get(e);
            if (p.pre) {
                float dot = 0.0f;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const auto w = weight(w_pre, (threadIdx.x + i * nt) * VEC);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float d = in.dy[i].get(e);
                        h[i][e] *= r2;                                           // n2
                        w3[i][e] = __builtin_fmaf(d, h[i][e], w3[i][e]);
                        dot = __builtin_fmaf(d * w.get(e), h[i][e], dot);
                    }
                }
                dot = block_sum(dot, slot()) * by_D;
                const float cd = p.D == 1 ? p.eps * r2 * r2 * r2 : r2, ch = p.D == 1 ? 0.0f : r2 * dot;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const auto w = weight(w_pre, (threadIdx.x + i * nt) * VEC);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        g[i][e] = __builtin_fmaf(cd * w.get(e), in.dy[i].get(e), __builtin_fmaf(-ch, h[i][e], g[i][e]));
                    }
                }
            }
            float dots[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (threadIdx.x + i * nt) * VEC;
                dots[i] = 0.0f;
                if (c < p.D) {
                    if (p.dres) Piece<RES, VEC>::store(reinterpret_cast<RES *>(p.dres) + row * p.D + c, g[i]);
                    Weight wp, ws;
                    if (p.post) wp = weight(w_post, cp[i]);
                    if (p.scale) ws = weight(w_scale, c);
                    float dz[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float w = p.post ? wp.get(e) : 1.0f, m = w * x[i][e];
                        const float a = act[i][e];
                        float dp = g[i][e];
                        if (p.scale) { w2[i][e] = __builtin_fmaf(dp, m * a, w2[i][e]); dp *= ws.get(e); }
                        dz[e] = dp * m * dact[i][e];
                        dp *= a;
                        if (p.post) w1[i][e] = __builtin_fmaf(dp, x[i][e], w1[i][e]);
                        g[i][e] = dp * w;
                        dots[i] = __builtin_fmaf(g[i][e], x[i][e], dots[i]);
                    }
                    if (p.dgate) Piece<IO, VEC>::store(reinterpret_cast<IO *>(p.dgate) + row * p.D + c, dz);
                }
            }
            if (p.post) group_sums<NV>(dots, of, how, pieces, per_group, wide, slot());
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (threadIdx.x + i * nt) * VEC;
                if (c < p.D) {
                    if (p.post) {
                        const float cg = p.width == 1 ? p.eps * r1[i] * r1[i] * r1[i] : r1[i], cx = p.width == 1 ? 0.0f : r1[i] * dots[i] * by_width;
#pragma unroll
                        for (int e = 0; e < VEC; ++e) g[i][e] = __builtin_fmaf(cg, g[i][e], -cx * x[i][e]);
                    }
                    Piece<IO, VEC>::store(reinterpret_cast<IO *>(p.dx) + row * p.D + c, g[i]);
                }
            }
        }
    };
    if constexpr (VEC == 1 && NV > 8) {           // no registers for a second row (4000 rows of 5001, bfloat16: backward 330 us with one, 178 without)
        for (; row < p.M; row += gridDim.x) {
            take(even);
            even.load(p, row + gridDim.x);
        }
    } else
        while (row < p.M) {                       // two rows a round: the next row's registers are never copied, which would wait for them
            odd.load(p, row + gridDim.x);
            take(even);
            row += gridDim.x;
            if (row >= p.M) break;
            even.load(p, row + gridDim.x);
            take(odd);
            row += gridDim.x;
        }
    if constexpr (BWD) {
        float *to = p.sums + (int64_t)blockIdx.x * 3 * p.D;
        if (p.dpost && p.post_shared) {           // one weight for all groups: theirs are added up here
            lds_barrier();
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (threadIdx.x + i * nt) * VEC;
                if (c < p.D)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) wide[c + e] = w1[i][e];
            }
            lds_barrier();
            for (int c = threadIdx.x; c < p.width; c += nt) {
                float s = 0.0f;
                for (int g = 0; g < p.groups; ++g) s += wide[g * p.width + c];
                to[c] = s;
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (threadIdx.x + i * nt) * VEC;
            if (c < p.D) {
                if (p.dpost && !p.post_shared) Piece<float, VEC>::store(to + c, w1[i]);
                if (p.dscale) Piece<float, VEC>::store(to + p.D + c, w2[i]);
                if (p.dpre) Piece<float, VEC>::store(to + 2 * (int64_t)p.D + c, w3[i]);
            }
        }
    }
}

// Sums over workgroups: 16 columns by 64 parts of the workgroups, in a fixed order.
__global__ __launch_bounds__(1024) void k_norm_sums(const NormParams p) {
    __shared__ float part[64][17];
    const int which = blockIdx.y, cl = threadIdx.x & 15, q = threadIdx.x >> 4, c = blockIdx.x * 16 + cl;
    float *to = which == 0 ? p.dpost : which == 1 ? p.dscale : p.dpre;
    if (!to) return;
    const int n = which == 0 && p.post_shared ? p.width : p.D;
    float s = 0.0f;
    if (c < n)
        for (int b = q; b < p.blocks; b += 64) s += p.sums[((int64_t)b * 3 + which) * p.D + c];
    part[q][cl] = s;
    __syncthreads();
    if (q < 4) {
        for (int i = 1; i < 16; ++i) s += part[q + 4 * i][cl];
        part[q][cl] = s;
    }
    __syncthreads();
    if (q == 0 && c < n) to[c] = (s + part[1][cl]) + (part[2][cl] + part[3][cl]);
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
           fits(p.dgate, p.D, es) && fits(p.dres, p.D, rs) && fits(p.sums, p.D, 4) &&
           fits(p.post, 0, 4) && fits(p.scale, 0, 4) && fits(p.pre, 0, 4);
}
static NormShape norm_shape(const NormParams &p) {
    NormShape s;
    s.vec = p.io && norm_rows_fit(p, 8) ? 8 : norm_rows_fit(p, 4) ? 4 : 1;       // 16 bytes of x
    const int pieces = p.D / s.vec, per_group = p.width / s.vec;
    s.nv = 1;                                        // pieces a thread: as few as 512 threads allow
    while ((pieces + s.nv - 1) / s.nv > 512) s.nv = s.nv == 8 ? 12 : s.nv == 12 ? 16 : 2 * s.nv;
    s.nt = ((pieces + s.nv - 1) / s.nv + 63) / 64 * 64;
    const bool pow2 = (per_group & (per_group - 1)) == 0;
    s.how = p.groups == 1 ? GROUP_ROW : pow2 && per_group <= 64 ? GROUP_LANES : GROUP_LDS;
    size_t wide = s.how == GROUP_LDS && p.post ? (size_t)(pieces + p.groups) : 0;
    if (p.dpost && p.post_shared && wide < (size_t)p.D) wide = (size_t)p.D;
    const size_t row = (size_t)weight_room(p.D);
    s.lds = sizeof(float) * (kSumSlots * 8 + (p.post ? p.post_shared ? (size_t)weight_room(p.width) : row : 0) + (p.scale ? row : 0) + (p.pre ? row : 0) + wide);
    return s;
}
template <class IO, class RES, int VEC, int NV, bool BWD> static hipError_t launch_norm_one(const NormParams &p, const NormShape &s, unsigned blocks, hipStream_t st) {
    auto k = k_block_norm<IO, RES, VEC, NV, BWD>;
    if (s.lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)s.lds) != hipSuccess)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(k, dim3(blocks), dim3(s.nt), s.lds, st, p, s.how);
    return hipGetLastError();
}
template <class IO, class RES, int VEC, bool BWD> static hipError_t launch_norm_nv(const NormParams &p, const NormShape &s, unsigned blocks, hipStream_t st) {
    switch (s.nv) {
        case 1: return launch_norm_one<IO, RES, VEC, 1, BWD>(p, s, blocks, st);
        case 2: return launch_norm_one<IO, RES, VEC, 2, BWD>(p, s, blocks, st);
        case 4: if constexpr (VEC <= 4) return launch_norm_one<IO, RES, VEC, 4, BWD>(p, s, blocks, st); break;
        case 8: if constexpr (VEC == 1) return launch_norm_one<IO, RES, VEC, 8, BWD>(p, s, blocks, st); break;
        case 12: if constexpr (VEC == 1) return launch_norm_one<IO, RES, VEC, 12, BWD>(p, s, blocks, st); break;
        case 16: if constexpr (VEC == 1) return launch_norm_one<IO, RES, VEC, 16, BWD>(p, s, blocks, st); break;
    }
    return hipErrorInvalidValue;
}
template <class IO, class RES, bool BWD> static hipError_t launch_norm_vec(const NormParams &p, unsigned blocks, hipStream_t st) {
    const NormShape s = norm_shape(p);
    if constexpr (sizeof(IO) == 2)
        if (s.vec == 8) return launch_norm_nv<IO, RES, 8, BWD>(p, s, blocks, st);
    if (s.vec == 4) return launch_norm_nv<IO, RES, 4, BWD>(p, s, blocks, st);
    return launch_norm_nv<IO, RES, 1, BWD>(p, s, blocks, st);
}
template <bool BWD> static hipError_t launch_norm(const NormParams &p, unsigned blocks, hipStream_t st) {
    if (p.io) return p.res_io ? launch_norm_vec<uint16_t, uint16_t, BWD>(p, blocks, st) : launch_norm_vec<uint16_t, float, BWD>(p, blocks, st);
    return launch_norm_vec<float, float, BWD>(p, blocks, st);
}
// Workgroups: as many as run at once, 24 wavefronts a compute unit forward and 12 backward (registers), each going on to further rows with the next
// one always under way; backward three rows at least once every compute unit
// has one, four once it has two, since a workgroup also leaves three rows of sums behind (1531 rows of 771, float32: 383 workgroups 21.3 us, 511 18.7).
static int norm_blocks(int64_t M, int waves, int waves_per_cu) {
    const int64_t n = 256 * (waves_per_cu / waves);
    return (int)(M < n ? M : n);
}
hipError_t launch_norm_fwd(const NormParams &p, hipStream_t s) { return launch_norm<false>(p, (unsigned)norm_blocks(p.M, norm_shape(p).nt / 64, 24), s); }
int norm_bwd_blocks(int64_t M, int D) {
    const int64_t three = (M + 2) / 3 < 512 ? (M + 2) / 3 : 512, four = (M + 3) / 4, most = three > four ? three : four;
    return norm_blocks(M <= 256 ? M : most > 256 ? most : 256, D <= 4096 ? (D + 511) / 512 : 8, 12);
}
hipError_t launch_norm_bwd(NormParams p, hipStream_t s) {
    const NormShape shape = norm_shape(p);        // fewer than there is room for, where narrow pieces make a row's workgroup larger
    const int each = shape.nv * shape.vec, waves = shape.nt / 64, room = (each >= 16 ? 8 : each >= 8 || shape.nv >= 4 ? 12 : 20) / waves;
    if (p.blocks > 256 * (room > 1 ? room : 1)) p.blocks = 256 * (room > 1 ? room : 1);
    hipError_t e = launch_norm<true>(p, (unsigned)p.blocks, s);
    if (e != hipSuccess || (!p.dpost && !p.dscale && !p.dpre)) return e;
    hipLaunchKernelGGL(k_norm_sums, dim3((unsigned)((p.D + 15) / 16), 3), dim3(1024), 0, s, p);
    return hipGetLastError();
}

}  // namespace lrnnx
