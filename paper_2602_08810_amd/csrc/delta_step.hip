// Gated delta rule, one step of a carried state S [dk,dv] of every batch entry and head, in place:
//     u = beta (v - exp(g) S^T k),   S <- exp(g) S + k u^T,   o = scale S^T q = scale (exp(g) S^T q + (k . q) u)
// Both products with the old state are taken in one pass, so the state is read once and written once from registers: the bytes of the state are
// what a call costs (4096 states of 128 x 128: 540 MB in 112 us, 97 % of the rate of a copy), and with few states the latency of one pass (16: 4.4 us).
// A workgroup takes 32 columns of one state: 8 threads of four columns each side by side, 32 threads along the rows.
#include "delta_common.hpp"

namespace lrnnx {

template <class IO, bool VEC> __global__ __launch_bounds__(256) void k_delta_step(const DeltaStepParams p) {
    constexpr int NR = 4;                                  // rows a thread (dk <= 128)
    __shared__ float sums[4][8][9];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cl = tid & 7, rl = tid >> 3;
    const int h = blockIdx.y, b = blockIdx.z, hk = h / (p.Hv / p.Hk), c = (blockIdx.x * 8 + cl) * 4;
    const IO *q = reinterpret_cast<const IO *>(p.q) + b * p.q_sb + hk * p.q_sh, *k = reinterpret_cast<const IO *>(p.k) + b * p.k_sb + hk * p.k_sh;
    const IO *v = reinterpret_cast<const IO *>(p.v) + b * p.v_sb + h * p.v_sh;
    float *S = p.state + ((int64_t)b * p.Hv + h) * p.dk * p.dv + c;
    const int left = p.dv - c;
    f32x4 x[NR];
    float kr[NR], qr[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int d = rl + 32 * i;
        x[i] = f32x4{};
        kr[i] = qr[i] = 0.0f;
        if (d < p.dk) {
            if (VEC) { if (left > 0) x[i] = *reinterpret_cast<const f32x4 *>(S + (int64_t)d * p.dv); }
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) if (e < left) x[i][e] = S[(int64_t)d * p.dv + e];
            kr[i] = load_io(k + d);
            qr[i] = load_io(q + d);
        }
    }
    const int io = sizeof(IO) == 2;
    const float a = __expf(load_gate(p.g, b * p.g_sb + h * p.g_sh, io, p.gate_io));
    const float be = load_gate(p.beta, b * p.be_sb + h * p.be_sh, io, p.gate_io);
    f32x4 vv = {};
#pragma unroll
    for (int e = 0; e < 4; ++e) if (e < left) vv[e] = load_io(v + c + e);
    float t[9] = {};                                       // S^T k, S^T q, k . q
#pragma unroll
    for (int i = 0; i < NR; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            t[e] = __builtin_fmaf(kr[i], x[i][e], t[e]);
            t[4 + e] = __builtin_fmaf(qr[i], x[i][e], t[4 + e]);
        }
        t[8] = __builtin_fmaf(kr[i], qr[i], t[8]);
    }
#pragma unroll
    for (int m = 8; m < 64; m <<= 1)
#pragma unroll
        for (int j = 0; j < 9; ++j) t[j] += __shfl_xor(t[j], m, 64);
    if (lane < 8)
#pragma unroll
        for (int j = 0; j < 9; ++j) sums[wave][cl][j] = t[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 9; ++j) t[j] = (sums[0][cl][j] + sums[1][cl][j]) + (sums[2][cl][j] + sums[3][cl][j]);
    f32x4 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = be * __builtin_fmaf(-a, t[e], vv[e]);
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int d = rl + 32 * i;
        if (d < p.dk) {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][e] = __builtin_fmaf(kr[i], u[e], a * x[i][e]);
            if (VEC) { if (left > 0) *reinterpret_cast<f32x4 *>(S + (int64_t)d * p.dv) = x[i]; }
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) if (e < left) S[(int64_t)d * p.dv + e] = x[i][e];
        }
    }
    if (rl == 0) {
        IO *o = reinterpret_cast<IO *>(p.o) + b * p.o_sb + h * p.o_sh + c;
#pragma unroll
        for (int e = 0; e < 4; ++e) if (e < left) store_io(o + e, p.scale * __builtin_fmaf(t[8], u[e], a * t[4 + e]));
    }
}

hipError_t launch_delta_step(const DeltaStepParams &p, int io, hipStream_t s) {
    const dim3 grid((unsigned)((p.dv + 31) / 32), (unsigned)p.Hv, (unsigned)p.B), block(256);
    const bool vec = p.dv % 4 == 0 && (reinterpret_cast<uintptr_t>(p.state) & 15) == 0;
    if (io) {
        if (vec) hipLaunchKernelGGL((k_delta_step<uint16_t, true>), grid, block, 0, s, p);
        else hipLaunchKernelGGL((k_delta_step<uint16_t, false>), grid, block, 0, s, p);
    } else {
        if (vec) hipLaunchKernelGGL((k_delta_step<float, true>), grid, block, 0, s, p);
        else hipLaunchKernelGGL((k_delta_step<float, false>), grid, block, 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace lrnnx
