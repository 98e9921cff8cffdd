// Global norm of many tensors, sqrt(sum g^2), and the tensors scaled to a largest norm: g min(1, max_norm / (norm + eps)).
// Squares are taken and added in double precision: no square of a float32 number over- or underflows there, and the sum's rounding is far below the
// result's. Their 64 lanes a clock keep up with memory (two instructions an element against half an element a lane and clock from HBM).
// A workgroup adds up one piece of one tensor, pieces are added by a second launch in a fixed order.  Bound by memory: the norm reads everything once, the scale reads and writes
// it once (8 tensors, 4e8 elements in bfloat16: 138 us, 5.8 TB/s, and 277, 5.8 TB/s); where nothing is to be scaled in place, nothing is read.
#include "grad_clip.hpp"
#include "conv_common.hpp"

namespace lrnnx {

// the tensor that a workgroup's piece belongs to
__device__ __forceinline__ int grad_tensor(const GradList &l, uint32_t piece) {
    int lo = 0, hi = l.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first[mid] <= piece) lo = mid; else hi = mid;
    }
    return lo;
}

template <class T> __device__ __forceinline__ double piece_squares(const T *g, int n) {
    constexpr int V = kFew<T>, U = 4;                      // accesses under way
    double s[2] = {};
    const int whole = n / V * V;
    for (int i = threadIdx.x * V; i < whole; i += 256 * V * U) {
        Few<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            v[u] = Few<T, V>{};
            if (i + u * 256 * V < whole) v[u].load(g + i + u * 256 * V);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) { const double x = v[u].get(e); s[e & 1] = __builtin_fma(x, x, s[e & 1]); }
    }
    if (threadIdx.x < n - whole) { const double x = load_io(g + whole + threadIdx.x); s[0] = __builtin_fma(x, x, s[0]); }
    return s[0] + s[1];
}
// Sum over the workgroup, for its first thread.
template <int THREADS> __device__ __forceinline__ double block_total(double s) {
    __shared__ double part[THREADS / 64];
#pragma unroll
    for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) s += part[i];
    return s;
}
__global__ __launch_bounds__(256) void k_grad_squares(const GradList l, double *sums) {
    const int t = grad_tensor(l, blockIdx.x);
    const int64_t at = (int64_t)(blockIdx.x - l.first[t]) * l.piece, left = l.n[t] - at;
    const int n = (int)(left < l.piece ? left : l.piece);
    double s = l.io[t] & 1 ? piece_squares(reinterpret_cast<const uint16_t *>(l.g[t]) + at, n) : piece_squares(reinterpret_cast<const float *>(l.g[t]) + at, n);
    s = block_total<256>(s);
    if (threadIdx.x == 0) sums[l.base + blockIdx.x] = s;
}
__global__ __launch_bounds__(1024) void k_grad_total(const double *sums, uint32_t count, float *norm) {
    double s = 0;
    for (uint32_t i = threadIdx.x; i < count; i += 1024 * 8) {
        double v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = i + u * 1024 < count ? sums[i + u * 1024] : 0.0;
#pragma unroll
        for (int u = 0; u < 8; ++u) s += v[u];
    }
    s = block_total<1024>(s);
    if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

template <class T, class O> __device__ __forceinline__ void piece_scale(const T *g, O *out, int n, float scale) {
    constexpr int V = sizeof(T) < sizeof(O) ? 4 : kFew<T>, U = 4;
    const int whole = n / V * V;
    for (int i = threadIdx.x * V; i < whole; i += 256 * V * U) {
        Few<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * 256 * V < whole) v[u].load(g + i + u * 256 * V);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * 256 * V < whole) {
                float x[V];
#pragma unroll
                for (int e = 0; e < V; ++e) x[e] = v[u].get(e) * scale;
                Few<O, V>::store(out + i + u * 256 * V, x);
            }
    }
    if (threadIdx.x < n - whole) store_io(out + whole + threadIdx.x, load_io(g + whole + threadIdx.x) * scale);
}
__global__ __launch_bounds__(256) void k_grad_scale(const GradList l, const float *norm, float max_norm, float eps, int in_place) {
    const float all = *norm + eps, scale = all <= max_norm ? 1.0f : max_norm / all;      // (a norm that is NaN stays; 0 / 0 is 1)
    if (in_place && scale == 1.0f) return;
    const int t = grad_tensor(l, blockIdx.x);
    const int64_t at = (int64_t)(blockIdx.x - l.first[t]) * l.piece, left = l.n[t] - at;
    const int n = (int)(left < l.piece ? left : l.piece);
    if (l.io[t] == 0) piece_scale(reinterpret_cast<const float *>(l.g[t]) + at, reinterpret_cast<float *>(l.out[t]) + at, n, scale);
    else if (l.io[t] == 3) piece_scale(reinterpret_cast<const uint16_t *>(l.g[t]) + at, reinterpret_cast<uint16_t *>(l.out[t]) + at, n, scale);
    else piece_scale(reinterpret_cast<const uint16_t *>(l.g[t]) + at, reinterpret_cast<float *>(l.out[t]) + at, n, scale);
}

hipError_t launch_grad_squares(const GradList &l, double *sums, hipStream_t s) {
    hipLaunchKernelGGL(k_grad_squares, dim3(l.first[l.count]), dim3(256), 0, s, l, sums);
    return hipGetLastError();
}
hipError_t launch_grad_total(const double *sums, uint32_t count, float *norm, hipStream_t s) {
    hipLaunchKernelGGL(k_grad_total, dim3(1), dim3(1024), 0, s, sums, count, norm);
    return hipGetLastError();
}
hipError_t launch_grad_scale(const GradList &l, const float *norm, float max_norm, float eps, bool in_place, hipStream_t s) {
    hipLaunchKernelGGL(k_grad_scale, dim3(l.first[l.count]), dim3(256), 0, s, l, norm, max_norm, eps, (int)in_place);
    return hipGetLastError();
}

}  // namespace lrnnx
