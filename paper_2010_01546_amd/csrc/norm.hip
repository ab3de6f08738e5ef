// Rows of a layer's input: norm by the root mean square with the residual's addition, its gradient, and rows in 8 bits.
//
//   h = x + r,  rho = 1 / sqrt(mean h^2 + eps),  y = rho h w;      8 bits: s = max |y| / 127, q = rint(y / s)
//   dx = rho w dy - h rho^3 / M sum(w dy h) + dh,                  dw = sum over rows of dy h rho
//
// Bound by memory: each input is read once and each output written once, a row stays in the registers of its group of threads (a
// wavefront up to 2048 features, a workgroup beyond), 16 bytes per lane and access.
// The sums over a row are float64 (a row of 1e20s has a norm too, and the cost hides behind the loads).  So is q: rho falls out of
// y / s = 127 h w / max |h w|, whose float32 rounding would put one value in 10^5 on the other side of a half.
#include "fw_internal.h"

namespace fw {
namespace {

template <class T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ void load8(const float* p, float (&x)[8]) { __builtin_memcpy(x, p, 32); }
    static __device__ __forceinline__ void store8(float* p, const float (&x)[8]) { __builtin_memcpy(p, x, 32); }
    static __device__ __forceinline__ float get(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
    static __device__ __forceinline__ float held(float v) { return v; }
};
template <> struct Elem<__bf16> {
    static __device__ __forceinline__ void load8(const __bf16* p, float (&x)[8]) {
        bf16x8 v;
        __builtin_memcpy(&v, p, 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
    }
    static __device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) {
        bf16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
        __builtin_memcpy(p, &v, 16);
    }
    static __device__ __forceinline__ float get(const __bf16* p) { return (float)*p; }
    static __device__ __forceinline__ void put(__bf16* p, float v) { *p = (__bf16)v; }
    static __device__ __forceinline__ float held(float v) { return (float)(__bf16)v; }
};

// 8 entries of a row of which `left` remain (rows need not be 16-byte aligned); zero beyond the end
template <class T> __device__ __forceinline__ void load8(const T* p, int left, float (&x)[8]) {
    if (left >= 8) { Elem<T>::load8(p, x); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < left ? Elem<T>::get(p + i) : 0.f;
}
template <class T> __device__ __forceinline__ void store8(T* p, int left, const float (&x)[8]) {
    if (left >= 8) { Elem<T>::store8(p, x); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) Elem<T>::put(p + i, x[i]);
}

// over the G threads of a row's group; every thread gets the result
template <int G, class Op> __device__ __forceinline__ double group_reduce(double v, double* red, Op op) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o, 64));
    if (G > 64) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();                     // the previous use of `red` is over
        if ((threadIdx.x & 63) == 0) red[wave] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int i = 1; i < G / 64; ++i) v = op(v, red[i]);
    }
    return v;
}
struct Sum { __device__ double operator()(double a, double b) const { return a + b; } };
struct Max { __device__ double operator()(double a, double b) const { return a > b ? a : b; } };

// NORM: rows of the root mean square norm, otherwise the rows as they are (8 bits only)
template <class T, int G, int NV, bool NORM>
__global__ __launch_bounds__(G < 256 ? 256 : G) void rows_kernel(const T* X, const T* R, int N, int M, const float* __restrict__ w, float eps,
                                                                 T* H, T* Y, signed char* __restrict__ q, float* __restrict__ qs) {
    __shared__ double red[16];
    const int t = threadIdx.x % G;
    const long long row = (long long)blockIdx.x * (blockDim.x / G) + threadIdx.x / G;
    if (row >= N) return;                    // whole wavefronts, and only where a group is one
    const size_t at = (size_t)row * M;
    float h[NV][8];
    double ss = 0.0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int m = 8 * (t + G * j);
        if (m >= M) break;
        load8(X + at + m, M - m, h[j]);
        if (NORM && R) {
            float r[8];
            load8(R + at + m, M - m, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[j][i] = Elem<T>::held(h[j][i] + r[i]);
        }
        if (NORM) {
#pragma unroll
            for (int i = 0; i < 8; ++i) ss += (double)h[j][i] * (double)h[j][i];
        }
    }
    double rho = 1.0;
    if (NORM) {
        if (H) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int m = 8 * (t + G * j);
                if (m < M) store8(H + at + m, M - m, h[j]);
            }
        }
        ss = group_reduce<G>(ss, red, Sum());
        rho = 1.0 / sqrt(ss / (double)M + (double)eps);
        if (Y) {
            const float rf = (float)rho;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int m = 8 * (t + G * j);
                if (m >= M) break;
                float y[8];
                if (w) load8(w + m, M - m, y);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = h[j][i] * rf * (w ? y[i] : 1.f);
                store8(Y + at + m, M - m, y);
            }
        }
    }
    if (!NORM || q) {
        double top = 0.0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int m = 8 * (t + G * j);
            if (m >= M) break;
            float f[8];
            if (NORM && w) load8(w + m, M - m, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double a = fabs(NORM && w ? (double)h[j][i] * (double)f[i] : (double)h[j][i]);
                top = fmax(top, a < __builtin_inf() ? a : __builtin_inf());   // NaN counts as infinite
            }
        }
        top = group_reduce<G>(top, red, Max());
        const bool fine = top > 0.0 && top < __builtin_inf() && rho > 0.0;
        const double inv = fine ? 127.0 / top : 0.0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int m = 8 * (t + G * j);
            if (m >= M) break;
            float f[8];
            if (NORM && w) load8(w + m, M - m, f);
            signed char b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double a = NORM && w ? (double)h[j][i] * (double)f[i] : (double)h[j][i];
                b[i] = fine ? (signed char)(int)rint(a * inv) : (signed char)0;
            }
            if (M - m >= 8) {
                __builtin_memcpy(q + at + m, b, 8);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < M - m) q[at + m + i] = b[i];
            }
        }
        if (t == 0) qs[row] = top == 0.0 && rho > 0.0 ? 0.f : fine ? (float)(rho * top / 127.0) : __builtin_nanf("");
    }
}

// Workgroups take rows in turn; each keeps the sums of its rows' dy h rho and leaves them in part[workgroup][M].
template <class T, int G, int NV>
__global__ __launch_bounds__(G < 256 ? 256 : G) void rms_grad_kernel(const T* __restrict__ H, int N, int M, const float* __restrict__ w, float eps,
                                                                     const T* dY, const T* dH, T* dX, float* __restrict__ part) {
    constexpr int RB = G < 256 ? 256 / G : 1;
    __shared__ double red[16];
    __shared__ float acc[RB > 1 ? RB * 8 * G * NV : 1];
    const int t = threadIdx.x % G, sub = threadIdx.x / G;
    float sum[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[j][i] = 0.f;
    for (long long row = (long long)blockIdx.x * RB + sub; row < N; row += (long long)gridDim.x * RB) {
        const size_t at = (size_t)row * M;
        float h[NV][8], v[NV][8];
        double ss = 0.0, dot = 0.0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int m = 8 * (t + G * j);
            if (m >= M) break;
            load8(H + at + m, M - m, h[j]);
            load8(dY + at + m, M - m, v[j]);
            float f[8];
            if (w) load8(w + m, M - m, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                ss += (double)h[j][i] * (double)h[j][i];
                dot += (double)h[j][i] * (w ? (double)v[j][i] * (double)f[i] : (double)v[j][i]);
            }
        }
        ss = group_reduce<G>(ss, red, Sum());
        dot = group_reduce<G>(dot, red, Sum());
        const double rho = 1.0 / sqrt(ss / (double)M + (double)eps);
        const float rf = (float)rho, cf = (float)(rho * rho * rho * dot / (double)M);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int m = 8 * (t + G * j);
            if (m >= M) break;
            if (part) {
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[j][i] += v[j][i] * (h[j][i] * rf);
            }
            if (dX) {
                float f[8], d[8];
                if (w) load8(w + m, M - m, f);
                if (dH) load8(dH + at + m, M - m, d);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float x = rf * (w ? v[j][i] * f[i] : v[j][i]) - h[j][i] * cf;
                    v[j][i] = dH ? x + d[i] : x;
                }
                store8(dX + at + m, M - m, v[j]);
            }
        }
    }
    if (!part) return;
    if (RB > 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[(sub * NV + j) * 8 * G + 8 * t + i] = sum[j][i];
        __syncthreads();
        for (int m = threadIdx.x; m < M; m += blockDim.x) {
            float s = 0.f;
#pragma unroll
            for (int r = 0; r < RB; ++r) s += acc[r * NV * 8 * G + m];
            part[(size_t)blockIdx.x * M + m] = s;
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int m = 8 * (t + G * j);
            if (m < M) store8(part + (size_t)blockIdx.x * M + m, M - m, sum[j]);
        }
    }
}

// dw[m] = sum of the workgroups' partial sums, in a fixed order: 16 slices of them, then the slices
__global__ __launch_bounds__(1024) void column_sum_kernel(const float* __restrict__ part, int P, int M, float* __restrict__ dw) {
    __shared__ float red[16][64];
    const int m = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
    float s = 0.f;
    if (m < M)
        for (int p = slice; p < P; p += 16) s += part[(size_t)p * M + m];
    red[slice][threadIdx.x & 63] = s;
    __syncthreads();
    if (slice == 0 && m < M) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v += red[i][threadIdx.x];
        dw[m] = v;
    }
}

inline int rows_per_group(int M) { return M <= 2048 ? 4 : 1; }
inline int grad_blocks(int N, int M) {
    const int rb = rows_per_group(M);
    const long long b = ((long long)N + rb - 1) / rb;
    return (int)(b < 1024 ? b : 1024);
}

template <class T, bool NORM>
fw_status rows_launch(const void* X, const void* R, int N, int M, const float* w, float eps, void* H, void* Y, signed char* q, float* qs,
                      hipStream_t st) {
    const int rb = rows_per_group(M);
    const dim3 grid((unsigned)(((long long)N + rb - 1) / rb));
    const T *x = reinterpret_cast<const T*>(X), *r = reinterpret_cast<const T*>(R);
    T *h = reinterpret_cast<T*>(H), *y = reinterpret_cast<T*>(Y);
#define FW_ROWS(G, NV) hipLaunchKernelGGL((rows_kernel<T, G, NV, NORM>), grid, dim3(G < 256 ? 256 : G), 0, st, x, r, N, M, w, eps, h, y, q, qs)
    if (M <= 512) FW_ROWS(64, 1);
    else if (M <= 1024) FW_ROWS(64, 2);
    else if (M <= 2048) FW_ROWS(64, 4);
    else if (M <= 8192) FW_ROWS(256, 4);
    else if (M <= 16384) FW_ROWS(512, 4);
    else FW_ROWS(1024, 4);
#undef FW_ROWS
    FW_LAUNCH_CHECK();
    return FW_OK;
}

template <class T>
fw_status grad_launch(const void* H, int N, int M, const float* w, float eps, const void* dY, const void* dH, void* dX, float* part,
                      hipStream_t st) {
    const dim3 grid(grad_blocks(N, M));
    const T *h = reinterpret_cast<const T*>(H), *dy = reinterpret_cast<const T*>(dY), *dh = reinterpret_cast<const T*>(dH);
    T* dx = reinterpret_cast<T*>(dX);
#define FW_GRAD(G, NV) hipLaunchKernelGGL((rms_grad_kernel<T, G, NV>), grid, dim3(G < 256 ? 256 : G), 0, st, h, N, M, w, eps, dy, dh, dx, part)
    if (M <= 512) FW_GRAD(64, 1);
    else if (M <= 1024) FW_GRAD(64, 2);
    else if (M <= 2048) FW_GRAD(64, 4);
    else if (M <= 8192) FW_GRAD(256, 4);
    else if (M <= 16384) FW_GRAD(512, 4);
    else FW_GRAD(1024, 4);
#undef FW_GRAD
    FW_LAUNCH_CHECK();
    return FW_OK;
}

}  // namespace

fw_status rms_norm(const void* X, const void* R, fw_dtype dt, int N, int M, const float* w, float eps, void* H, void* Y, signed char* q,
                   float* qs, hipStream_t st) {
    return dt == FW_BF16 ? rows_launch<__bf16, true>(X, R, N, M, w, eps, H, Y, q, qs, st)
                         : rows_launch<float, true>(X, R, N, M, w, eps, H, Y, q, qs, st);
}

fw_status int8_rows(const void* X, fw_dtype dt, int N, int M, signed char* q, float* qs, hipStream_t st) {
    return dt == FW_BF16 ? rows_launch<__bf16, false>(X, nullptr, N, M, nullptr, 0.f, nullptr, nullptr, q, qs, st)
                         : rows_launch<float, false>(X, nullptr, N, M, nullptr, 0.f, nullptr, nullptr, q, qs, st);
}

size_t rms_norm_grad_workspace_bytes(int N, int M) { return align_up((size_t)grad_blocks(N, M) * M * sizeof(float), 256); }

fw_status rms_norm_grad(const void* H, fw_dtype dt, int N, int M, const float* w, float eps, const void* dY, const void* dH, void* dX,
                        float* dw, void* ws, hipStream_t st) {
    float* part = dw ? reinterpret_cast<float*>(ws) : nullptr;
    const fw_status rc = dt == FW_BF16 ? grad_launch<__bf16>(H, N, M, w, eps, dY, dH, dX, part, st)
                                       : grad_launch<float>(H, N, M, w, eps, dY, dH, dX, part, st);
    if (rc != FW_OK || !dw) return rc;
    hipLaunchKernelGGL(column_sum_kernel, dim3((M + 63) / 64), dim3(1024), 0, st, part, grad_blocks(N, M), M, dw);
    FW_LAUNCH_CHECK();
    return FW_OK;
}

}  // namespace fw
