// Gated feed-forward block and its gradient:
//   g = X Wg^T + bg,  u = X Wu^T + bu,  H = act(g) u;      kept for the backward pass: Z[0] = u act'(g), Z[1] = act(g)
//   dg = dH Z[0],  du = dH Z[1],   dX = dg Wg + du Wu,   dWg = dg^T (X - 1 mu^T),  dWu = du^T (X - 1 mu^T),  db = column sums
#include "fw_internal.h"
#include "tile_product.h"

namespace fw {
namespace {

// value and slope of the activation
__device__ __forceinline__ void activation(fw_act act, float g, float& a, float& da) {
    if (act == FW_ACT_SILU) {
        const float s = 1.f / (1.f + expf(-g));
        a = g * s;
        da = s * (1.f + g * (1.f - s));
    } else if (act == FW_ACT_GELU) {
        const float p = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        a = g * p;
        da = p + g * expf(-0.5f * g * g) * 0.39894228040143268f;
    } else if (act == FW_ACT_GELU_TANH) {
        const float k = 0.79788456080286536f, t = tanhf(k * (g + 0.044715f * g * g * g));
        a = 0.5f * g * (1.f + t);
        da = 0.5f * (1.f + t) + 0.5f * g * (1.f - t * t) * k * (1.f + 0.134145f * g * g);
    } else {
        a = g > 0.f ? g : 0.f;
        da = g > 0.f ? 1.f : 0.f;
    }
}

template <class T>
__global__ __launch_bounds__(256) void gate_kernel(const float* __restrict__ gu, size_t n, int S, const float* __restrict__ bg,
                                                   const float* __restrict__ bu, fw_act act, T* __restrict__ H, T* __restrict__ Z) {
    for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (size_t)gridDim.x * 256) {
        const int s = (int)(e % S);
        const float g = gu[e] + (bg ? bg[s] : 0.f), u = gu[n + e] + (bu ? bu[s] : 0.f);
        float a, da;
        activation(act, g, a, da);
        H[e] = (T)(a * u);
        if (Z) { Z[e] = (T)(u * da); Z[n + e] = (T)a; }
    }
}

template <class T>
__global__ __launch_bounds__(256) void gate_grad_kernel(const T* __restrict__ dH, const T* __restrict__ Z, size_t n, T* __restrict__ D) {
    for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (size_t)gridDim.x * 256) {
        const float d = (float)dH[e];
        D[e] = (T)(d * (float)Z[e]);
        D[n + e] = (T)(d * (float)Z[n + e]);
    }
}

// sums[s] of the columns of D [2][N][S], gate's first
template <class T>
__global__ __launch_bounds__(256) void bias_grad_kernel(const T* __restrict__ D, int N, int S, float* __restrict__ sums, T* __restrict__ dbg,
                                                        T* __restrict__ dbu) {
    const int s = blockIdx.x * 256 + threadIdx.x;
    if (s >= S) return;
    const T* p = D + (size_t)blockIdx.y * N * S + s;
    float v = 0.f;
    for (int n = 0; n < N; ++n) v += (float)p[(size_t)n * S];
    sums[blockIdx.y * S + s] = v;
    if (dbg) (blockIdx.y ? dbu : dbg)[s] = (T)v;
}

inline unsigned blocks_for(size_t n) { return (unsigned)((n + 255) / 256 < 16384 ? (n + 255) / 256 : 16384); }

template <class T>
fw_status forward(const T* X, int N, int M, int S, const T* Wg, const T* Wu, const float* bg, const float* bu, fw_act act, T* H, T* Z,
                  float* gu, hipStream_t st) {
    const size_t n = (size_t)N * S;
    for (int k = 0; k < 2; ++k) {
        float* out = gu + k * n;
        const fw_status rc = strided_product<float>(X, M, 1, k ? Wu : Wg, M, 1, N, S, M,
                                                    [=] __device__(long long r, int c, float v) { out[r * S + c] = v; }, st);
        if (rc != FW_OK) return rc;
    }
    hipLaunchKernelGGL(gate_kernel<T>, dim3(blocks_for(n)), dim3(256), 0, st, gu, n, S, bg, bu, act, H, Z);
    FW_LAUNCH_CHECK();
    return FW_OK;
}

template <class T>
fw_status backward(const T* X, int N, int M, int S, const T* Wg, const T* Wu, const T* Z, const T* dH, const float* mu, T* dX, T* dWg, T* dWu,
                   T* dbg, T* dbu, char* ws, hipStream_t st) {
    const size_t n = (size_t)N * S;
    T* D = reinterpret_cast<T*>(ws);
    float* sums = reinterpret_cast<float*>(ws + align_up(2 * n * sizeof(T), 256));
    float* wide = reinterpret_cast<float*>(ws + align_up(2 * n * sizeof(T), 256) + align_up(2 * (size_t)S * sizeof(float), 256));
    hipLaunchKernelGGL(gate_grad_kernel<T>, dim3(blocks_for(n)), dim3(256), 0, st, dH, Z, n, D);
    FW_LAUNCH_CHECK();
    if (dbg || mu) {
        hipLaunchKernelGGL(bias_grad_kernel<T>, dim3((S + 255) / 256, 2), dim3(256), 0, st, D, N, S, sums, dbg, dbu);
        FW_LAUNCH_CHECK();
    }
    if (dX) {
        fw_status rc = strided_product<float>(D, S, 1, Wg, 1, M, N, M, S, [=] __device__(long long r, int c, float v) { wide[r * M + c] = v; }, st);
        if (rc != FW_OK) return rc;
        rc = strided_product<float>(D + n, S, 1, Wu, 1, M, N, M, S,
                                    [=] __device__(long long r, int c, float v) { dX[r * M + c] = (T)(wide[r * M + c] + v); }, st);
        if (rc != FW_OK) return rc;
    }
    for (int k = 0; dWg && k < 2; ++k) {
        T* out = k ? dWu : dWg;
        const float* sum = sums + k * S;
        const fw_status rc = strided_product<float>(D + k * n, 1, S, X, 1, M, S, M, N, [=] __device__(long long r, int c, float v) {
            out[r * M + c] = (T)(mu ? v - sum[r] * mu[c] : v);
        }, st);
        if (rc != FW_OK) return rc;
    }
    return FW_OK;
}

}  // namespace

size_t gated_forward_workspace_bytes(fw_dtype, int N, int, int S) { return align_up(2 * (size_t)N * S * sizeof(float), 256); }
size_t gated_grad_workspace_bytes(fw_dtype dt, int N, int M, int S) {
    return align_up(2 * (size_t)N * S * (dt == FW_BF16 ? 2 : 4), 256) + align_up(2 * (size_t)S * sizeof(float), 256) +
           align_up((size_t)N * M * sizeof(float), 256);
}

fw_status gated_forward(const void* X, fw_dtype dt, int N, int M, int S, const void* Wg, const void* Wu, const float* bg, const float* bu,
                        fw_act act, void* H, void* Z, void* ws, hipStream_t st) {
    float* gu = reinterpret_cast<float*>(ws);
    if (dt == FW_BF16)
        return forward((const __bf16*)X, N, M, S, (const __bf16*)Wg, (const __bf16*)Wu, bg, bu, act, (__bf16*)H, (__bf16*)Z, gu, st);
    return forward((const float*)X, N, M, S, (const float*)Wg, (const float*)Wu, bg, bu, act, (float*)H, (float*)Z, gu, st);
}

fw_status gated_grad(const void* X, fw_dtype dt, int N, int M, int S, const void* Wg, const void* Wu, const void* Z, const void* dH,
                     const float* mu, void* dX, void* dWg, void* dWu, void* dbg, void* dbu, void* ws, hipStream_t st) {
    char* w = reinterpret_cast<char*>(ws);
    if (dt == FW_BF16)
        return backward((const __bf16*)X, N, M, S, (const __bf16*)Wg, (const __bf16*)Wu, (const __bf16*)Z, (const __bf16*)dH, mu, (__bf16*)dX,
                        (__bf16*)dWg, (__bf16*)dWu, (__bf16*)dbg, (__bf16*)dbu, w, st);
    return backward((const float*)X, N, M, S, (const float*)Wg, (const float*)Wu, (const float*)Z, (const float*)dH, mu, (float*)dX,
                    (float*)dWg, (float*)dWu, (float*)dbg, (float*)dbu, w, st);
}

}  // namespace fw
