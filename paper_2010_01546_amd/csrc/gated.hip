// Gated feed-forward block and its gradient:
//   g = X Wg^T + bg,  u = X Wu^T + bu,  H = act(g) u;      kept for the backward pass: Z[0] = u act'(g), Z[1] = act(g)
//   dg = dH Z[0],  du = dH Z[1],   dX = dg Wg + du Wu,   dWg = dg^T (X - 1 mu^T),  dWu = du^T (X - 1 mu^T),  db = column sums
//
// bfloat16: both projections in one launch, the panel of weights holding the same columns of Wg and Wu, so that a lane has g and u of
// an element in its registers when the sums are done (tile_product.h).  The backward pass forms D = [dg | du] once, rounded to
// bfloat16, [N][2 Sp] with Sp = S rounded up to 64 and zeros between, and takes two products of it: dX = D [Wg; Wu], whose contraction runs
// over the rows of both weight matrices, and [dWg; dWu] = D^T X.  Operands that are contraction-major in memory are turned on the
// way out of LDS, not in memory.  mu is taken out of the sums: D^T (X - 1 mu^T) = D^T X - (D^T 1) mu^T, with D^T 1 summed from the
// rounded D, so that the identity is exact but for float32 sums.
// float32: products with float32 accuracy on the bfloat16 matrix cores (gemm_planes.hip), operands transposed in the workspace.
#include "fw_internal.h"
#include "tile_product.h"

namespace fw {
namespace {

// value and slope of the activation; exp and the reciprocal of the hardware, a few units in the last place of max(|g|, 1)
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __expf(-g)); }
template <int ACT> __device__ __forceinline__ void activation(float g, float& a, float& da) {
    if constexpr (ACT == FW_ACT_SILU) {
        const float s = sigmoid(g);
        a = g * s;
        da = s * (1.f + g * (1.f - s));
    } else if constexpr (ACT == FW_ACT_GELU) {
        const float p = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        a = g * p;
        da = p + g * __expf(-0.5f * g * g) * 0.39894228040143268f;
    } else if constexpr (ACT == FW_ACT_GELU_TANH) {
        // (1 + tanh z) / 2 = sigmoid(2 z)
        const float k = 0.79788456080286536f, p = sigmoid(2.f * k * (g + 0.044715f * g * g * g));
        a = g * p;
        da = p + 2.f * g * p * (1.f - p) * k * (1.f + 0.134145f * g * g);
    } else {
        a = g > 0.f ? g : 0.f;
        da = g > 0.f ? 1.f : 0.f;
    }
}
template <class F> __device__ __forceinline__ void with_activation(int act, const F& f) {
    if (act == FW_ACT_SILU) f(std::integral_constant<int, FW_ACT_SILU>());
    else if (act == FW_ACT_GELU) f(std::integral_constant<int, FW_ACT_GELU>());
    else if (act == FW_ACT_GELU_TANH) f(std::integral_constant<int, FW_ACT_GELU_TANH>());
    else f(std::integral_constant<int, FW_ACT_RELU>());
}

// ---- epilogues of the bfloat16 products: four entries of a row
struct GateEpilogue {
    __bf16* H;
    float* Z;
    const float *bg, *bu;
    int N, S, act;
    __device__ __forceinline__ void apply(int n, int s, const floatx4& gate, const floatx4& up) const {
        if (n >= N || s >= S) return;
        float b[4], c[4], h[4];
        tile_vector(bg, s, S, b);
        tile_vector(bu, s, S, c);
        with_activation(act, [&](auto ACT) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float u = up[i] + c[i];
                float a, da;
                activation<decltype(ACT)::value>(gate[i] + b[i], a, da);
                h[i] = a * u;
                b[i] = u * da;
                c[i] = a;
            }
        });
        const size_t e = (size_t)n * S + s;
        tile_store(H + e, s, S, h);
        if (Z) {
            tile_store(Z + e, s, S, b);
            tile_store(Z + (size_t)N * S + e, s, S, c);
        }
    }
};
struct RowsEpilogue {                     // dX
    __bf16* out;
    int N, M;
    __device__ __forceinline__ void apply(int n, int m, const floatx4& acc) const {
        if (n >= N || m >= M) return;
        const float v[4] = {acc[0], acc[1], acc[2], acc[3]};
        tile_store(out + (size_t)n * M + m, m, M, v);
    }
};
struct WeightsEpilogue {                  // rows below Sp are the gate's, the others the up projection's
    __bf16 *dWg, *dWu;
    const float *sums, *mu;
    int S, Sp, M;
    __device__ __forceinline__ void apply(int r, int m, const floatx4& acc) const {
        const int s = r >= Sp ? r - Sp : r;
        if (s >= S || m >= M) return;
        float v[4] = {acc[0], acc[1], acc[2], acc[3]};
        if (mu) {
            const float d = sums[r];
            float c[4];
            tile_vector(mu, m, M, c);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] -= d * c[i];
        }
        tile_store((r >= Sp ? dWu : dWg) + (size_t)s * M + m, m, M, v);
    }
};

// ---- elementwise passes
// float32: g and u [2][N][S] before the biases -> H, Z
__global__ __launch_bounds__(256) void gate_kernel(const float* __restrict__ gu, size_t n, int S, const float* __restrict__ bg,
                                                   const float* __restrict__ bu, int act, float* __restrict__ H, float* __restrict__ Z) {
    for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (size_t)gridDim.x * 256) {
        const int s = (int)(e % S);
        const float g = gu[e] + (bg ? bg[s] : 0.f), u = gu[n + e] + (bu ? bu[s] : 0.f);
        with_activation(act, [&](auto ACT) {
            float a, da;
            activation<decltype(ACT)::value>(g, a, da);
            H[e] = a * u;
            if (Z) { Z[e] = u * da; Z[n + e] = a; }
        });
    }
}

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void load4(const __bf16* p, float (&x)[4]) {
    bf16x4 v;
    __builtin_memcpy(&v, p, 8);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)v[i];
}
__device__ __forceinline__ void load4(const float* p, float (&x)[4]) { __builtin_memcpy(x, p, 16); }
__device__ __forceinline__ void store4(__bf16* p, float (&x)[4]) {     // x: as rounded
    bf16x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = (__bf16)x[i]; x[i] = (float)v[i]; }
    __builtin_memcpy(p, &v, 8);
}
__device__ __forceinline__ void store4(float* p, float (&x)[4]) { __builtin_memcpy(p, x, 16); }

constexpr int GG_ROWS = 64;      // rows of a workgroup: 16 for each of its four wavefronts, 256 columns
// D[n] = [dg | du] of row n, each Sp wide (zeros past S); part[block of rows][2 Sp]: sums over the block's rows, or null
template <class T>
__global__ __launch_bounds__(256) void gate_grad_kernel(const T* __restrict__ dH, const float* __restrict__ Z, int N, int S, int Sp,
                                                        T* __restrict__ D, float* __restrict__ part) {
    __shared__ float red[4][2][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int s = blockIdx.x * 256 + 4 * lane;
    const int n0 = blockIdx.y * GG_ROWS + wave * (GG_ROWS / 4), n1 = min(n0 + GG_ROWS / 4, N);
    float sg[4] = {}, su[4] = {};
    if (s < Sp) {
        for (int n = n0; n < n1; ++n) {
            const size_t e = (size_t)n * S + s;
            float h[4], p[4], q[4];
            if (s + 4 <= S) {
                load4(dH + e, h);
                load4(Z + e, p);
                load4(Z + (size_t)N * S + e, q);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool in = s + i < S;
                    h[i] = in ? (float)dH[e + i] : 0.f;
                    p[i] = in ? Z[e + i] : 0.f;
                    q[i] = in ? Z[(size_t)N * S + e + i] : 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) { p[i] *= h[i]; q[i] *= h[i]; }
            T* d = D + (size_t)n * 2 * Sp + s;
            store4(d, p);
            store4(d + Sp, q);
#pragma unroll
            for (int i = 0; i < 4; ++i) { sg[i] += p[i]; su[i] += q[i]; }
        }
    }
    if (!part) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) { red[wave][0][4 * lane + i] = sg[i]; red[wave][1][4 * lane + i] = su[i]; }
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < Sp) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            part[((size_t)blockIdx.y * 2 + k) * Sp + c] =
                red[0][k][threadIdx.x] + red[1][k][threadIdx.x] + red[2][k][threadIdx.x] + red[3][k][threadIdx.x];
    }
}

// sums[c] = the blocks' partial sums, in a fixed order; the biases' gradients where they are asked for
template <class T>
__global__ __launch_bounds__(1024) void bias_grad_kernel(const float* __restrict__ part, int blocks, int S, int Sp, float* __restrict__ sums,
                                                         T* __restrict__ dbg, T* __restrict__ dbu) {
    __shared__ float red[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
    float v = 0.f;
    if (c < 2 * Sp)
        for (int p = slice; p < blocks; p += 16) v += part[(size_t)p * 2 * Sp + c];
    red[slice][threadIdx.x & 63] = v;
    __syncthreads();
    if (slice || c >= 2 * Sp) return;
    v = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += red[i][threadIdx.x];
    sums[c] = v;
    const int s = c >= Sp ? c - Sp : c;
    if (dbg && s < S) (c >= Sp ? dbu : dbg)[s] = (T)v;
}

// rows of M bfloat16 numbers to rows of Mp (a multiple of 8), zeros behind
__global__ __launch_bounds__(256) void pad_rows_kernel(const __bf16* __restrict__ in, int M, int Mp, size_t n8, bf16x8* __restrict__ out) {
    const int c8 = Mp / 8;
    for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < n8; e += (size_t)gridDim.x * 256) {
        const size_t r = e / c8;
        const int m = 8 * (int)(e - r * c8);
        const __bf16* p = in + r * M + m;
        bf16x8 v;
        if (m + 8 <= M) {
            __builtin_memcpy(&v, p, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = m + i < M ? p[i] : (__bf16)0.f;
        }
        out[e] = v;
    }
}

// out[c][col0 + r] = in[r][c] - mu[c], float32, row length `pitch`; rows r from R to Rp are written as zeros
__global__ __launch_bounds__(256) void transpose_kernel(const float* __restrict__ in, int R, int C, int in_pitch, const float* __restrict__ mu,
                                                        float* __restrict__ out, size_t pitch, int col0, int Rp) {
    __shared__ float t[32][33];
    const int r0 = blockIdx.x * 32, c0 = blockIdx.y * 32, x = threadIdx.x & 31, y = threadIdx.x >> 5;
#pragma unroll
    for (int k = 0; k < 32; k += 8) {
        const int r = r0 + y + k, c = c0 + x;
        t[y + k][x] = r < R && c < C ? in[(size_t)r * in_pitch + c] - (mu ? mu[c] : 0.f) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 32; k += 8) {
        const int c = c0 + y + k, r = r0 + x;
        if (c < C && r < Rp) out[(size_t)c * pitch + col0 + r] = t[x][y + k];
    }
}

inline unsigned blocks_for(size_t n) { return (unsigned)((n + 255) / 256 < 16384 ? (n + 255) / 256 : 16384); }
inline int up8(int m) { return (m + 7) / 8 * 8; }
inline int up64(int s) { return (s + 63) / 64 * 64; }
inline int row_blocks(int N) { return (N + GG_ROWS - 1) / GG_ROWS; }
inline const char* bytes(const void* p) { return reinterpret_cast<const char*>(p); }

fw_status pad_rows(const void* in, int R, int M, void* out, hipStream_t st) {
    const size_t n8 = (size_t)R * (up8(M) / 8);
    hipLaunchKernelGGL(pad_rows_kernel, dim3(blocks_for(n8)), dim3(256), 0, st, reinterpret_cast<const __bf16*>(in), M, up8(M), n8,
                       reinterpret_cast<bf16x8*>(out));
    FW_LAUNCH_CHECK();
    return FW_OK;
}
fw_status transpose(const float* in, int R, int C, int in_pitch, const float* mu, float* out, size_t pitch, int col0, int Rp, hipStream_t st) {
    hipLaunchKernelGGL(transpose_kernel, dim3((Rp + 31) / 32, (C + 31) / 32), dim3(256), 0, st, in, R, C, in_pitch, mu, out, pitch, col0, Rp);
    FW_LAUNCH_CHECK();
    return FW_OK;
}

// carving of a workspace
struct Carve {
    char* base;
    size_t used = 0;
    void* take(size_t n) {
        void* p = base ? base + used : nullptr;
        used += align_up(n, 256);
        return p;
    }
};

// ---- the products' plans
TileProduct forward_plan(int N, int M, int S) {
    TileProduct g = {};
    g.R = N; g.C = S; g.chunks = up8(M) / 8;
    g.stages = g.part = (g.chunks + 7) / 8;
    tile_plan(g, true);
    return g;
}
TileProduct rows_plan(int N, int M, int S) {
    TileProduct g = {};
    g.R = N; g.C = M; g.chunks = 2 * up64(S) / 8; g.klen = S;
    g.part = up64(S) / 64; g.stages = 2 * g.part;
    tile_plan(g, false);
    return g;
}
TileProduct weights_plan(int N, int M, int S) {
    TileProduct g = {};
    g.R = 2 * up64(S); g.C = M; g.klen = N;
    g.part = g.stages = (N + 63) / 64;
    tile_plan(g, false);
    return g;
}

struct ForwardWs { void *X, *Wg, *Wu, *partial; float* gu; size_t total; };
ForwardWs forward_ws(fw_dtype dt, int N, int M, int S, void* ws) {
    Carve c = {reinterpret_cast<char*>(ws)};
    ForwardWs w = {};
    if (dt == FW_F32) {
        w.gu = reinterpret_cast<float*>(c.take(2 * (size_t)N * S * 4));
    } else {
        if (M % 8) {
            w.X = c.take((size_t)N * up8(M) * 2);
            w.Wg = c.take((size_t)S * up8(M) * 2);
            w.Wu = c.take((size_t)S * up8(M) * 2);
        }
        w.partial = c.take(tile_partial_bytes(forward_plan(N, M, S)));
    }
    w.total = c.used;
    return w;
}
struct GradWs { void *D, *X, *Wg, *Wu, *partial; float *part, *sums, *Wt, *Dt, *Xt; size_t total; };
GradWs grad_ws(fw_dtype dt, int N, int M, int S, void* ws) {
    Carve c = {reinterpret_cast<char*>(ws)};
    GradWs w = {};
    const size_t Sp = up64(S);
    w.D = c.take((size_t)N * 2 * Sp * (dt == FW_BF16 ? 2 : 4));
    w.part = reinterpret_cast<float*>(c.take((size_t)row_blocks(N) * 2 * Sp * 4));
    w.sums = reinterpret_cast<float*>(c.take(2 * Sp * 4));
    if (dt == FW_F32) {
        w.Wt = reinterpret_cast<float*>(c.take((size_t)M * 2 * Sp * 4));
        w.Dt = reinterpret_cast<float*>(c.take((size_t)N * 2 * Sp * 4));
        w.Xt = reinterpret_cast<float*>(c.take((size_t)N * M * 4));
    } else {
        if (M % 8) {
            w.X = c.take((size_t)N * up8(M) * 2);
            w.Wg = c.take((size_t)S * up8(M) * 2);
            w.Wu = c.take((size_t)S * up8(M) * 2);
        }
        const size_t a = tile_partial_bytes(rows_plan(N, M, S)), b = tile_partial_bytes(weights_plan(N, M, S));
        w.partial = c.take(a > b ? a : b);
    }
    w.total = c.used;
    return w;
}

fw_status forward_f32(const float* X, int N, int M, int S, const float* Wg, const float* Wu, const float* bg, const float* bu, fw_act act,
                      float* H, float* Z, void* ws, hipStream_t st) {
    const size_t n = (size_t)N * S;
    float* gu = forward_ws(FW_F32, N, M, S, ws).gu;
    for (int k = 0; k < 2; ++k) {
        GemmEpilogue e = {};
        e.out = gu + k * n; e.taps = 1;
        const fw_status rc = gemm_planes(X, false, N, S, M, k ? Wu : Wg, e, false, st);
        if (rc != FW_OK) return rc;
    }
    hipLaunchKernelGGL(gate_kernel, dim3(blocks_for(n)), dim3(256), 0, st, gu, n, S, bg, bu, (int)act, H, Z);
    FW_LAUNCH_CHECK();
    return FW_OK;
}

fw_status forward_bf16(const void* X, int N, int M, int S, const void* Wg, const void* Wu, const float* bg, const float* bu, fw_act act,
                       void* H, float* Z, void* ws, hipStream_t st) {
    const ForwardWs w = forward_ws(FW_BF16, N, M, S, ws);
    if (M % 8) {             // 16-byte loads need aligned rows
        fw_status rc = pad_rows(X, N, M, w.X, st);
        if (rc == FW_OK) rc = pad_rows(Wg, S, M, w.Wg, st);
        if (rc == FW_OK) rc = pad_rows(Wu, S, M, w.Wu, st);
        if (rc != FW_OK) return rc;
        X = w.X; Wg = w.Wg; Wu = w.Wu;
    }
    TileProduct g = forward_plan(N, M, S);
    g.a = bytes(X); g.b0 = bytes(Wg); g.b1 = bytes(Wu);
    g.apitch = g.bpitch = 2ll * up8(M);
    g.partial = w.partial;
    return tile_product<false, false, false, true>(g, GateEpilogue{reinterpret_cast<__bf16*>(H), Z, bg, bu, N, S, (int)act}, st);
}

template <class T>
fw_status gate_grad(const T* dH, const float* Z, int N, int S, const GradWs& w, bool sums, T* dbg, T* dbu, hipStream_t st) {
    const int Sp = up64(S);
    hipLaunchKernelGGL(gate_grad_kernel<T>, dim3((Sp + 255) / 256, row_blocks(N)), dim3(256), 0, st, dH, Z, N, S, Sp, reinterpret_cast<T*>(w.D),
                       sums ? w.part : nullptr);
    FW_LAUNCH_CHECK();
    if (!sums) return FW_OK;
    hipLaunchKernelGGL(bias_grad_kernel<T>, dim3((2 * Sp + 63) / 64), dim3(1024), 0, st, w.part, row_blocks(N), S, Sp, w.sums, dbg, dbu);
    FW_LAUNCH_CHECK();
    return FW_OK;
}

fw_status grad_f32(const float* X, int N, int M, int S, const float* Wg, const float* Wu, const float* Z, const float* dH, const float* mu,
                   float* dX, float* dWg, float* dWu, float* dbg, float* dbu, void* ws, hipStream_t st) {
    const GradWs w = grad_ws(FW_F32, N, M, S, ws);
    const int Sp = up64(S);
    float* D = reinterpret_cast<float*>(w.D);
    fw_status rc = gate_grad<float>(dH, Z, N, S, w, dbg != nullptr, dbg, dbu, st);
    if (rc != FW_OK) return rc;
    GemmEpilogue e = {};
    e.taps = 1;
    if (dX) {
        rc = transpose(Wg, S, M, M, nullptr, w.Wt, 2 * (size_t)Sp, 0, Sp, st);
        if (rc == FW_OK) rc = transpose(Wu, S, M, M, nullptr, w.Wt, 2 * (size_t)Sp, Sp, Sp, st);
        e.out = dX;
        if (rc == FW_OK) rc = gemm_planes(D, false, N, M, 2 * Sp, w.Wt, e, false, st);
        if (rc != FW_OK) return rc;
    }
    if (dWg) {
        rc = transpose(X, N, M, M, mu, w.Xt, (size_t)N, 0, N, st);
        if (rc == FW_OK) rc = transpose(D, N, 2 * Sp, 2 * Sp, nullptr, w.Dt, (size_t)N, 0, N, st);
        for (int k = 0; k < 2 && rc == FW_OK; ++k) {
            e.out = k ? dWu : dWg;
            rc = gemm_planes(w.Dt + (size_t)k * Sp * N, false, S, M, N, w.Xt, e, false, st);
        }
    }
    return rc;
}

fw_status grad_bf16(const void* X, int N, int M, int S, const void* Wg, const void* Wu, const float* Z, const __bf16* dH, const float* mu,
                    __bf16* dX, __bf16* dWg, __bf16* dWu, __bf16* dbg, __bf16* dbu, void* ws, hipStream_t st) {
    const GradWs w = grad_ws(FW_BF16, N, M, S, ws);
    const int Sp = up64(S);
    fw_status rc = gate_grad<__bf16>(dH, Z, N, S, w, dbg || (mu && dWg), dbg, dbu, st);
    if (rc != FW_OK) return rc;
    if (M % 8 && dX) {
        rc = pad_rows(Wg, S, M, w.Wg, st);
        if (rc == FW_OK) rc = pad_rows(Wu, S, M, w.Wu, st);
        if (rc != FW_OK) return rc;
        Wg = w.Wg; Wu = w.Wu;
    }
    if (dX) {
        TileProduct g = rows_plan(N, M, S);
        g.a = bytes(w.D); g.b0 = bytes(Wg); g.b1 = bytes(Wu);
        g.apitch = 4ll * Sp; g.bpitch = 2ll * up8(M);
        g.partial = w.partial;
        rc = tile_product<false, false, true, false>(g, RowsEpilogue{dX, N, M}, st);
        if (rc != FW_OK) return rc;
    }
    if (dWg) {
        if (M % 8) {
            rc = pad_rows(X, N, M, w.X, st);
            if (rc != FW_OK) return rc;
            X = w.X;
        }
        TileProduct g = weights_plan(N, M, S);
        g.a = bytes(w.D); g.b0 = g.b1 = bytes(X);
        g.apitch = 4ll * Sp; g.bpitch = 2ll * up8(M);
        g.partial = w.partial;
        rc = tile_product<false, true, true, false>(g, WeightsEpilogue{dWg, dWu, w.sums, mu, S, Sp, M}, st);
    }
    return rc;
}

}  // namespace

size_t gated_forward_workspace_bytes(fw_dtype dt, int N, int M, int S) { return forward_ws(dt, N, M, S, nullptr).total; }
size_t gated_grad_workspace_bytes(fw_dtype dt, int N, int M, int S) { return grad_ws(dt, N, M, S, nullptr).total; }

fw_status gated_forward(const void* X, fw_dtype dt, int N, int M, int S, const void* Wg, const void* Wu, const float* bg, const float* bu,
                        fw_act act, void* H, float* Z, void* ws, hipStream_t st) {
    if (dt == FW_BF16) return forward_bf16(X, N, M, S, Wg, Wu, bg, bu, act, H, Z, ws, st);
    return forward_f32((const float*)X, N, M, S, (const float*)Wg, (const float*)Wu, bg, bu, act, (float*)H, Z, ws, st);
}

fw_status gated_grad(const void* X, fw_dtype dt, int N, int M, int S, const void* Wg, const void* Wu, const float* Z, const void* dH,
                     const float* mu, void* dX, void* dWg, void* dWu, void* dbg, void* dbu, void* ws, hipStream_t st) {
    if (dt == FW_BF16)
        return grad_bf16(X, N, M, S, Wg, Wu, Z, (const __bf16*)dH, mu, (__bf16*)dX, (__bf16*)dWg, (__bf16*)dWu, (__bf16*)dbg, (__bf16*)dbu, ws, st);
    return grad_f32((const float*)X, N, M, S, (const float*)Wg, (const float*)Wu, Z, (const float*)dH, mu, (float*)dX, (float*)dWg, (float*)dWu,
                    (float*)dbg, (float*)dbu, ws, st);
}

}  // namespace fw
