// Gated feed-forward block and its gradient:
//   g = X Wg^T + bg,  u = X Wu^T + bu,  H = act(g) u;      kept for the backward pass: Z[0] = u act'(g), Z[1] = act(g)
//   dg = dH Z[0],  du = dH Z[1],   dX = dg Wg + du Wu,   dWg = dg^T (X - 1 mu^T),  dWu = du^T (X - 1 mu^T),  db = column sums
//
// bfloat16: both projections in one launch, the panel of weights holding the same columns of Wg and Wu, so that a lane has g and u of
// an element in its registers when the sums are done (tile_product.h).  The backward pass forms D = [dg | du] once, rounded to
// bfloat16 (small N S: to two bfloat16 numbers, see two_planes), [N][2 Sp] with Sp = S rounded up to 64 and zeros between, and takes two products of it: dX = D [Wg; Wu], whose contraction runs
// over the rows of both weight matrices, and [dWg; dWu] = D^T X.  Operands that are contraction-major in memory are turned on the
// way out of LDS, not in memory.  mu is taken out of the sums: D^T (X - 1 mu^T) = D^T X - (D^T 1) mu^T, with D^T 1 summed from the
// rounded D, so that the identity is exact but for float32 sums.
// float32: the same products with every operand as three bfloat16 planes (tile_product.h), split in one pass over X and the weights, D
// when it is formed.  X is centred on mu as it is split.
// float32 with few rows: float32 matrix instructions on the operands as they are (few_product_kernel), one row without them.
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
        const float c = fminf(fmaxf(g, -64.f), 64.f);        // p (1 - p) is zero beyond; g^2 may be infinite
        da = p + 2.f * c * p * (1.f - p) * k * (1.f + 0.134145f * c * c);
    } else {
        a = g <= 0.f ? 0.f : g;               // NaN stays NaN
        da = g <= 0.f ? 0.f : g > 0.f ? 1.f : g;
    }
}
template <class F> __device__ __forceinline__ void with_activation(int act, const F& f) {
    if (act == FW_ACT_SILU) f(std::integral_constant<int, FW_ACT_SILU>());
    else if (act == FW_ACT_GELU) f(std::integral_constant<int, FW_ACT_GELU>());
    else if (act == FW_ACT_GELU_TANH) f(std::integral_constant<int, FW_ACT_GELU_TANH>());
    else f(std::integral_constant<int, FW_ACT_RELU>());
}

// ---- epilogues: four entries of a row.  FIX (operands in planes: an infinite number has none): entries that are not finite are computed
// once more, in float32.
__device__ __forceinline__ bool all_finite(const floatx4& v) {
    return fabsf(v[0]) <= 3.402823466e38f && fabsf(v[1]) <= 3.402823466e38f && fabsf(v[2]) <= 3.402823466e38f && fabsf(v[3]) <= 3.402823466e38f;
}
template <class T, bool FIX> struct GateEpilogue {
    T* H;
    float* Z;
    const float *bg, *bu;
    int N, S, act;
    const float *X, *Wg, *Wu;             // FIX: the operands as they were
    int M;
    __device__ __noinline__ float dot(int n, int s, bool up) const {
        const float *x = X + (size_t)n * M, *w = (up ? Wu : Wg) + (size_t)s * M;
        float v = 0.f;
        for (int m = 0; m < M; ++m) v = fmaf(x[m], w[m], v);
        return v;
    }
    __device__ __forceinline__ void apply(int n, int s, floatx4 gate, floatx4 up) const {
        if (n >= N || s >= S) return;
        if (FIX && !(all_finite(gate) && all_finite(up))) {
            for (int i = 0; i < 4 && s + i < S; ++i) { gate[i] = dot(n, s + i, false); up[i] = dot(n, s + i, true); }
        }
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
// what the gradients are computed from once more
template <class T> struct GradInputs { const T *X, *Wg, *Wu; const float* Z; const T* dH; const float* mu; int N, M, S; };
template <class T, bool FIX> struct RowsEpilogue {           // dX
    T* out;
    int N, M;
    GradInputs<T> in;
    __device__ __noinline__ float dot(int n, int m) const {
        float v = 0.f;
        for (int s = 0; s < in.S; ++s) {
            const size_t e = (size_t)n * in.S + s, w = (size_t)s * M + m;
            v = fmaf((float)in.dH[e] * in.Z[e], (float)in.Wg[w], v);
            v = fmaf((float)in.dH[e] * in.Z[(size_t)N * in.S + e], (float)in.Wu[w], v);
        }
        return v;
    }
    __device__ __forceinline__ void apply(int n, int m, floatx4 acc) const {
        if (n >= N || m >= M) return;
        if (FIX && !all_finite(acc))
            for (int i = 0; i < 4 && m + i < M; ++i) acc[i] = dot(n, m + i);
        const float v[4] = {acc[0], acc[1], acc[2], acc[3]};
        tile_store(out + (size_t)n * M + m, m, M, v);
    }
};
template <class T, bool FIX> struct WeightsEpilogue {        // rows below Sp are the gate's, the others the up projection's
    T *dWg, *dWu;
    const float *sums, *mu;               // mu: taken out here (bfloat16), or null
    int S, Sp, M;
    GradInputs<T> in;
    __device__ __noinline__ float dot(int s, bool up, int m) const {
        const float c = in.mu ? in.mu[m] : 0.f;
        float v = 0.f;
        for (int n = 0; n < in.N; ++n) {
            const size_t e = (size_t)n * S + s;
            v = fmaf((float)in.dH[e] * in.Z[(up ? (size_t)in.N * S : 0) + e], (float)in.X[(size_t)n * M + m] - c, v);
        }
        return v;
    }
    __device__ __forceinline__ void apply(int r, int m, floatx4 acc) const {
        const int s = r >= Sp ? r - Sp : r;
        if (s >= S || m >= M) return;
        const bool again = FIX && !all_finite(acc);
        if (again)
            for (int i = 0; i < 4 && m + i < M; ++i) acc[i] = dot(s, r >= Sp, m + i);
        float v[4] = {acc[0], acc[1], acc[2], acc[3]};
        if (mu && !again) {
            const float d = sums[r];
            float c[4];
            tile_vector(mu, m, M, c);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] -= d * c[i];
        }
        tile_store((r >= Sp ? dWu : dWg) + (size_t)s * M + m, m, M, v);
    }
};

// float32, one row: a wavefront takes the two weight rows of an output.  Bound by the one read of the weights (4172
// features to 7040: 48.0 us, 4.9 TB/s; on the matrix cores as for more rows 55.6).
__global__ __launch_bounds__(256) void one_row_kernel(const float* __restrict__ X, int M, int S, const float* __restrict__ Wg,
                                                      const float* __restrict__ Wu, GateEpilogue<float, false> epi) {
    const int lane = threadIdx.x & 63, s = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (s >= S) return;
    const float *wg = Wg + (size_t)s * M, *wu = Wu + (size_t)s * M;
    float g = 0.f, u = 0.f;
    const int whole = M / 256 * 256;
#pragma unroll 2
    for (int m = 4 * lane; m < whole; m += 256) {
        float4 a, b, x;
        __builtin_memcpy(&a, wg + m, 16);
        __builtin_memcpy(&b, wu + m, 16);
        __builtin_memcpy(&x, X + m, 16);
        g = fmaf(x.x, a.x, fmaf(x.y, a.y, fmaf(x.z, a.z, fmaf(x.w, a.w, g))));
        u = fmaf(x.x, b.x, fmaf(x.y, b.y, fmaf(x.z, b.z, fmaf(x.w, b.w, u))));
    }
    for (int m = whole + lane; m < M; m += 64) {
        g = fmaf(X[m], wg[m], g);
        u = fmaf(X[m], wu[m], u);
    }
    g = wave_sum(g); u = wave_sum(u);
    if (lane) return;
    with_activation(epi.act, [&](auto ACT) {
        float a, da;
        activation<decltype(ACT)::value>(g + (epi.bg ? epi.bg[s] : 0.f), a, da);
        u += epi.bu ? epi.bu[s] : 0.f;
        epi.H[s] = a * u;
        if (epi.Z) { epi.Z[s] = u * da; epi.Z[(size_t)S + s] = a; }
    });
}

// ---- elementwise passes

// three bfloat16 planes of a float32 number
__device__ __forceinline__ void planes_of(float x, __bf16& h, __bf16& m, __bf16& l) {
    h = (__bf16)x;
    const float r = x - (float)h;
    m = (__bf16)r;
    l = (__bf16)(r - (float)m);
}

// float32 matrices to planes [3][Rp][Mp], zeros past R and M; mu: taken out of the rows, or null.  The matrix goes by blockIdx.y.
struct Split { const float* in[3]; __bf16* out[3]; int R[3], Rp[3]; const float* mu[3]; };
__global__ __launch_bounds__(256) void split_planes_kernel(Split s, int M, int Mp) {
    const int k = blockIdx.y, c8 = Mp / 8, R = s.R[k];
    const size_t n8 = (size_t)s.Rp[k] * c8, plane = n8 * 8;
    const float* mu = s.mu[k];
    for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < n8; e += (size_t)gridDim.x * 256) {
        const size_t r = e / c8;
        const int m = 8 * (int)(e - r * c8);
        float x[8];
        const float* p = s.in[k] + r * M + m;
        if (r < R && m + 8 <= M) {
            __builtin_memcpy(x, p, 32);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = r < R && m + i < M ? p[i] : 0.f;
        }
        bf16x8 h, mm, l;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __bf16 a, b, c;
            planes_of(mu && r < R && m + i < M ? x[i] - mu[m + i] : x[i], a, b, c);
            h[i] = a; mm[i] = b; l[i] = c;
        }
        bf16x8* o = reinterpret_cast<bf16x8*>(s.out[k]) + e;
        o[0] = h;
        o[plane / 8] = mm;
        o[plane / 4] = l;
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
// D[n] = [dg | du] of row n, each Sp wide (zeros past S), as P planes [P][Np][2 Sp] (float32: three, zeros past N).  A workgroup has 256 columns
// and `rows` rows, a wavefront a quarter of these, four at a time (their loads go out together).
// part[block of rows][4][Sp] or null: sums over the block's rows of dg and du as they are (for the biases) and as rounded (for mu).
template <class T, int P>
__global__ __launch_bounds__(256) void gate_grad_kernel(const T* __restrict__ dH, const float* __restrict__ Z, int N, int Np, int S, int Sp,
                                                        int rows, __bf16* __restrict__ D, float* __restrict__ part) {
    __shared__ float red[4][4][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int s = blockIdx.x * 256 + 4 * lane;
    const int n0 = blockIdx.y * rows + wave * (rows / 4), end = P == 3 ? Np : N, n1 = min(n0 + rows / 4, end);
    float sum[4][4] = {};
    auto put = [&](__bf16* d, const float (&x)[4], float (&exact)[4], float (&rounded)[4]) __attribute__((always_inline)) {
        bf16x4 h, m, l;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __bf16 a, b, c;
            planes_of(x[i], a, b, c);
            h[i] = a; m[i] = b; l[i] = c;
            exact[i] += x[i];
            rounded[i] += P == 2 ? (float)a + (float)b : (float)a;
        }
        *reinterpret_cast<bf16x4*>(d) = h;
        const size_t plane = (size_t)Np * 2 * Sp;
        if (P > 1) *reinterpret_cast<bf16x4*>(d + plane) = m;
        if (P > 2) *reinterpret_cast<bf16x4*>(d + 2 * plane) = l;
    };
    auto rows_at = [&](auto WHOLE, int n) __attribute__((always_inline)) {       // WHOLE: four columns and four rows, all there
        float h[4][4], p[4][4], q[4][4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const size_t e = (size_t)(n + r) * S + s;
            if constexpr (decltype(WHOLE)::value) {
                load4(dH + e, h[r]);
                load4(Z + e, p[r]);
                load4(Z + (size_t)N * S + e, q[r]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool in = n + r < N && s + i < S;
                    h[r][i] = in ? (float)dH[e + i] : 0.f;
                    p[r][i] = in ? Z[e + i] : 0.f;
                    q[r][i] = in ? Z[(size_t)N * S + e + i] : 0.f;
                }
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (!decltype(WHOLE)::value && n + r >= n1) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) { p[r][i] *= h[r][i]; q[r][i] *= h[r][i]; }
            __bf16* d = D + (size_t)(n + r) * 2 * Sp + s;
            put(d, p[r], sum[0], sum[2]);
            put(d + Sp, q[r], sum[1], sum[3]);
        }
    };
    if (s < Sp) {
        for (int n = n0; n < n1; n += 4) {
            if (s + 4 <= S && n + 4 <= min(n1, N)) rows_at(std::true_type(), n);
            else rows_at(std::false_type(), n);
        }
    }
    if (!part) return;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[wave][k][4 * lane + i] = sum[k][i];
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < Sp) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            part[((size_t)blockIdx.y * 4 + k) * Sp + c] =
                red[0][k][threadIdx.x] + red[1][k][threadIdx.x] + red[2][k][threadIdx.x] + red[3][k][threadIdx.x];
    }
}

// sums[c] = the blocks' partial sums, in a fixed order: of dg and du for the biases' gradients, of their rounded values for mu
template <class T>
__global__ __launch_bounds__(1024) void bias_grad_kernel(const float* __restrict__ part, int blocks, int S, int Sp, float* __restrict__ sums,
                                                         T* __restrict__ dbg, T* __restrict__ dbu) {
    __shared__ float red[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;    // Sp is a multiple of 64
    const bool rounded = c >= 2 * Sp;
    if (!rounded && !dbg) return;                                                   // the whole workgroup
    float v = 0.f;
    for (int p = slice; p < blocks; p += 16) v += part[(size_t)p * 4 * Sp + c];
    red[slice][threadIdx.x & 63] = v;
    __syncthreads();
    if (slice) return;
    v = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += red[i][threadIdx.x];
    if (rounded) sums[c - 2 * Sp] = v;
    else if (c % Sp < S) (c >= Sp ? dbu : dbg)[c % Sp] = (T)v;
}

// matrices of M bfloat16 columns to rows of Mp (a multiple of 8), zeros behind; the matrix goes by blockIdx.y
struct Pad { const __bf16* in[3]; bf16x8* out[3]; int R[3]; };
__global__ __launch_bounds__(256) void pad_rows_kernel(Pad s, int M, int Mp) {
    const int k = blockIdx.y, c8 = Mp / 8;
    const size_t n8 = (size_t)s.R[k] * c8;
    for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < n8; e += (size_t)gridDim.x * 256) {
        const size_t r = e / c8;
        const int m = 8 * (int)(e - r * c8);
        const __bf16* p = s.in[k] + r * M + m;
        bf16x8 v;
        if (m + 8 <= M) {
            __builtin_memcpy(&v, p, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = m + i < M ? p[i] : (__bf16)0.f;
        }
        s.out[k][e] = v;
    }
}

// Up to 64 rows float32 products are bound by the one read of the weights or nearly so; in planes these are written and read again (4172
// features to 7040, 17 rows: 202 us against 68.6, 64 rows: 204 against 118, 86 rows: 215 against 200, 128 rows of 1153 to 1001: 27 against 37).
constexpr int FEW_F32 = 64;

inline unsigned blocks_for(size_t n) { return (unsigned)((n + 255) / 256 < 16384 ? (n + 255) / 256 : 16384); }
inline int up8(int m) { return (m + 7) / 8 * 8; }
inline int up64(int s) { return (s + 63) / 64 * 64; }
// bfloat16: D in two planes, 16 bits, where the rounding to 8 bits does not average out: it adds an error as large as that of rounding the
// result, 1.42 times the latter together, but up to 1.8 times where a few entries make up the sum (11 x 64, S = 64).  The products then
// go over the weights twice; small ones are bound by their launches.
inline bool two_planes(fw_dtype dt, int N, int S) { return dt == FW_BF16 && (long long)N * S <= 1 << 19; }
// rows of a workgroup of gate_grad_kernel: 64, or 16 where that leaves compute units without work (777 x 1001: 13.9 us with 64)
inline int grad_rows(int N, int S) { return (long long)((N + 63) / 64) * ((S + 255) / 256) >= 1024 ? 64 : 16; }
inline int row_blocks(int N, int S) { return (up64(N) + grad_rows(N, S) - 1) / grad_rows(N, S); }
inline const char* bytes(const void* p) { return reinterpret_cast<const char*>(p); }

struct PadList {
    Pad s = {};
    int n = 0, rows = 0;
    void add(const void* in, int R, void* out) {
        s.in[n] = reinterpret_cast<const __bf16*>(in);
        s.out[n] = reinterpret_cast<bf16x8*>(out);
        s.R[n++] = R;
        rows = R > rows ? R : rows;
    }
    fw_status launch(int M, hipStream_t st) const {
        if (!n) return FW_OK;
        hipLaunchKernelGGL(pad_rows_kernel, dim3(blocks_for((size_t)rows * (up8(M) / 8)), n), dim3(256), 0, st, s, M, up8(M));
        FW_LAUNCH_CHECK();
        return FW_OK;
    }
};
fw_status split_planes(const Split& s, int matrices, int M, hipStream_t st) {
    int rows = 0;
    for (int k = 0; k < matrices; ++k) rows = s.Rp[k] > rows ? s.Rp[k] : rows;
    hipLaunchKernelGGL(split_planes_kernel, dim3(blocks_for((size_t)rows * (up64(M) / 8)), matrices), dim3(256), 0, st, s, M, up64(M));
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

// ---- the products' plans; float32 (planes): over padded operands
TileProduct forward_plan(fw_dtype dt, int N, int M, int S) {
    TileProduct g = {};
    g.R = N; g.C = S; g.chunks = up8(M) / 8;
    g.stages = g.once = g.part = (g.chunks + 7) / 8;
    tile_plan(g, true, dt == FW_F32, dt == FW_F32 ? 6 : 5);         // of two sums an entry of H and two of Z
    return g;
}
TileProduct rows_plan(fw_dtype dt, int N, int M, int S) {
    TileProduct g = {};
    g.R = N; g.C = M; g.chunks = 2 * up64(S) / 8; g.klen = S;
    g.part = up64(S) / 64; g.once = 2 * g.part; g.stages = two_planes(dt, N, S) ? 2 * g.once : g.once;
    tile_plan(g, false, dt == FW_F32, dt == FW_F32 ? 4 : 2);
    return g;
}
TileProduct weights_plan(fw_dtype dt, int N, int M, int S) {
    TileProduct g = {};
    g.R = 2 * up64(S); g.C = M; g.klen = N;
    g.part = g.once = (N + 63) / 64; g.stages = two_planes(dt, N, S) ? 2 * g.once : g.once;
    tile_plan(g, false, dt == FW_F32, dt == FW_F32 ? 4 : 2);
    return g;
}

size_t plane3_bytes(int R, int M) { return 6 * (size_t)R * up64(M); }
struct ForwardWs { void *X, *Wg, *Wu, *partial; size_t total; };
ForwardWs forward_ws(fw_dtype dt, int N, int M, int S, void* ws) {
    Carve c = {reinterpret_cast<char*>(ws)};
    ForwardWs w = {};
    if (dt == FW_F32) {
        if (N > FEW_F32) {
            w.X = c.take(plane3_bytes(N, M));
            w.Wg = c.take(plane3_bytes(S, M));
            w.Wu = c.take(plane3_bytes(S, M));
        }
    } else if (M % 8 && N > TILE_FEW) {
        w.X = c.take((size_t)N * up8(M) * 2);
        w.Wg = c.take((size_t)S * up8(M) * 2);
        w.Wu = c.take((size_t)S * up8(M) * 2);
    }
    if (N > (dt == FW_BF16 ? TILE_FEW : FEW_F32)) w.partial = c.take(tile_partial_bytes(forward_plan(dt, N, M, S)));
    w.total = c.used;
    return w;
}
struct GradWs { void *D, *X, *Wg, *Wu, *partial; float *part, *sums; size_t total; };
GradWs grad_ws(fw_dtype dt, int N, int M, int S, void* ws) {
    Carve c = {reinterpret_cast<char*>(ws)};
    GradWs w = {};
    const size_t Sp = up64(S);
    w.D = c.take(dt == FW_F32 ? plane3_bytes(up64(N), 2 * (int)Sp) : (size_t)N * 2 * Sp * (two_planes(dt, N, S) ? 4 : 2));
    w.part = reinterpret_cast<float*>(c.take((size_t)row_blocks(N, S) * 4 * Sp * 4));
    w.sums = reinterpret_cast<float*>(c.take(2 * Sp * 4));
    if (dt == FW_F32) {
        w.X = c.take(plane3_bytes(up64(N), M));
        w.Wg = c.take(plane3_bytes((int)Sp, M));
        w.Wu = c.take(plane3_bytes((int)Sp, M));
    } else if (M % 8) {
        w.X = c.take((size_t)N * up8(M) * 2);
        w.Wg = c.take((size_t)S * up8(M) * 2);
        w.Wu = c.take((size_t)S * up8(M) * 2);
    }
    const size_t a = tile_partial_bytes(rows_plan(dt, N, M, S)), b = tile_partial_bytes(weights_plan(dt, N, M, S));
    w.partial = c.take(a > b ? a : b);
    w.total = c.used;
    return w;
}

fw_status forward_f32(const float* X, int N, int M, int S, const float* Wg, const float* Wu, const float* bg, const float* bu, fw_act act,
                      float* H, float* Z, void* ws, hipStream_t st) {
    const ForwardWs w = forward_ws(FW_F32, N, M, S, ws);
    if (N <= FEW_F32) {
        const GateEpilogue<float, false> epi = {H, Z, bg, bu, N, S, (int)act};
        const FewProduct few = {bytes(X), bytes(Wg), bytes(Wu), N, S, 4 * M};
        if (N > 32) return few_product<TILE_F32, true, 4>(few, epi, st);
        if (N > 16) return few_product<TILE_F32, true, 2>(few, epi, st);
        if (N > 1) return few_product<TILE_F32, true, 1>(few, epi, st);
        hipLaunchKernelGGL(one_row_kernel, dim3((S + 3) / 4), dim3(256), 0, st, X, M, S, Wg, Wu, epi);
        FW_LAUNCH_CHECK();
        return FW_OK;
    }
    const GateEpilogue<float, true> epi = {H, Z, bg, bu, N, S, (int)act, X, Wg, Wu, M};
    const Split s = {{X, Wg, Wu}, {(__bf16*)w.X, (__bf16*)w.Wg, (__bf16*)w.Wu}, {N, S, S}, {N, S, S}, {}};
    const fw_status rc = split_planes(s, 3, M, st);
    if (rc != FW_OK) return rc;
    TileProduct g = forward_plan(FW_F32, N, M, S);
    g.a = bytes(w.X); g.b0 = bytes(w.Wg); g.b1 = bytes(w.Wu);
    g.apitch = g.bpitch = 2ll * up64(M);
    g.aplane = N * g.apitch; g.bplane = S * g.bpitch;
    g.partial = w.partial;
    return tile_product<TILE_PLANES, false, false, true>(g, epi, st);
}

fw_status forward_bf16(const void* X, int N, int M, int S, const void* Wg, const void* Wu, const float* bg, const float* bu, fw_act act,
                       void* H, float* Z, void* ws, hipStream_t st) {
    const ForwardWs w = forward_ws(FW_BF16, N, M, S, ws);
    const GateEpilogue<__bf16, false> epi = {reinterpret_cast<__bf16*>(H), Z, bg, bu, N, S, (int)act};
    if (N <= TILE_FEW) return few_product<TILE_BF16, true>({bytes(X), bytes(Wg), bytes(Wu), N, S, 2 * M}, epi, st);
    if (M % 8) {             // 16-byte loads need aligned rows
        PadList pads;
        pads.add(X, N, w.X);
        pads.add(Wg, S, w.Wg);
        pads.add(Wu, S, w.Wu);
        const fw_status rc = pads.launch(M, st);
        if (rc != FW_OK) return rc;
        X = w.X; Wg = w.Wg; Wu = w.Wu;
    }
    TileProduct g = forward_plan(FW_BF16, N, M, S);
    g.a = bytes(X); g.b0 = bytes(Wg); g.b1 = bytes(Wu);
    g.apitch = g.bpitch = 2ll * up8(M);
    g.partial = w.partial;
    return tile_product<TILE_BF16, false, false, true>(g, epi, st);
}

template <class T>
fw_status gate_grad(const T* dH, const float* Z, int N, int S, const GradWs& w, bool rounded, T* dbg, T* dbu, hipStream_t st) {
    const int Sp = up64(S);
    const bool sums = rounded || dbg;
    const auto launch = [&](auto P) {
        hipLaunchKernelGGL((gate_grad_kernel<T, decltype(P)::value>), dim3((Sp + 255) / 256, row_blocks(N, S)), dim3(256), 0, st, dH, Z, N,
                           decltype(P)::value == 3 ? up64(N) : N, S, Sp, grad_rows(N, S), reinterpret_cast<__bf16*>(w.D), sums ? w.part : nullptr);
    };
    if constexpr (std::is_same<T, float>::value) launch(std::integral_constant<int, 3>());
    else if (two_planes(FW_BF16, N, S)) launch(std::integral_constant<int, 2>());
    else launch(std::integral_constant<int, 1>());
    FW_LAUNCH_CHECK();
    if (!sums) return FW_OK;
    hipLaunchKernelGGL(bias_grad_kernel<T>, dim3((rounded ? 4 : 2) * Sp / 64), dim3(1024), 0, st, w.part, row_blocks(N, S), S, Sp, w.sums, dbg, dbu);
    FW_LAUNCH_CHECK();
    return FW_OK;
}

fw_status grad_f32(const float* X, int N, int M, int S, const float* Wg, const float* Wu, const float* Z, const float* dH, const float* mu,
                   float* dX, float* dWg, float* dWu, float* dbg, float* dbu, void* ws, hipStream_t st) {
    const GradWs w = grad_ws(FW_F32, N, M, S, ws);
    const int Sp = up64(S), Np = up64(N);
    fw_status rc = gate_grad<float>(dH, Z, N, S, w, false, dbg, dbu, st);
    if (rc != FW_OK) return rc;
    const GradInputs<float> in = {X, Wg, Wu, Z, dH, mu, N, M, S};
    Split s = {};
    int k = 0;
    const auto add = [&](const float* p, void* out, int R, int Rp, const float* c) { s.in[k] = p; s.out[k] = (__bf16*)out; s.R[k] = R; s.Rp[k] = Rp; s.mu[k++] = c; };
    if (dWg) add(X, w.X, N, Np, mu);
    if (dX) { add(Wg, w.Wg, S, Sp, nullptr); add(Wu, w.Wu, S, Sp, nullptr); }
    if (k) rc = split_planes(s, k, M, st);
    if (rc != FW_OK) return rc;
    if (dX) {
        TileProduct g = rows_plan(FW_F32, N, M, S);
        g.a = bytes(w.D); g.b0 = bytes(w.Wg); g.b1 = bytes(w.Wu);
        g.apitch = 4ll * Sp; g.bpitch = 2ll * up64(M);
        g.aplane = Np * g.apitch; g.bplane = Sp * g.bpitch;
        g.partial = w.partial;
        rc = tile_product<TILE_PLANES, false, true, false>(g, RowsEpilogue<float, true>{dX, N, M, in}, st);
        if (rc != FW_OK) return rc;
    }
    if (dWg) {
        TileProduct g = weights_plan(FW_F32, N, M, S);
        g.a = bytes(w.D); g.b0 = g.b1 = bytes(w.X);
        g.apitch = 4ll * Sp; g.bpitch = 2ll * up64(M);
        g.aplane = Np * g.apitch; g.bplane = Np * g.bpitch;
        g.partial = w.partial;
        rc = tile_product<TILE_PLANES, true, true, false>(g, WeightsEpilogue<float, true>{dWg, dWu, nullptr, nullptr, S, Sp, M, in}, st);
    }
    return rc;
}

fw_status grad_bf16(const void* X, int N, int M, int S, const void* Wg, const void* Wu, const float* Z, const __bf16* dH, const float* mu,
                    __bf16* dX, __bf16* dWg, __bf16* dWu, __bf16* dbg, __bf16* dbu, void* ws, hipStream_t st) {
    const GradWs w = grad_ws(FW_BF16, N, M, S, ws);
    const int Sp = up64(S);
    const bool two = two_planes(FW_BF16, N, S);
    const GradInputs<__bf16> in = {(const __bf16*)X, (const __bf16*)Wg, (const __bf16*)Wu, Z, dH, mu, N, M, S};       // as they came, not padded
    fw_status rc = gate_grad<__bf16>(dH, Z, N, S, w, mu && dWg, dbg, dbu, st);
    if (rc != FW_OK) return rc;
    if (M % 8) {
        PadList pads;
        if (dX) { pads.add(Wg, S, w.Wg); pads.add(Wu, S, w.Wu); }
        if (dWg) pads.add(X, N, w.X);
        rc = pads.launch(M, st);
        if (rc != FW_OK) return rc;
        X = w.X; Wg = w.Wg; Wu = w.Wu;
    }
    if (dX) {
        TileProduct g = rows_plan(FW_BF16, N, M, S);
        g.a = bytes(w.D); g.b0 = bytes(Wg); g.b1 = bytes(Wu);
        g.apitch = 4ll * Sp; g.bpitch = 2ll * up8(M); g.aplane = N * g.apitch;
        g.partial = w.partial;
        rc = two ? tile_product<TILE_BF16, false, true, false>(g, RowsEpilogue<__bf16, true>{dX, N, M, in}, st)
                 : tile_product<TILE_BF16, false, true, false>(g, RowsEpilogue<__bf16, false>{dX, N, M, in}, st);
        if (rc != FW_OK) return rc;
    }
    if (dWg) {
        TileProduct g = weights_plan(FW_BF16, N, M, S);
        g.a = bytes(w.D); g.b0 = g.b1 = bytes(X);
        g.apitch = 4ll * Sp; g.bpitch = 2ll * up8(M); g.aplane = N * g.apitch;
        g.partial = w.partial;
        rc = two ? tile_product<TILE_BF16, true, true, false>(g, WeightsEpilogue<__bf16, true>{dWg, dWu, w.sums, mu, S, Sp, M, in}, st)
                 : tile_product<TILE_BF16, true, true, false>(g, WeightsEpilogue<__bf16, false>{dWg, dWu, w.sums, mu, S, Sp, M, in}, st);
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
