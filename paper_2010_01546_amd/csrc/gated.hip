// Gated feed-forward block and its gradient:
//   g = X Wg^T + bg,  u = X Wu^T + bu,  H = act(g) u;      kept for the backward pass: Z[0] = u act'(g), Z[1] = act(g)
//   dg = dH Z[0],  du = dH Z[1],   dX = dg Wg + du Wu,   dWg = dg^T (X - 1 mu^T),  dWu = du^T (X - 1 mu^T),  db = column sums
//
// bfloat16: both projections in one launch, the panel of weights holding the same columns of Wg and Wu, so that a lane has g and u of
// an element in its registers when the sums are done (tile_product.h).  The backward pass forms D = [dg | du] once, rounded to
// bfloat16 (small N S: as two bfloat16 numbers, two_planes), [N][2 Sp] with Sp = S rounded up to 64 and zeros between, and takes two
// products of it: dX = D [Wg; Wu], whose contraction runs over the rows of both weight matrices, and [dWg; dWu] = D^T X.  Operands that
// are contraction-major in memory are turned on the way out of LDS, not in memory.  mu is taken out of the sums: D^T (X - 1 mu^T) =
// D^T X - (D^T 1) mu^T, with D^T 1 summed from D as it is held, so that the identity is exact but for float32 sums.
// 8192 x 4608 to 12288, each launch as a pass of all of them has it: projections 1650 to 1780 us (Z stored; alone and without Z 1290, 1.44 PFLOP/s),
// D 291 to 300 (the rate of HBM), dX 1250 to 1530 (1.2 to 1.48 PFLOP/s), dWg and dWu 1350 to 1850 (1.0 to 1.37): the power limit, lower ends
// after a few passes.
// float32: the same products with every operand as three bfloat16 planes (tile_product.h), split in one pass over X and the weights, D
// when it is formed.  X is centred on mu as it is split.
// float32 with few rows: float32 matrix instructions on the operands as they are (few_product_kernel, few_rows_grad_kernel,
// few_weights_grad_kernel), the projections of one row without them.
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

// ---- epilogues: four entries of a row, 16 x 16 of a wavefront.  FIX (operands in planes: an infinite number has none): where an entry of the 16 x
// 16 is not finite they are computed once more on the float32 matrix instructions, and those entries replaced.  (Entry by entry would take
// minutes for a large matrix full of NaN.)
__device__ __forceinline__ bool finite(float v) { return fabsf(v) <= 3.402823466e38f; }
__device__ __forceinline__ bool not_finite(const floatx4& v) {
    return __builtin_amdgcn_ballot_w64(!(finite(v[0]) && finite(v[1]) && finite(v[2]) && finite(v[3]))) != 0;
}
// adds 16 x 16 results: row(k), column(k): the entries at k of the lane's row, of its 16 lanes' column
template <class Row, class Column> __device__ __forceinline__ void block_in_f32(floatx4& acc, int K, const Row& row, const Column& column) {
    const int q = (threadIdx.x & 63) >> 4;
#pragma unroll 4
    for (int k0 = 0; k0 < K; k0 += 4) {
        const int k = min(k0 + q, K - 1);
        const bool in = k0 + q < K;
        const float x = column(k), y = row(k);
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(in ? x : 0.f, in ? y : 0.f, acc, 0, 0, 0);
    }
}
// the column that a lane brings, where its results begin at column c
__device__ __forceinline__ int column_of(int c, int columns) {
    const int lane = threadIdx.x & 63;
    return min(c - 4 * (lane >> 4) + (lane & 15), columns - 1);
}
__device__ __forceinline__ void replace(floatx4& v, const floatx4& by) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = finite(v[i]) ? v[i] : by[i];
}
template <class T, bool FIX> struct GateEpilogue {
    T* H;
    float* Z;
    const float *bg, *bu;
    int N, S, act;
    const float *X, *Wg, *Wu;             // FIX: the operands as they were
    int M;
    __device__ __noinline__ floatx4 again(int n, int s, const float* W) const {
        const float *x = X + (size_t)min(n, N - 1) * M, *w = W + (size_t)column_of(s, S) * M;
        floatx4 v = {0.f, 0.f, 0.f, 0.f};
        block_in_f32(v, M, [&](int m) { return x[m]; }, [&](int m) { return w[m]; });
        return v;
    }
    __device__ __forceinline__ void apply(int n, int s, floatx4 gate, floatx4 up) const {
        if (FIX && not_finite(gate)) replace(gate, again(n, s, Wg));
        if (FIX && not_finite(up)) replace(up, again(n, s, Wu));
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
// what the gradients are computed from once more
template <class T> struct GradInputs { const T *X, *Wg, *Wu; const float* Z; const T* dH; const float* mu; int N, M, S; };
template <class T, bool FIX> struct RowsEpilogue {           // dX
    T* out;
    int N, M;
    GradInputs<T> in;
    __device__ __noinline__ floatx4 again(int n, int m) const {
        const size_t at = (size_t)min(n, N - 1) * in.S;
        const int c = column_of(m, M);
        floatx4 v = {0.f, 0.f, 0.f, 0.f};
        block_in_f32(v, in.S, [&](int s) { return (float)in.dH[at + s] * in.Z[at + s]; }, [&](int s) { return (float)in.Wg[(size_t)s * M + c]; });
        block_in_f32(v, in.S, [&](int s) { return (float)in.dH[at + s] * in.Z[(size_t)N * in.S + at + s]; },
                     [&](int s) { return (float)in.Wu[(size_t)s * M + c]; });
        return v;
    }
    __device__ __forceinline__ void apply(int n, int m, floatx4 acc) const {
        if (FIX && not_finite(acc)) replace(acc, again(n, m));
        if (n >= N || m >= M) return;
        const float v[4] = {acc[0], acc[1], acc[2], acc[3]};
        tile_store(out + (size_t)n * M + m, m, M, v);
    }
};
template <class T, bool FIX> struct WeightsEpilogue {        // rows below Sp are the gate's, the others the up projection's
    T *dWg, *dWu;
    const float *sums, *mu;               // mu: taken out here (bfloat16), or null
    int S, Sp, M;
    GradInputs<T> in;
    __device__ __noinline__ floatx4 again(int s, bool up, int m) const { return again_here(s, up, m); }
    __device__ __forceinline__ floatx4 again_here(int s, bool up, int m) const {
        const size_t at = (up ? (size_t)in.N * S : 0) + s;
        const int c = column_of(m, M);
        const float mean = in.mu ? in.mu[c] : 0.f;
        floatx4 v = {0.f, 0.f, 0.f, 0.f};
        block_in_f32(v, in.N, [&](int n) { return (float)in.dH[(size_t)n * S + s] * in.Z[(size_t)n * S + at]; },
                     [&](int n) { return (float)in.X[(size_t)n * M + c] - mean; });
        return v;
    }
    __device__ __forceinline__ void apply(int r, int m, floatx4 v) const {
        const int s = r >= Sp ? r - Sp : r;
        if (mu) {
            const float d = sums[min(r, 2 * Sp - 1)];
            float c[4];
            tile_vector(mu, m, M, c);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] -= d * c[i];
        }
        if (FIX && not_finite(v)) replace(v, again(min(s, S - 1), r >= Sp, m));
        if (s >= S || m >= M) return;
        const float out[4] = {v[0], v[1], v[2], v[3]};
        tile_store((r >= Sp ? dWu : dWg) + (size_t)s * M + m, m, M, out);
    }
};

// The same in bfloat16 without FIX, with mu: D^T X - (D^T 1) mu^T is inf - inf where the formula has an infinity.  Once a wavefront has stored
// its results it looks through the sums and the means behind them, and computes those again that come of one which is not finite, 16 x 16 at a time;
// each lane stores where it has stored before.  (2048 x 2304 x 6144 with D: 187 us, without this 185; looked for among the results, as FIX does, 201.)
struct CentredEpilogue : WeightsEpilogue<__bf16, false> {
    __device__ __forceinline__ void finish(int r0, int rows, int m0, int columns) const {
        const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
        bool fine = true;
        for (int i = lane; i < rows; i += 64) fine &= finite(sums[min(r0 + i, 2 * Sp - 1)]);
        for (int i = lane; i < columns; i += 64) fine &= finite(mu[min(m0 + i, M - 1)]);
        if (__builtin_amdgcn_ballot_w64(!fine) == 0) return;
        for (int r = r0 + l16; r - l16 < r0 + rows; r += 16) {
            const int s = r >= Sp ? r - Sp : r;
            const float d = sums[min(r, 2 * Sp - 1)];
            const bool none = has_nan(min(s, S - 1), r >= Sp, d);
            for (int m = m0 + 4 * q; m - 4 * q < m0 + columns; m += 16) {
                float c[4];
                tile_vector(mu, m, M, c);
                if (__builtin_amdgcn_ballot_w64(!none && !(finite(d) && finite(c[0]) && finite(c[1]) && finite(c[2]) && finite(c[3]))) == 0) continue;
                const floatx4 v = again_here(min(s, S - 1), r >= Sp, m);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (s < S && m + i < M && !(finite(d) && finite(c[i]))) (r >= Sp ? dWu : dWg)[(size_t)s * M + m + i] = (__bf16)v[i];
            }
        }
    }
    // whether the lane's column of D, one of 16 whose sums are d, has a NaN: its results are NaN then, and there already.  The four lanes of a
    // column take its entries in turn, until there is nothing more to find.
    __device__ __forceinline__ bool has_nan(int s, bool up, float d) const {
        const int lane = threadIdx.x & 63;
        const size_t at = (up ? (size_t)in.N * S : 0) + s;
        bool mine = false, column = false;
        for (int n = lane >> 4; n - (lane >> 4) < in.N && __builtin_amdgcn_ballot_w64(d != d && !column); n += 16) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const size_t e = (size_t)min(n + i, in.N - 1) * S;
                const float p = (float)in.dH[e + s] * in.Z[e + at];
                mine |= p != p;
            }
            const unsigned long long b = __builtin_amdgcn_ballot_w64(mine);
            column = ((b | b >> 16 | b >> 32 | b >> 48) >> (lane & 15)) & 1;
        }
        return column;
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

// ---- float32 gradients of few rows, on the float32 matrix instructions and the weights as they are.
// D[block of 16 s][gate, up][block of 16 n][lane][i] = dg or du of row n = lane % 16 and s = 4 (lane / 16) + i of the blocks, zeros past N and S:
// the second operand of four v_mfma_f32_16x16x4_f32, 1 KB that a wavefront loads at once.  dbg, dbu: sums over the rows, or null.
// A workgroup has a block of 16 s, a wavefront 16 rows of it.
__global__ __launch_bounds__(256) void few_pack_kernel(const float* __restrict__ dH, const float* __restrict__ Z, int N, int S, float* __restrict__ D,
                                                       float* __restrict__ dbg, float* __restrict__ dbu) {
    __shared__ float red[4][2][16];
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, a = threadIdx.x >> 6, NA = blockDim.x >> 6;
    const int n = 16 * a + l16, s = 16 * blockIdx.x + 4 * q;
    float d[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {                    // loads of clamped places rather than branches: all of them go out together
        const bool in = n < N && s + i < S;
        const size_t e = (size_t)min(n, N - 1) * S + min(s + i, S - 1);
        const float h = dH[e], z = Z[e], y = Z[(size_t)N * S + e];
        d[0][i] = in ? h * z : 0.f;
        d[1][i] = in ? h * y : 0.f;
    }
#pragma unroll
    for (int g = 0; g < 2; ++g)
        *reinterpret_cast<float4*>(D + (((size_t)blockIdx.x * 2 + g) * NA + a) * 256 + 4 * lane) = make_float4(d[g][0], d[g][1], d[g][2], d[g][3]);
    if (!dbg) return;
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int k = 1; k < 16; k *= 2) d[g][i] += __shfl_xor(d[g][i], k);
            if (l16 == 0) red[a][g][4 * q + i] = d[g][i];
        }
    __syncthreads();
    const int t = threadIdx.x, to = 16 * blockIdx.x + (t & 15);
    if (t >= 32 || to >= S) return;
    float v = red[0][t >> 4][t & 15];
    for (int k = 1; k < NA; ++k) v += red[k][t >> 4][t & 15];
    (t >> 4 ? dbu : dbg)[to] = v;
}

// dX (one row of 4172 features, 7040: 60 us, 3.9 TB/s of the weights): a workgroup has 64 columns and a run of blocks of s, its wavefronts
// take these in turn and add up their sums.  A lane holds four columns next to each other of the rows 4 q + i of a block (whole cache
// lines); the last lanes' are moved back to end with the row, so that some columns are computed twice, alike.  out: dX, or [run][N][M].
template <int NA>
__global__ __launch_bounds__(512) void few_rows_grad_kernel(const float* __restrict__ D, const float* __restrict__ Wg, const float* __restrict__ Wu,
                                                            int N, int M, int S, int per_run, float* __restrict__ out) {
    constexpr int NW = 8;
    __shared__ floatx4 red[NW][4][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
    const int m0 = blockIdx.x * 64, m = min(m0 + 4 * l16, M - 4);
    const int blocks = (S + 15) / 16, end = min(((int)blockIdx.y + 1) * per_run, blocks);
    floatx4 acc[NA][4];
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[a][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    const auto load = [&](floatx4 (&w)[2][4], int b) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int s = 16 * b + 4 * q + i;
                const float* p = (g ? Wu : Wg) + (size_t)s * M + m;
                __builtin_memcpy(&w[g][i], b < end && s < S ? reinterpret_cast<const char*>(p) : reinterpret_cast<const char*>(&tile_zero), 16);
            }
    };
    floatx4 w[2][4], next[2][4];
    load(next, blockIdx.y * per_run + wave);
    for (int b = blockIdx.y * per_run + wave; b < end; b += NW) {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k >> 2][k & 3] = next[k >> 2][k & 3];
        load(next, b + NW);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int a = 0; a < NA; ++a) {
                const floatx4 d = *reinterpret_cast<const floatx4*>(D + (((size_t)b * 2 + g) * NA + a) * 256 + 4 * lane);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[a][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[g][i][j], d[i], acc[a][j], 0, 0, 0);
            }
    }
    out += (size_t)blockIdx.y * N * M;
#pragma unroll
    for (int a = 0; a < NA; ++a) {
        if (a) __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) red[wave][j][lane] = acc[a][j];
        __syncthreads();
        if (wave < 4 && 16 * a + l16 < N) {
            floatx4 v = red[0][wave][lane];
#pragma unroll
            for (int k = 1; k < NW; ++k)
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] += red[k][wave][lane][r];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int c = m0 + 4 * (4 * q + r);
                if (c < M) out[(size_t)(16 * a + l16) * M + min(c, M - 4) + wave] = v[r];
            }
        }
    }
}

// out[e] = the runs' sums, in order
__global__ __launch_bounds__(256) void few_sum_kernel(const float* __restrict__ part, int runs, int n, float* __restrict__ out) {
    const int e = blockIdx.x * 256 + threadIdx.x;
    if (e >= n) return;
    float v = part[e];
    for (int r = 1; r < runs; ++r) v += part[(size_t)r * n + e];
    out[e] = v;
}

// dWg and dWu: a wavefront has 64 x 64 entries of both, a workgroup two times two of these.  Bound by writing them (one row, 4172 features, 7040:
// 85 us, 2.8 TB/s), from about 50 rows on by the matrix instructions.
__global__ __launch_bounds__(256) void few_weights_grad_kernel(const float* __restrict__ D, int NA, const float* __restrict__ X,
                                                               const float* __restrict__ mu, int N, int M, int S, float* __restrict__ dWg,
                                                               float* __restrict__ dWu) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
    const int m0 = blockIdx.x * 128 + 64 * (wave & 1), s0 = blockIdx.y * 128 + 64 * (wave >> 1), blocks = (S + 15) / 16;
    if (m0 >= M || s0 >= S) return;
    int m[4];
    float c[4];
    const float* d[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        m[j] = min(m0 + 16 * j + l16, M - 1);
        c[j] = mu ? mu[m[j]] : 0.f;
        d[j] = D + (size_t)min(s0 / 16 + j, blocks - 1) * 2 * NA * 256 + 64 * (l16 >> 2) + (l16 & 3);
    }
    floatx4 acc[2][4][4];
#pragma unroll
    for (int k = 0; k < 32; ++k) acc[k >> 4][(k >> 2) & 3][k & 3] = floatx4{0.f, 0.f, 0.f, 0.f};
    struct Step { float x[4], y[2][4]; };
    const auto load = [&](Step& t, int n) __attribute__((always_inline)) {
        const int nx = min(n, N - 1), ny = min(n, 16 * NA - 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            t.x[j] = X[(size_t)nx * M + m[j]];
#pragma unroll
            for (int g = 0; g < 2; ++g) t.y[g][j] = d[j][(g * NA + ny / 16) * 256 + 4 * (ny % 16)];
        }
    };
    constexpr int AHEAD = 4;
    Step step[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) load(step[k], 4 * k + q);
    for (int n0 = 0; n0 < N; n0 += 4 * AHEAD) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int n = n0 + 4 * k + q;
            float x[4], y[2][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {            // rows past the end: zeros of both
                x[j] = n < N ? step[k].x[j] - c[j] : 0.f;
                y[0][j] = n < N ? step[k].y[0][j] : 0.f;
                y[1][j] = n < N ? step[k].y[1][j] : 0.f;
            }
            load(step[k], n + 4 * AHEAD);
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[g][i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[g][i], acc[g][i][j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = s0 + 16 * i + l16;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float v[4] = {acc[g][i][j][0], acc[g][i][j][1], acc[g][i][j][2], acc[g][i][j][3]};
                if (s < S) tile_store((g ? dWu : dWg) + (size_t)s * M + m0 + 16 * j + 4 * q, m0 + 16 * j + 4 * q, M, v);
            }
        }
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

// float32 projections on the operands as they are: up to 64 rows, which the one read of the weights bounds or nearly so; in planes these are
// written and read again (4172 features to 7040, 17 rows: 202 us against 68.6, 64 rows: 204 against 117, 86 rows: 215 against 200).  More than
// 32 rows of few columns are too few workgroups (64 x 4000 to 64: 22.6 us in planes against 43).
inline bool few_forward(fw_dtype dt, int N, int M, int S) {
    return dt == FW_F32 ? N <= 32 || (N <= 64 && S >= 256) : few_rows(N, S, M % 8 == 0, true);
}

inline unsigned blocks_for(size_t n) { return (unsigned)((n + 255) / 256 < 16384 ? (n + 255) / 256 : 16384); }
inline int up8(int m) { return (m + 7) / 8 * 8; }
inline int up64(int s) { return (s + 63) / 64 * 64; }
// bfloat16: D in two planes, 16 bits, where the rounding to 8 bits does not average out: it adds an error as large as that of rounding the
// result, 1.42 times the latter together, but up to 1.8 times where a few entries make up the sum (11 x 64, S = 64).  The products then
// go over X or the weights twice, and their epilogue looks for results that are not finite: next to nothing where launches bound them, but
// large weights have few rows on this side too (4608 features, 12288: 42 rows in two planes dX 89 us, dWg and dWu 149; 43 rows in one 58 and
// 96; 576 to 2304: 227 rows 30 and 24, 228 rows 21 and 16).
constexpr int kTwoPlanes = 1 << 19;
inline bool two_planes(fw_dtype dt, int N, int S) { return dt == FW_BF16 && (long long)N * S <= kTwoPlanes; }
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
    tile_plan(g, false, dt == FW_F32, dt == FW_F32 ? 4 : 2, true);
    return g;
}

// float32 gradients on the operands as they are.  Both of 4172 features to 7040, one row: 387 us in planes against 151; 64 rows: 392 against 279,
// of 576 to 2304: 59 against 55, of 300 to 1000: 44 against 50.  (86 rows as eight blocks of 16: no faster than in planes.)
inline bool few_grad(fw_dtype dt, int N, int M, int S) {
    return dt == FW_F32 && M >= 4 && (N <= 32 || (N <= 64 && (long long)M * S >= 1 << 20));
}
// blocks of 16 rows, and runs of blocks of s that give each of 512 workgroups two blocks a wavefront or more
inline int few_blocks(int N) { return N <= 16 ? 1 : N <= 32 ? 2 : 4; }
inline int few_runs(int M, int S) {
    const int most = (S + 15) / 16 / 16, want = 512 / ((M + 63) / 64), runs = want < most ? want : most;
    return runs > 1 ? runs : 1;
}

size_t plane3_bytes(int R, int M) { return 6 * (size_t)R * up64(M); }
struct ForwardWs { void *X, *Wg, *Wu, *partial; size_t total; };
ForwardWs forward_ws(fw_dtype dt, int N, int M, int S, void* ws) {
    Carve c = {reinterpret_cast<char*>(ws)};
    ForwardWs w = {};
    const bool few = few_forward(dt, N, M, S);
    if (dt == FW_F32) {
        if (!few) {
            w.X = c.take(plane3_bytes(N, M));
            w.Wg = c.take(plane3_bytes(S, M));
            w.Wu = c.take(plane3_bytes(S, M));
        }
    } else if (M % 8 && !few) {
        w.X = c.take((size_t)N * up8(M) * 2);
        w.Wg = c.take((size_t)S * up8(M) * 2);
        w.Wu = c.take((size_t)S * up8(M) * 2);
    }
    if (!few) w.partial = c.take(tile_partial_bytes(forward_plan(dt, N, M, S)));
    w.total = c.used;
    return w;
}
struct GradWs { void *D, *X, *Wg, *Wu, *partial; float *part, *sums; size_t total; };
GradWs grad_ws(fw_dtype dt, int N, int M, int S, void* ws) {
    Carve c = {reinterpret_cast<char*>(ws)};
    GradWs w = {};
    const size_t Sp = up64(S);
    if (few_grad(dt, N, M, S)) {
        w.D = c.take((size_t)((S + 15) / 16) * 2 * few_blocks(N) * 1024);
        w.partial = c.take(few_runs(M, S) > 1 ? (size_t)few_runs(M, S) * N * M * 4 : 0);
        w.total = c.used;
        return w;
    }
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
    if (few_forward(FW_F32, N, M, S)) {
        const GateEpilogue<float, false> epi = {H, Z, bg, bu, N, S, (int)act};
        const FewProduct few = {bytes(X), bytes(Wg), bytes(Wu), N, S, 4 * M};
        if (N > 1) return few_product<TILE_F32, true>(few, epi, st);
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
    if (few_forward(FW_BF16, N, M, S)) return few_product<TILE_BF16, true>({bytes(X), bytes(Wg), bytes(Wu), N, S, 2 * M}, epi, st);
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
    if (few_grad(FW_F32, N, M, S)) {
        const auto with_blocks = [&](auto NA) {
            constexpr int na = decltype(NA)::value;
            float* D = reinterpret_cast<float*>(w.D);
            hipLaunchKernelGGL(few_pack_kernel, dim3((S + 15) / 16), dim3(64 * na), 0, st, dH, Z, N, S, D, dbg, dbu);
            FW_LAUNCH_CHECK();
            if (dX) {
                const int want = few_runs(M, S), per = ((S + 15) / 16 + want - 1) / want, runs = ((S + 15) / 16 + per - 1) / per;
                hipLaunchKernelGGL(few_rows_grad_kernel<na>, dim3((M + 63) / 64, runs), dim3(512), 0, st, D, Wg, Wu, N, M, S, per,
                                   runs > 1 ? reinterpret_cast<float*>(w.partial) : dX);
                FW_LAUNCH_CHECK();
                if (runs > 1) {
                    hipLaunchKernelGGL(few_sum_kernel, dim3((N * M + 255) / 256), dim3(256), 0, st, reinterpret_cast<const float*>(w.partial), runs, N * M, dX);
                    FW_LAUNCH_CHECK();
                }
            }
            if (dWg) {
                hipLaunchKernelGGL(few_weights_grad_kernel, dim3((M + 127) / 128, (S + 127) / 128), dim3(256), 0, st, D, na, X, mu, N, M, S, dWg, dWu);
                FW_LAUNCH_CHECK();
            }
            return FW_OK;
        };
        if (N <= 16) return with_blocks(std::integral_constant<int, 1>());
        if (N <= 32) return with_blocks(std::integral_constant<int, 2>());
        return with_blocks(std::integral_constant<int, 4>());
    }
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
        const WeightsEpilogue<__bf16, true> fix = {dWg, dWu, w.sums, mu, S, Sp, M, in};
        const WeightsEpilogue<__bf16, false> plain = {dWg, dWu, w.sums, mu, S, Sp, M, in};
        rc = two ? tile_product<TILE_BF16, true, true, false>(g, fix, st)
             : mu ? tile_product<TILE_BF16, true, true, false>(g, CentredEpilogue{plain}, st)
                  : tile_product<TILE_BF16, true, true, false>(g, plain, st);
    }
    return rc;
}

}  // namespace

void gated_tiles(int product, fw_dtype dt, int N, int M, int S, TileChoice* c) {
    if (product == 0 ? few_forward(dt, N, M, S) : few_grad(dt, N, M, S)) *c = {1};
    else *c = tile_choice(product == 0 ? forward_plan(dt, N, M, S) : product == 1 ? rows_plan(dt, N, M, S) : weights_plan(dt, N, M, S), product == 0);
}
size_t gated_forward_workspace_bytes(fw_dtype dt, int N, int M, int S) { return forward_ws(dt, N, M, S, nullptr).total; }
size_t gated_grad_workspace_bytes(fw_dtype dt, int N, int M, int S) { return grad_ws(dt, N, M, S, nullptr).total; }
int gated_grad_two_planes_rows(fw_dtype dt, int S) { return dt == FW_BF16 ? kTwoPlanes / S : 0; }

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
