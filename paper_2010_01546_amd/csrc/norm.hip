// Rows of a layer's input: norm by the root mean square with the residual's addition, its gradient, and rows in 8 bits.
//
//   h = x + r,  rho = 1 / sqrt(mean h^2 + eps),  y = rho h w;      8 bits: s = max |y| / 127, q = rint(y / s)
//   dx = rho w dy - h rho^3 / M sum(w dy h) + dh,                  dw = sum over rows of dy h rho
//
// 8192 x 4608 bfloat16 with residual: norm 57 us a pass among others (5.3 TB/s), gradient 72 (4.2 TB/s); the kernels by themselves, after
// other work, 50 and 66 + 5 (the sum over the workgroups' dw).
// Bound by memory: each input is read once and each output written once, a row stays in the registers of its group of threads (a
// wavefront up to 2048 features, a workgroup beyond), 8 entries per lane and access.
// The sums over a row are float64 (a row of 1e20s has a norm too, and the cost hides behind the loads).  So is q: rho falls out of
// y / s = 127 h w / max |h w|, whose float32 rounding would put one value in 10^5 on the other side of a half.  127 / top is taken as
// two numbers (half of a row's largest entry is a tie at 63.5, common in bfloat16; 127 / 158 rounded makes it 63.4999...).
#include "fw_internal.h"
#include "lane_sums.h"
#include <type_traits>

namespace fw {
namespace {

// 8 entries of a row as they lie in memory (rows need not be 16-byte aligned)
template <class T> struct Eight;
template <> struct Eight<float> {
    float v[8];
    __device__ __forceinline__ float get(int i) const { return v[i]; }
    static __device__ __forceinline__ float held(float x) { return x; }
};
template <> struct Eight<__bf16> {
    unsigned v[4];
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }
    static __device__ __forceinline__ float held(float x) { return (float)(__bf16)x; }
};

// How rows end.  WHOLE: a multiple of 8 entries.  RAGGED: the last lane's 8 entries are moved back to end with the row and `skip` of
// them, which belong to the lane before, count as zero and are not stored.  SHORT: less than 8 entries, one lane, entry by entry.
// Rows end in the threads' last access (with_shape), the others are all there: `last` is a constant after unrolling, which keeps the
// ragged kernels' registers near the whole ones' (8192 x 4609 bfloat16: norm with residual 94 us without, 74 with, gradient 126 and 85).
enum { WHOLE, RAGGED, SHORT };
template <int END> struct Place {
    int start, skip, count;       // entries skip .. count - 1 of the 8 from `start` on are this lane's
    bool any, last;
    __device__ __forceinline__ Place(int m, int M, bool last)
        : start(END == RAGGED && last ? min(m, M - 8) : m), skip(END == RAGGED && last ? m - start : 0), count(END == SHORT ? M : 8), any(!last || m < M), last(last) {}
    __device__ __forceinline__ bool mine(int i) const { return END == WHOLE || !last || (END == RAGGED ? i >= skip : i < count); }
    template <class T> __device__ __forceinline__ void load(const T* row, Eight<T>& x) const {
        if (END == SHORT) {
            T e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = i < count ? row[i] : (T)0.f;
            __builtin_memcpy(&x, e, sizeof(x));
        } else {
            __builtin_memcpy(&x, row + start, sizeof(x));
        }
    }
    template <class T> __device__ __forceinline__ void store(T* row, const float (&x)[8]) const {
        T e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = (T)x[i];
        if (END == WHOLE || !last || (END == RAGGED && skip == 0)) {
            __builtin_memcpy(row + start, e, sizeof(e));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (mine(i)) row[start + i] = e[i];
        }
    }
};

// Sum and maximum over a wavefront, in every lane
__device__ __forceinline__ double lanes_sum(double v) {
    v = fold32(v, v);
    v = fold16(v, v);
    return sum16(v);
}
__device__ __forceinline__ double lanes_max(double v) {
    union { double d; unsigned i[2]; } x, y;
    x.d = v; y.d = v;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const auto r = __builtin_amdgcn_permlane32_swap(x.i[k], y.i[k], false, false);
        x.i[k] = r[0]; y.i[k] = r[1];
    }
    x.d = y.d = fmax(x.d, y.d);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const auto r = __builtin_amdgcn_permlane16_swap(x.i[k], y.i[k], false, false);
        x.i[k] = r[0]; y.i[k] = r[1];
    }
    x.d = fmax(x.d, y.d);
#define FW_MAX16(c) y.i[0] = __builtin_amdgcn_update_dpp(0, x.i[0], c, 0xf, 0xf, true); y.i[1] = __builtin_amdgcn_update_dpp(0, x.i[1], c, 0xf, 0xf, true); x.d = fmax(x.d, y.d)
    FW_MAX16(0xB1);      // lanes 1,0,3,2
    FW_MAX16(0x4E);      // lanes 2,3,0,1
    FW_MAX16(0x141);     // half of 16 mirrored
    FW_MAX16(0x140);     // 16 mirrored
#undef FW_MAX16
    return x.d;
}

// NORM: rows of the root mean square norm, otherwise the rows as they are (8 bits only)
template <class T, int G, int NV, int END, bool NORM>
__global__ __launch_bounds__(G < 256 ? 256 : G) void rows_kernel(const T* X, const T* R, int N, int M, const float* __restrict__ w, float eps,
                                                                 T* H, T* Y, signed char* __restrict__ q, float* __restrict__ qs) {
    __shared__ double red[2][16];
    constexpr bool WAVE = G == 64;
    const int t = threadIdx.x % G;
    const long long row = WAVE ? (long long)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (row >= N) return;                    // whole wavefronts, and only where a group is one
    const size_t at = (size_t)row * M;
    const bool eight = !NORM || q;
    float h[NV][8];
    Eight<float> f[NV];
    double ss = 0.0, top = 0.0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int m = 8 * (t + G * j);
#pragma unroll
        for (int i = 0; i < 8; ++i) { h[j][i] = 0.f; f[j].v[i] = 1.f; }
        const Place<END> p(m, M, j == NV - 1);
        if (!p.any) continue;
        Eight<T> x, r;
        p.load(X + at, x);
        if (NORM && R) p.load(R + at, r);
        if (NORM && w) p.load(w, f[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v = x.get(i);
            if (NORM && R) v = Eight<T>::held(v + r.get(i));
            h[j][i] = p.mine(i) ? v : 0.f;
        }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int m = 8 * (t + G * j);
        const Place<END> p(m, M, j == NV - 1);
        if (NORM && H && p.any) p.store(H + at, h[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (NORM) ss += (double)h[j][i] * (double)h[j][i];
            if (eight) {
                const double a = fabs(NORM && p.mine(i) ? (double)h[j][i] * (double)f[j].v[i] : (double)h[j][i]);
                top = fmax(top, a < __builtin_inf() ? a : __builtin_inf());   // NaN counts as infinite
            }
        }
    }
    if (NORM) ss = lanes_sum(ss);
    if (eight) top = lanes_max(top);
    if (!WAVE) {
        if ((threadIdx.x & 63) == 0) { red[0][threadIdx.x >> 6] = ss; red[1][threadIdx.x >> 6] = top; }
        __syncthreads();
        ss = 0.0;
#pragma unroll
        for (int i = 0; i < G / 64; ++i) { ss += red[0][i]; top = fmax(top, red[1][i]); }
    }
    const double rho = NORM ? 1.0 / sqrt(ss / (double)M + (double)eps) : 1.0;
    if (NORM && Y) {
        const float rf = (float)rho;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int m = 8 * (t + G * j);
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = h[j][i] * rf * f[j].v[i];
            const Place<END> p(m, M, j == NV - 1);
            if (p.any) p.store(Y + at, y);
        }
    }
    if (!eight) return;
    const bool fine = top > 0.0 && top < __builtin_inf() && rho > 0.0;
    // 127 / top as two numbers: v times it, rounded once, is a half where it is one (and, for products with w, within 2^-48 of one)
    const double inv = fine ? 127.0 / top : 0.0, rest = fine ? fma(-inv, top, 127.0) / top : 0.0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int m = 8 * (t + G * j);
        const Place<END> p(m, M, j == NV - 1);
        if (!p.any) continue;
        signed char b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double v = (double)h[j][i] * (double)f[j].v[i];
            b[i] = fine ? (signed char)(int)rint(fma(v, inv, v * rest)) : (signed char)0;
        }
        if (END == WHOLE || j < NV - 1 || (END == RAGGED && p.skip == 0)) {
            __builtin_memcpy(q + at + p.start, b, 8);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (p.mine(i)) q[at + p.start + i] = b[i];
        }
    }
    if (t == 0) qs[row] = top == 0.0 && rho > 0.0 ? 0.f : fine ? (float)(rho * top / 127.0) : __builtin_nanf("");
}

// Workgroups take rows in turn; each keeps the sums of its rows' dy h rho and leaves them in part[workgroup][Mp].  The next row's h and dy
// are asked for before this row's sums go round the wavefronts (a row of a workgroup waits for memory, then for its sums, then stores:
// one after the other that took 136 us for 8192 x 4608 in bfloat16).
template <class T, int G, int NV, int END>
__global__ __launch_bounds__(G < 256 ? 256 : G) void rms_grad_kernel(const T* __restrict__ H, int N, int M, int Mp, const float* __restrict__ w,
                                                                     float eps, const T* dY, const T* dH, T* dX, float* __restrict__ part) {
    constexpr bool WAVE = G == 64;
    constexpr int RB = WAVE ? 4 : 1, SPAN = 512 * NV;
    __shared__ double red[2][16][2];
    __shared__ float acc[WAVE ? RB * SPAN : 1];
    const int t = threadIdx.x % G, sub = WAVE ? threadIdx.x >> 6 : 0, wave = threadIdx.x >> 6;
    float sum[NV][8];
    Eight<float> f[NV];
    Eight<T> h[NV], v[NV], d[NV];
    const long long step = (long long)gridDim.x * RB;
    long long row = (long long)blockIdx.x * RB + sub;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int m = 8 * (t + G * j);
        const Place<END> p(m, M, j == NV - 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) { sum[j][i] = 0.f; f[j].v[i] = 1.f; }
        h[j] = v[j] = d[j] = Eight<T>{};
        if (p.any && w) p.load(w, f[j]);
        if (p.any && row < N) {
            p.load(H + (size_t)row * M, h[j]);
            p.load(dY + (size_t)row * M, v[j]);
        }
    }
    for (int turn = 0; row < N; row += step, turn ^= 1) {
        const size_t at = (size_t)row * M;
        Eight<T> nh[NV], nv[NV];
        double ss = 0.0, dot = 0.0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int m = 8 * (t + G * j);
            const Place<END> p(m, M, j == NV - 1);
            if (p.any && dH) p.load(dH + at, d[j]);
            nh[j] = h[j]; nv[j] = v[j];
            if (p.any && row + step < N) {
                p.load(H + at + step * M, nh[j]);
                p.load(dY + at + step * M, nv[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const Place<END> p(8 * (t + G * j), M, j == NV - 1);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double x = p.mine(i) ? (double)h[j].get(i) : 0.0;
                ss += x * x;
                dot += p.mine(i) ? x * (double)(v[j].get(i) * f[j].get(i)) : 0.0;
            }
        }
        ss = lanes_sum(ss);
        dot = lanes_sum(dot);
        if (!WAVE) {                             // two sets in turn: a set is written again only after the barrier of the next row
            if ((threadIdx.x & 63) == 0) { red[turn][wave][0] = ss; red[turn][wave][1] = dot; }
            __syncthreads();
            ss = dot = 0.0;
#pragma unroll
            for (int i = 0; i < G / 64; ++i) { ss += red[turn][i][0]; dot += red[turn][i][1]; }
        }
        const double rho = 1.0 / sqrt(ss / (double)M + (double)eps);
        const float rf = (float)rho, cf = (float)(rho * rho * dot / (double)M);      // rho^3 may lie outside float32
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int m = 8 * (t + G * j);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float hr = h[j].get(i) * rf, vv = v[j].get(i);
                sum[j][i] += vv * hr;
                x[i] = rf * (vv * f[j].get(i)) - hr * cf;
                if (dH) x[i] += d[j].get(i);
            }
            const Place<END> p(m, M, j == NV - 1);
            if (dX && p.any) p.store(dX + at, x);
            h[j] = nh[j]; v[j] = nv[j];
        }
    }
    if (!part) return;
    if (WAVE) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const Place<END> p(8 * (t + G * j), M, j == NV - 1);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (p.any && p.mine(i)) acc[sub * SPAN + p.start + i] = sum[j][i];
        }
        __syncthreads();
        for (int m = threadIdx.x; m < M; m += blockDim.x) {
            float s = 0.f;
#pragma unroll
            for (int r = 0; r < RB; ++r) s += acc[r * SPAN + m];
            part[(size_t)blockIdx.x * Mp + m] = s;
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const Place<END> p(8 * (t + G * j), M, j == NV - 1);
            if (p.any) p.store(part + (size_t)blockIdx.x * Mp, sum[j]);
        }
    }
}

// dw[m] = sum of the workgroups' partial sums, in a fixed order: 64 slices of them, then the slices.  16 columns of a workgroup.
__global__ __launch_bounds__(256) void column_sum_kernel(const float* __restrict__ part, int P, int M, int Mp, float* __restrict__ dw) {
    __shared__ float red[64][17];
    const int q = threadIdx.x & 3, slice = threadIdx.x >> 2, m = blockIdx.x * 16 + 4 * q;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m < M)
#pragma unroll 4
        for (int p = slice; p < P; p += 64) {
            const float4 v = *reinterpret_cast<const float4*>(part + (size_t)p * Mp + m);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    red[slice][4 * q] = s.x; red[slice][4 * q + 1] = s.y; red[slice][4 * q + 2] = s.z; red[slice][4 * q + 3] = s.w;
    __syncthreads();
    // 16 threads of a column add four slices each, then one of them adds those
    const int c = threadIdx.x & 15, part16 = threadIdx.x >> 4;
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) v += red[4 * part16 + i][c];
    __syncthreads();
    red[part16][c] = v;
    __syncthreads();
    if (threadIdx.x < 16 && blockIdx.x * 16 + c < M) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v += red[i][c];
        dw[blockIdx.x * 16 + c] = v;
    }
}

inline int rows_per_group(int M) { return M <= 2048 ? 4 : 1; }
inline int grad_blocks(int N, int M) {
    const int rb = rows_per_group(M);
    const long long b = ((long long)N + rb - 1) / rb;
    return (int)(b < 512 ? b : 512);
}
inline int up4(int m) { return (m + 3) / 4 * 4; }

// calls f(threads of a row, accesses of each, how rows end): as few accesses of 8 entries as hold the row, which ends in the last of them.  (4608 features: 256 threads with
// three accesses, 58 us for 8192 rows; 320 with two, 77 us.  2048 gradient rows of 12288: 512 with three, 46.6 us; 1024 with two, 55.)
template <class F> void with_shape(int M, const F& f) {
    using std::integral_constant;
    auto with_end = [&](auto G, auto NV) {
        if (M % 8 == 0) f(G, NV, integral_constant<int, WHOLE>());
        else f(G, NV, integral_constant<int, RAGGED>());
    };
    if (M < 8) f(integral_constant<int, 64>(), integral_constant<int, 1>(), integral_constant<int, SHORT>());
    else if (M <= 512) with_end(integral_constant<int, 64>(), integral_constant<int, 1>());
    else if (M <= 1024) with_end(integral_constant<int, 64>(), integral_constant<int, 2>());
    else if (M <= 1536) with_end(integral_constant<int, 64>(), integral_constant<int, 3>());
    else if (M <= 2048) with_end(integral_constant<int, 64>(), integral_constant<int, 4>());
    else if (M <= 4096) with_end(integral_constant<int, 256>(), integral_constant<int, 2>());
    else if (M <= 6144) with_end(integral_constant<int, 256>(), integral_constant<int, 3>());
    else if (M <= 8192) with_end(integral_constant<int, 512>(), integral_constant<int, 2>());
    else if (M <= 12288) with_end(integral_constant<int, 512>(), integral_constant<int, 3>());
    else if (M <= 16384) with_end(integral_constant<int, 512>(), integral_constant<int, 4>());
    else if (M <= 24576) with_end(integral_constant<int, 1024>(), integral_constant<int, 3>());
    else with_end(integral_constant<int, 1024>(), integral_constant<int, 4>());
}

template <class T, bool NORM>
fw_status rows_launch(const void* X, const void* R, int N, int M, const float* w, float eps, void* H, void* Y, signed char* q, float* qs,
                      hipStream_t st) {
    const int rb = rows_per_group(M);
    const dim3 grid((unsigned)(((long long)N + rb - 1) / rb));
    with_shape(M, [&](auto G, auto NV, auto END) {
        constexpr int g = decltype(G)::value;
        hipLaunchKernelGGL((rows_kernel<T, g, decltype(NV)::value, decltype(END)::value, NORM>), grid, dim3(g < 256 ? 256 : g), 0, st,
                           reinterpret_cast<const T*>(X), reinterpret_cast<const T*>(R), N, M, w, eps, reinterpret_cast<T*>(H),
                           reinterpret_cast<T*>(Y), q, qs);
    });
    FW_LAUNCH_CHECK();
    return FW_OK;
}

template <class T>
fw_status grad_launch(const void* H, int N, int M, const float* w, float eps, const void* dY, const void* dH, void* dX, float* part,
                      hipStream_t st) {
    const dim3 grid(grad_blocks(N, M));
    with_shape(M, [&](auto G, auto NV, auto END) {
        constexpr int g = decltype(G)::value;
        hipLaunchKernelGGL((rms_grad_kernel<T, g, decltype(NV)::value, decltype(END)::value>), grid, dim3(g < 256 ? 256 : g), 0, st,
                           reinterpret_cast<const T*>(H), N, M, up4(M), w, eps, reinterpret_cast<const T*>(dY), reinterpret_cast<const T*>(dH),
                           reinterpret_cast<T*>(dX), part);
    });
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

size_t rms_norm_grad_workspace_bytes(int N, int M) { return align_up((size_t)grad_blocks(N, M) * up4(M) * sizeof(float), 256); }

fw_status rms_norm_grad(const void* H, fw_dtype dt, int N, int M, const float* w, float eps, const void* dY, const void* dH, void* dX,
                        float* dw, void* ws, hipStream_t st) {
    float* part = dw ? reinterpret_cast<float*>(ws) : nullptr;
    const fw_status rc = dt == FW_BF16 ? grad_launch<__bf16>(H, N, M, w, eps, dY, dH, dX, part, st)
                                       : grad_launch<float>(H, N, M, w, eps, dY, dH, dX, part, st);
    if (rc != FW_OK || !dw) return rc;
    hipLaunchKernelGGL(column_sum_kernel, dim3((M + 15) / 16), dim3(256), 0, st, part, grad_blocks(N, M), M, up4(M), dw);
    FW_LAUNCH_CHECK();
    return FW_OK;
}

}  // namespace fw
