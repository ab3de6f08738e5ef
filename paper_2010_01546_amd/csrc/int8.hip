// Product of rows in 8 bits with weights in 8 bits, a scale per token and per channel:
//   Y[n][s] = sx[n] sw[s] sum_m Xq[n][m] Wq[s][m] + b[s],   the sums exact in 32-bit integers (tile_product.h)
// 8192 x 4608 to 12288: 421 to 457 us by card and pass (2.0 to 2.2 POP/s, the power limit); 16 x 12288 to 4608: 14.7 us from HBM (3.8 TB/s),
// 11.6 with the weights in the last-level cache.
#include "fw_internal.h"
#include "tile_product.h"

namespace fw {
namespace {

inline int up16(int m) { return (m + 15) / 16 * 16; }

template <class T> struct ScaleEpilogue {
    T* Y;
    const float *sx, *sw, *b;
    int N, S;
    __device__ __forceinline__ void apply(int n, int s, const intx4& acc) const {
        if (n >= N || s >= S) return;
        float w[4], c[4], y[4];
        tile_vector(sw, s, S, w);
        tile_vector(b, s, S, c);
        const float x = sx[n];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (float)acc[i] * x * w[i] + c[i];
        if (fabsf(x) > 0x1p96f) {             // a sum of up to 2^30 times x may leave float32 on the way to a result that is inside it
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = (float)acc[i] * (x * 0x1p-40f) * w[i] * 0x1p40f + c[i];
        }
        tile_store(Y + (size_t)n * S + s, s, S, y);
    }
};

// rows of M bytes to rows of Mp (a multiple of 16), zeros behind
__global__ __launch_bounds__(256) void pad_bytes_kernel(const signed char* __restrict__ in, int M, int Mp, size_t n16, uint4* __restrict__ out) {
    const int c16 = Mp / 16;
    for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < n16; e += (size_t)gridDim.x * 256) {
        const size_t r = e / c16;
        const int m = 16 * (int)(e - r * c16);
        const signed char* p = in + r * M + m;
        union { uint4 v; signed char c[16]; } u;
        if (m + 16 <= M) {
            __builtin_memcpy(&u, p, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) u.c[i] = m + i < M ? p[i] : (signed char)0;
        }
        out[e] = u.v;
    }
}

fw_status pad_bytes(const signed char* in, int R, int M, void* out, hipStream_t st) {
    const size_t n = (size_t)R * (up16(M) / 16), blocks = (n + 255) / 256;
    hipLaunchKernelGGL(pad_bytes_kernel, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, st, in, M, up16(M), n,
                       reinterpret_cast<uint4*>(out));
    FW_LAUNCH_CHECK();
    return FW_OK;
}

TileProduct plan(int N, int M, int S) {
    TileProduct g = {};
    g.R = N; g.C = S; g.chunks = up16(M) / 16;
    g.stages = g.once = g.part = (g.chunks + 7) / 8;
    tile_plan(g, false, false, 2);
    return g;
}
size_t padded_bytes(int R, int M) { return M % 16 ? align_up((size_t)R * up16(M), 256) : 0; }

}  // namespace

void int8_tiles(int N, int M, int S, TileChoice* c) {
    if (few_rows(N, S, M % 16 == 0, false)) *c = {1};
    else *c = tile_choice(plan(N, M, S), false);
}

size_t int8_product_workspace_bytes(int N, int M, int S) {
    if (few_rows(N, S, M % 16 == 0, false)) return 0;
    return padded_bytes(N, M) + padded_bytes(S, M) + tile_partial_bytes(plan(N, M, S));
}

fw_status int8_product(const signed char* Xq, const float* sx, int N, int M, int S, const signed char* Wq, const float* sw, const float* b,
                       void* Y, fw_dtype dt, void* ws, hipStream_t st) {
    char* w = reinterpret_cast<char*>(ws);
    if (few_rows(N, S, M % 16 == 0, false)) {
        const FewProduct few = {reinterpret_cast<const char*>(Xq), reinterpret_cast<const char*>(Wq), nullptr, N, S, M};
        if (dt == FW_BF16) return few_product<TILE_I8, false>(few, ScaleEpilogue<__bf16>{reinterpret_cast<__bf16*>(Y), sx, sw, b, N, S}, st);
        return few_product<TILE_I8, false>(few, ScaleEpilogue<float>{reinterpret_cast<float*>(Y), sx, sw, b, N, S}, st);
    }
    TileProduct g = plan(N, M, S);
    g.a = reinterpret_cast<const char*>(Xq);
    g.b0 = reinterpret_cast<const char*>(Wq);
    if (M % 16) {            // 16-byte loads need aligned rows
        fw_status rc = pad_bytes(Xq, N, M, w, st);
        if (rc == FW_OK) rc = pad_bytes(Wq, S, M, w + padded_bytes(N, M), st);
        if (rc != FW_OK) return rc;
        g.a = w;
        g.b0 = w + padded_bytes(N, M);
    }
    g.b1 = g.b0;
    g.apitch = g.bpitch = up16(M);
    g.partial = w ? w + padded_bytes(N, M) + padded_bytes(S, M) : nullptr;
    if (dt == FW_BF16)
        return tile_product<TILE_I8, false, false, false>(g, ScaleEpilogue<__bf16>{reinterpret_cast<__bf16*>(Y), sx, sw, b, N, S}, st);
    return tile_product<TILE_I8, false, false, false>(g, ScaleEpilogue<float>{reinterpret_cast<float*>(Y), sx, sw, b, N, S}, st);
}

}  // namespace fw
