// Product of rows in 8 bits with weights in 8 bits, a scale per token and per channel:
//   Y[n][s] = sx[n] sw[s] sum_m Xq[n][m] Wq[s][m] + b[s],   the sums exact in 32-bit integers
#include "fw_internal.h"
#include "tile_product.h"

namespace fw {

size_t int8_product_workspace_bytes(int, int, int) { return 0; }

template <class T>
static fw_status run(const signed char* Xq, const float* sx, int N, int M, int S, const signed char* Wq, const float* sw, const float* b, T* Y,
                     hipStream_t st) {
    return strided_product<int>(Xq, M, 1, Wq, M, 1, N, S, M, [=] __device__(long long r, int c, int v) {
        Y[r * S + c] = (T)((float)v * sx[r] * sw[c] + (b ? b[c] : 0.f));
    }, st);
}

fw_status int8_product(const signed char* Xq, const float* sx, int N, int M, int S, const signed char* Wq, const float* sw, const float* b,
                       void* Y, fw_dtype dt, void*, hipStream_t st) {
    return dt == FW_BF16 ? run(Xq, sx, N, M, S, Wq, sw, b, (__bf16*)Y, st) : run(Xq, sx, N, M, S, Wq, sw, b, (float*)Y, st);
}

}  // namespace fw
