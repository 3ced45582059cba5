// Rows to 8-bit integers with one scale each.
//   v_j = x_j c_j;  a = max_j |v_j|;  scale = a / 127;  code_j = rne(v_j * (127 / a)), each step rounded once to fp32.
// a < 2^-110 (127 / a nears the largest float): scale 0, codes 0.  An infinity or a NaN in the row: scale NaN, codes 0, so
// that whatever is computed with the row is NaN.
#include "qamw_product.hpp"

namespace qamw {
namespace {

constexpr int QT = 256;          // threads of a workgroup, which has one row

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    for (int d = 32; d; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return v;
}

// Two sweeps over the row; the second one finds it in the caches.
template <int DTYPE>
__global__ __launch_bounds__(QT) void k_quantize_any(const void *X, int d, int64_t ldx, const float *col_scale, int8_t *codes,
                                                     int64_t ldc, float *scales) {
    __shared__ uint32_t part[QT / WAVE];
    const int64_t row = blockIdx.x, at = row * ldx;
    uint32_t most = 0;           // of the bits of |v|: orders finite values, then infinity, then NaNs
    for (int j = threadIdx.x; j < d; j += QT) {
        const float v = Elem<DTYPE>::load(X, at + j) * (col_scale ? col_scale[j] : 1.0f);
        most = max(most, __float_as_uint(v) & 0x7FFFFFFFu);
    }
    most = wave_max(most);
    if (threadIdx.x % WAVE == 0) part[threadIdx.x / WAVE] = most;
    __syncthreads();
    for (int w = 0; w < QT / WAVE; ++w) most = max(most, part[w]);
    const float a = __uint_as_float(most);
    const bool finite = most < 0x7F800000u, some = finite && a >= 0x1p-110f;
    const float inv = some ? 127.0f / a : 0.0f;
    if (threadIdx.x == 0) scales[row] = some ? a / 127.0f : finite ? 0.0f : __uint_as_float(0x7FC00000u);
    for (int j = threadIdx.x; j < d; j += QT) {
        const float v = Elem<DTYPE>::load(X, at + j) * (col_scale ? col_scale[j] : 1.0f);
        codes[row * ldc + j] = some ? (int8_t)(int)rintf(v * inv) : (int8_t)0;
    }
}

}  // namespace

hipError_t launch_int8_quantize(const void *X, int dtype, int64_t m, int d, int64_t ldx, const float *col_scale, int8_t *codes,
                                int64_t ldc, float *scales, hipStream_t stream) {
    if (m == 0) return hipSuccess;
    if (dtype == 0)
        k_quantize_any<0><<<dim3((uint32_t)m), QT, 0, stream>>>(X, d, ldx, col_scale, codes, ldc, scales);
    else
        k_quantize_any<1><<<dim3((uint32_t)m), QT, 0, stream>>>(X, d, ldx, col_scale, codes, ldc, scales);
    return hipGetLastError();
}

}  // namespace qamw
