// Rows to 8-bit integers with one scale each.
//   v_j = x_j c_j;  a = max_j |v_j|;  scale = a / 127;  code_j = rne(v_j * (127 / a)), each step rounded once to fp32.
// a < 2^-110 (127 / a nears the largest float): scale 0, codes 0.  An infinity or a NaN in the row: scale NaN, codes 0, so
// that whatever is computed with the row is NaN.
// Memory bounds it: 4 or 2 bytes a value are read and one is written.
#include "qamw_product_tile.hpp"

namespace qamw {
namespace {

// ---- rows of whole 16 bytes ------------------------------------------------------------------------------------------------
//
// TR threads have a row and hold its values, EIGHTS groups of 8 each, between the maximum and the codes: one read of X.  Groups past
// the end of the row are loaded as zeros, from beyond the buffer's end.  TR and EIGHTS are the fewest threads and groups that hold the
// row, so that short rows waste no lanes.  8192 rows of 4096: bf16 17.3 us (5.8 TB/s; the sweeps below 47 us), fp32 24.5 us (6.8; 52);
// 512 rows of 13824 bf16 6.2 us (the sweeps 19).
template <int DTYPE, int TR, int EIGHTS>
__global__ __launch_bounds__(TR < 256 ? 256 : TR) void k_quantize(const char *X, int m, int d, int64_t ldx, const float *col_scale,
                                                                  int8_t *codes, int64_t ldc, float *scales) {
    constexpr int ROWS = TR < 256 ? 256 / TR : 1, SPAN = TR * 8;
    __shared__ uint32_t part[TR / WAVE];
    const int tid = threadIdx.x % TR;
    const int64_t row = (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TR) : 0);
    if (ROWS > 1 && row >= m) return;                      // whole waves; rows of one wave meet no barrier
    const auto xb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(X + row * ldx * (DTYPE ? 2 : 4)), 0, d * (DTYPE ? 2 : 4), 0x00020000);
    const auto cb = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(col_scale), 0, col_scale ? d * 4 : 0, 0x00020000);
    Eight<DTYPE> raw[EIGHTS];
    Eight<0> col[EIGHTS];
#pragma unroll
    for (int i = 0; i < EIGHTS; ++i) raw[i].load(xb, (uint32_t)(i * SPAN + tid * 8) * (DTYPE ? 2 : 4));
    if (col_scale)
#pragma unroll
        for (int i = 0; i < EIGHTS; ++i) col[i].load(cb, (uint32_t)(i * SPAN + tid * 8) * 4);
    float v[EIGHTS][8];
    uint32_t most = 0;           // of the bits of |v|: orders finite values, then infinity, then NaNs
#pragma unroll
    for (int i = 0; i < EIGHTS; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            v[i][k] = raw[i].value(k);
            if (col_scale) v[i][k] *= col[i].value(k);
            most = max(most, __float_as_uint(v[i][k]) & 0x7FFFFFFFu);
        }
    most = wave_max(most);
    if (TR > WAVE) {
        if (tid % WAVE == 0) part[tid / WAVE] = most;
        __syncthreads();
        most = wave_max(part[tid % (TR / WAVE)]);
    }
    const Quantiser z(most);
    if (tid == 0) scales[row] = z.scale;
#pragma unroll
    for (int i = 0; i < EIGHTS; ++i) {
        const int j = i * SPAN + tid * 8;
        if (j >= d) continue;
        uint32_t c[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) c[k / 4] |= z.code(v[i][k]) << (k % 4 * 8);
        *reinterpret_cast<uint2 *>(codes + row * ldc + j) = {c[0], c[1]};
    }
}

template <int DTYPE>
hipError_t launch_whole(const void *X, int64_t m, int d, int64_t ldx, const float *col_scale, int8_t *codes, int64_t ldc, float *scales,
                        hipStream_t stream) {
    const char *x = static_cast<const char *>(X);
    const uint32_t n = (uint32_t)m;
    if (d <= 512) k_quantize<DTYPE, 64, 1><<<(n + 3) / 4, 256, 0, stream>>>(x, n, d, ldx, col_scale, codes, ldc, scales);
    else if (d <= 1024) k_quantize<DTYPE, 64, 2><<<(n + 3) / 4, 256, 0, stream>>>(x, n, d, ldx, col_scale, codes, ldc, scales);
    else if (d <= 2048) k_quantize<DTYPE, 256, 1><<<n, 256, 0, stream>>>(x, n, d, ldx, col_scale, codes, ldc, scales);
    else if (d <= 4096) k_quantize<DTYPE, 512, 1><<<n, 512, 0, stream>>>(x, n, d, ldx, col_scale, codes, ldc, scales);
    else if (d <= 8192) k_quantize<DTYPE, 512, 2><<<n, 512, 0, stream>>>(x, n, d, ldx, col_scale, codes, ldc, scales);
    else k_quantize<DTYPE, 512, 4><<<n, 512, 0, stream>>>(x, n, d, ldx, col_scale, codes, ldc, scales);
    return hipGetLastError();
}
constexpr int Q_MOST = 512 * 8 * 4;

// ---- every shape and alignment ---------------------------------------------------------------------------------------------

constexpr int QT = 256;          // threads of a workgroup, which has one row

// Rows that do not begin or end on 16 bytes, and ones of more than Q_MOST values: two sweeps, the second one finds the row in the caches.
// 8192 rows of 4096 bf16 in 47 us.
template <int DTYPE>
__global__ __launch_bounds__(QT) void k_quantize_any(const void *X, int d, int64_t ldx, const float *col_scale, int8_t *codes,
                                                     int64_t ldc, float *scales) {
    __shared__ uint32_t part[QT / WAVE];
    const int64_t row = blockIdx.x, at = row * ldx;
    uint32_t most = 0;
    for (uint32_t j = threadIdx.x; j < (uint32_t)d; j += QT) {             // unsigned: the last step may pass 2^31
        const float v = Elem<DTYPE>::load(X, at + j) * (col_scale ? col_scale[j] : 1.0f);
        most = max(most, __float_as_uint(v) & 0x7FFFFFFFu);
    }
    most = wave_max(most);
    if (threadIdx.x % WAVE == 0) part[threadIdx.x / WAVE] = most;
    __syncthreads();
    const Quantiser z(wave_max(part[threadIdx.x % (QT / WAVE)]));
    if (threadIdx.x == 0) scales[row] = z.scale;
    for (uint32_t j = threadIdx.x; j < (uint32_t)d; j += QT)
        codes[row * ldc + j] = (int8_t)z.code(Elem<DTYPE>::load(X, at + j) * (col_scale ? col_scale[j] : 1.0f));
}

}  // namespace

hipError_t launch_int8_quantize(const void *X, int dtype, int64_t m, int d, int64_t ldx, const float *col_scale, int8_t *codes,
                                int64_t ldc, float *scales, hipStream_t stream) {
    if (m == 0) return hipSuccess;
    auto at = [](const void *q) { return reinterpret_cast<uintptr_t>(q); };
    if (d % 8 == 0 && d <= Q_MOST && (at(X) | at(col_scale)) % 16 == 0 && ldx * (dtype == 0 ? 4 : 2) % 16 == 0 && at(codes) % 8 == 0 && ldc % 8 == 0)
        return dtype == 0 ? launch_whole<0>(X, m, d, ldx, col_scale, codes, ldc, scales, stream)
                          : launch_whole<1>(X, m, d, ldx, col_scale, codes, ldc, scales, stream);
    if (dtype == 0)
        k_quantize_any<0><<<dim3((uint32_t)m), QT, 0, stream>>>(X, d, ldx, col_scale, codes, ldc, scales);
    else
        k_quantize_any<1><<<dim3((uint32_t)m), QT, 0, stream>>>(X, d, ldx, col_scale, codes, ldc, scales);
    return hipGetLastError();
}

}  // namespace qamw
