// Rows to 4-bit floating point with a scale for every 32 columns, and back.
//   v_j = x_j c_j;  a = max |v| of the block;  e = max(floor(log2 a) - 2, -127);  code_j = the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to v_j 2^-e.
// A wave has 16 blocks of a row, a lane 8 neighbours, four lanes a block.  Memory bounds it: 4 or 2 bytes a value on one side, 17 / 32 on the other.
#include "qamw_mx4.hpp"

namespace qamw {
namespace {

constexpr int MQ_THREADS = 256, MQ_WAVES = MQ_THREADS / WAVE, MQ_SPAN = WAVE * 8;

template <int DTYPE, bool SCALED>
__global__ __launch_bounds__(MQ_THREADS) void k_mx4_quantize(const void *X, int64_t waves, int groups, int d, int64_t ldx, const float *col_scale,
                                                             uint8_t *codes, int64_t ldc, uint8_t *scales, int64_t lds) {
    using E = typename Elem<DTYPE>::type;
    const int lane = threadIdx.x % WAVE;
    const int64_t id = (int64_t)blockIdx.x * MQ_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    if (id >= waves) return;
    const int64_t row = id / groups;
    const int g = (int)(id % groups);
    const int64_t j = (int64_t)g * MQ_SPAN + lane * 8;
    const E *x = static_cast<const E *>(X) + row * ldx + j;
    float v[8];
    if (j + 8 <= d) {                                       // wherever they lie: the memory instructions take any address
        const auto e = *reinterpret_cast<const Unaligned<E, 8> *>(x);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = DTYPE == 1 ? __uint_as_float((uint32_t)e.v[i] << 16) : (float)e.v[i];
        if (SCALED) {
            const auto c = *reinterpret_cast<const Unaligned<float, 8> *>(col_scale + j);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= c.v[i];
        }
    } else
        for (int i = 0; i < 8; ++i) v[i] = j + i < d ? Elem<DTYPE>::load(x, i) * (SCALED ? col_scale[j + i] : 1.0f) : 0.0f;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    const Mx4Scale s(quad_max(most));
    const int64_t block = j / 32;
    if (block * 32 < d) *reinterpret_cast<uint32_t *>(codes + row * ldc + j / 2) = mx4_codes(v, s);
    if (lane % 4 == 0) scales[row * lds + g * 16 + mx4_scale_at(lane / 4)] = block * 32 < d ? (uint8_t)s.byte : 0;
}

template <bool OBF16>
__global__ __launch_bounds__(MQ_THREADS) void k_mx4_dequantize(const uint8_t *codes, int64_t ldc, const uint8_t *scales, int64_t lds, int64_t waves,
                                                               int groups, int d, void *out, int64_t ldo) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const int lane = threadIdx.x % WAVE;
    const int64_t id = (int64_t)blockIdx.x * MQ_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    if (id >= waves) return;
    const int64_t row = id / groups;
    const int g = (int)(id % groups);
    const int64_t j = (int64_t)g * MQ_SPAN + lane * 8;
    if (j >= d) return;
    const uint32_t c = *reinterpret_cast<const uint32_t *>(codes + row * ldc + j / 2);
    const float p = mx4_power(scales[row * lds + g * 16 + mx4_scale_at(lane / 4)]);
    const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
    const f2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
    const float lo[4] = {a[0] * p, a[1] * p, b[0] * p, b[1] * p}, hi[4] = {e[0] * p, e[1] * p, f[0] * p, f[1] * p};
    const int64_t at = row * ldo + j;
    const int there = (int)min((int64_t)8, d - j);
    store_y4<OBF16>(out, at, lo, there);
    if (there > 4) store_y4<OBF16>(out, at + 4, hi, there - 4);
}

}  // namespace

hipError_t launch_mx4_quantize(const void *X, int dtype, int64_t m, int d, int64_t ldx, const float *col_scale, uint8_t *codes, uint8_t *scales,
                               hipStream_t stream) {
    if (m == 0) return hipSuccess;
    const int64_t groups = ((int64_t)d + MQ_SPAN - 1) / MQ_SPAN, waves = m * groups, blocks = (waves + MQ_WAVES - 1) / MQ_WAVES;
    if (blocks * MQ_THREADS > 0xFFFFFFFFll) return hipErrorNotSupported;
    const int64_t ldc = mx4_code_bytes(d), lds = mx4_scale_bytes(d);
    const dim3 g((uint32_t)blocks);
    if (dtype == 0) {
        if (col_scale) k_mx4_quantize<0, true><<<g, MQ_THREADS, 0, stream>>>(X, waves, (int)groups, d, ldx, col_scale, codes, ldc, scales, lds);
        else k_mx4_quantize<0, false><<<g, MQ_THREADS, 0, stream>>>(X, waves, (int)groups, d, ldx, col_scale, codes, ldc, scales, lds);
    } else {
        if (col_scale) k_mx4_quantize<1, true><<<g, MQ_THREADS, 0, stream>>>(X, waves, (int)groups, d, ldx, col_scale, codes, ldc, scales, lds);
        else k_mx4_quantize<1, false><<<g, MQ_THREADS, 0, stream>>>(X, waves, (int)groups, d, ldx, col_scale, codes, ldc, scales, lds);
    }
    return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t m, int d, void *out, int out_dtype, int64_t ldo,
                                 hipStream_t stream) {
    if (m == 0) return hipSuccess;
    const int64_t groups = ((int64_t)d + MQ_SPAN - 1) / MQ_SPAN, waves = m * groups, blocks = (waves + MQ_WAVES - 1) / MQ_WAVES;
    if (blocks * MQ_THREADS > 0xFFFFFFFFll) return hipErrorNotSupported;
    const int64_t ldc = mx4_code_bytes(d), lds = mx4_scale_bytes(d);
    const dim3 g((uint32_t)blocks);
    if (out_dtype == 1) k_mx4_dequantize<true><<<g, MQ_THREADS, 0, stream>>>(codes, ldc, scales, lds, waves, (int)groups, d, out, ldo);
    else k_mx4_dequantize<false><<<g, MQ_THREADS, 0, stream>>>(codes, ldc, scales, lds, waves, (int)groups, d, out, ldo);
    return hipGetLastError();
}

}  // namespace qamw
