// The norms around a block, with its gate and the scale of the stream:
//   b' = b / sqrt(mean b^2 + eps) w_b;  h' = h + scale (gate b');  x = h' / sqrt(mean h'^2 + eps) w, of h' as it is stored.
// Memory bounds it: h, b and a gate of every value are read once, h' and x written once.
#include "qamw_mx4.hpp"

namespace qamw {
namespace {

constexpr int BN_THREADS = 256, BN_WAVES = BN_THREADS / WAVE, BN_SPAN = BN_THREADS * 8;

// The sum over the workgroup in a fixed order, the same in every lane.
__device__ __forceinline__ float sum_of_all(float v, float *part) {
    v = wave_add(v);
    __syncthreads();
    if (threadIdx.x % WAVE == 0) part[threadIdx.x / WAVE] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < BN_WAVES; ++w) s += part[w];
    return s;
}

template <int DTYPE> __device__ __forceinline__ void load_8(const void *from, int64_t at, int there, float (&v)[8]) {
    using E = typename Elem<DTYPE>::type;
    const E *x = static_cast<const E *>(from) + at;
    if (there >= 8) {
        const auto e = *reinterpret_cast<const Unaligned<E, 8> *>(x);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = DTYPE == 1 ? __uint_as_float((uint32_t)e.v[i] << 16) : (float)e.v[i];
        return;
    }
    for (int i = 0; i < 8; ++i) v[i] = i < there ? Elem<DTYPE>::load(x, i) : 0.0f;
}
template <int DTYPE> __device__ __forceinline__ void store_8(void *to, int64_t at, int there, const float (&v)[8]) {
    const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
    store_y4<DTYPE == 1>(to, at, lo, there);
    if (there > 4) store_y4<DTYPE == 1>(to, at + 4, hi, there - 4);
}
template <int DTYPE> __device__ __forceinline__ float rounded(float v) {
    return DTYPE == 1 ? __uint_as_float(bf16_rne_bits(v) << 16) : v;
}

// A workgroup has a row, a thread 8 neighbours of every BN_SPAN.
template <int DTYPE, int OUT>
__global__ __launch_bounds__(BN_THREADS) void k_block_norm(BlockNorm q) {
    __shared__ float part[BN_WAVES];
    __shared__ uint32_t parts[BN_WAVES];
    const int64_t row = blockIdx.x;
    const int64_t at_h = row * q.ldh, at_b = row * q.ldb, at_g = row * q.ldg, at_o = row * q.ldho;
    float r_block = 1.0f;
    if (q.block_weight) {
        float s = 0.0f, v[8];
        for (int64_t j = threadIdx.x * 8; j < q.d; j += BN_SPAN) {
            load_8<DTYPE>(q.block, at_b + j, (int)min((int64_t)8, q.d - j), v);
            for (int i = 0; i < 8; ++i) s = fmaf(v[i], v[i], s);
        }
        r_block = 1.0f / sqrtf(sum_of_all(s, part) / (float)q.d + q.eps);
    }
    // h' of eight columns, as it is stored
    auto stream = [&](int64_t j, int there, float (&v)[8]) {
        load_8<DTYPE>(q.h, at_h + j, there, v);
        if (!q.block) return;
        float b[8], w[8];
        load_8<DTYPE>(q.block, at_b + j, there, b);
        if (q.block_weight) {
            load_8<0>(q.block_weight, j, there, w);
            for (int i = 0; i < 8; ++i) b[i] = b[i] * r_block * w[i];
        }
        if (q.gate) {
            load_8<DTYPE>(q.gate, at_g + j, there, w);
            for (int i = 0; i < 8; ++i) b[i] *= w[i];
        }
        for (int i = 0; i < 8; ++i) v[i] = rounded<DTYPE>(fmaf(q.scale, b[i], v[i]));
    };
    float s = 0.0f;
    for (int64_t j = threadIdx.x * 8; j < q.d; j += BN_SPAN) {
        float v[8];
        const int there = (int)min((int64_t)8, q.d - j);
        stream(j, there, v);
        if (q.block) store_8<DTYPE>(q.h_out, at_o + j, there, v);
        for (int i = 0; i < 8; ++i) s = fmaf(v[i], v[i], s);
    }
    const float r = 1.0f / sqrtf(sum_of_all(s, part) / (float)q.d + q.eps);
    auto normed = [&](int64_t j, int there, float (&v)[8]) {
        float w[8];
        if (q.block) load_8<DTYPE>(q.h_out, at_o + j, there, v);   // this thread's own stores
        else load_8<DTYPE>(q.h, at_h + j, there, v);
        if (q.weight) load_8<0>(q.weight, j, there, w);
        for (int i = 0; i < 8; ++i) {
            v[i] = v[i] * r;
            if (q.weight) v[i] *= w[i];
        }
    };
    uint32_t most = 0;
    if (OUT == 2) {
        float v[8];
        for (int64_t j = threadIdx.x * 8; j < q.d; j += BN_SPAN) {
            normed(j, (int)min((int64_t)8, q.d - j), v);
            for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        }
        most = wave_max(most);
        if (threadIdx.x % WAVE == 0) parts[threadIdx.x / WAVE] = most;
        __syncthreads();
        for (int w = 0; w < BN_WAVES; ++w) most = max(most, parts[w]);
    }
    const Quantiser z(most);
    if (OUT == 2 && threadIdx.x == 0) static_cast<float *>(q.x_scales)[row] = z.scale;
    const int64_t end = OUT == 3 ? (q.d + 511) / 512 * 512 : q.d;   // in 4 bits whole groups of 16 blocks: their scales are all written
    for (int64_t j = threadIdx.x * 8; j < end; j += BN_SPAN) {
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        const int there = (int)min((int64_t)8, q.d - j);
        if (there > 0) normed(j, there, v);
        if (OUT <= 1) store_8<OUT>(q.x, row * q.ldx + j, there, v);
        if (OUT == 2) {
            uint8_t *to = static_cast<uint8_t *>(q.x) + row * q.ldx + j;
            for (int i = 0; i < there && i < 8; ++i) to[i] = (uint8_t)z.code(v[i]);
        }
        if (OUT == 3) {
            uint32_t largest = 0;
            for (int i = 0; i < 8; ++i) largest = max(largest, i < there ? __float_as_uint(v[i]) & 0x7FFFFFFFu : 0);
            const Mx4Scale sc(quad_max(largest));
            for (int i = 0; i < 8; ++i) v[i] = i < there ? v[i] : 0.0f;
            const bool is = j / 32 * 32 < q.d;
            if (is) *reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(q.x) + row * mx4_code_bytes(q.d) + j / 2) = mx4_codes(v, sc);
            if (threadIdx.x % 4 == 0)
                static_cast<uint8_t *>(q.x_scales)[row * mx4_scale_bytes(q.d) + j / 512 * 16 + mx4_scale_at((int)(j % 512 / 32))] = is ? (uint8_t)sc.byte : 0;
        }
    }
}

template <int DTYPE> hipError_t launch_type(const BlockNorm &q) {
    const dim3 g((uint32_t)q.m);
    switch (q.x_dtype) {
    case 0: k_block_norm<DTYPE, 0><<<g, BN_THREADS, 0, q.stream>>>(q); break;
    case 1: k_block_norm<DTYPE, 1><<<g, BN_THREADS, 0, q.stream>>>(q); break;
    case 2: k_block_norm<DTYPE, 2><<<g, BN_THREADS, 0, q.stream>>>(q); break;
    default: k_block_norm<DTYPE, 3><<<g, BN_THREADS, 0, q.stream>>>(q); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_block_norm(const BlockNorm &q) {
    if (q.m == 0) return hipSuccess;
    return q.dtype == 0 ? launch_type<0>(q) : launch_type<1>(q);
}

}  // namespace qamw
