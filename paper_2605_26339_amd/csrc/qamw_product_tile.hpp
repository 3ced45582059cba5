// What the product kernels share: operand types, the tile that a workgroup has, and the last step.
#pragma once
#include "qamw_product.hpp"

namespace qamw {

typedef int pr_i32x4_t __attribute__((ext_vector_type(4)));
typedef float pr_f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 pr_bf16x8_t __attribute__((ext_vector_type(8)));

// 16 rows of W times 16 rows of X over 64 bytes of each: lane l holds bytes 16 (l / 16) .. + 16 of row l % 16 of both operands,
// and gets W rows 4 (l / 16) .. + 4 of the column that is X row l % 16.  int8 and bf16 lay their bytes out alike.
template <bool I8> struct Mfma;
template <> struct Mfma<true> {
    using acc_t = pr_i32x4_t;
    using elem_t = int8_t;
    static constexpr int ELEM = 1;
    static __device__ __forceinline__ acc_t mul(pr_i32x4_t w, pr_i32x4_t x, acc_t c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, c, 0, 0, 0);
    }
};
template <> struct Mfma<false> {
    using acc_t = pr_f32x4_t;
    using elem_t = uint16_t;
    static constexpr int ELEM = 2;
    static __device__ __forceinline__ acc_t mul(pr_i32x4_t w, pr_i32x4_t x, acc_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pr_bf16x8_t, w), __builtin_bit_cast(pr_bf16x8_t, x), c, 0, 0, 0);
    }
};

// The device side of a Product.
struct ProductArgs {
    const char *X, *W;
    const float *x_scales, *w_scales;
    const int32_t *rows, *offsets;
    void *Y;
    int64_t ldx, ldw, expert_stride;     // in bytes
    int64_t ldy;                         // in elements
    int m, x_rows, n_experts, d_out, d_in;
};

inline ProductArgs args_of(const Product &p) {
    const int64_t e = p.i8 ? 1 : 2;
    return {static_cast<const char *>(p.X), static_cast<const char *>(p.W), p.x_scales, p.w_scales, p.rows, p.offsets, p.Y,
            p.ldx * e, p.ldw * e, p.expert_stride * e, p.ldy, p.m, p.x_rows, p.n_experts, p.d_out, p.d_in};
}

// Rows row0 .. row0 + n of the product, which are expert `expert`'s; n = 0: nothing to do.
struct RowTile {
    int expert, row0, n;
};

// The tiles of at most BM rows are counted over the experts in order; an expert has the row tiles first .. first + tiles.  Every wave
// of a workgroup finds them by itself: a lane has an expert, and a prefix sum over lanes says where its tiles begin.  Offsets are
// held within 0 .. m, so that no value of theirs makes a tile of rows that are not there.
struct ExpertTiles {
    int expert, first, tiles, start, end;      // rows start .. end
};
template <int BM, typename Visit> __device__ __forceinline__ int visit_tiles(const ProductArgs &a, Visit visit) {
    const int lane = threadIdx.x % WAVE;
    int before = 0;
    for (int e0 = 0; e0 < a.n_experts; e0 += WAVE) {
        const int e = e0 + lane;
        const bool is = e < a.n_experts;
        const int lo = is ? min(max(a.offsets[e], 0), a.m) : 0;
        const int hi = is ? min(max(a.offsets[e + 1], lo), a.m) : lo;
        const int tiles = (hi - lo) / BM + ((hi - lo) % BM != 0);
        int upto = tiles;
        for (int d = 1; d < WAVE; d <<= 1) {
            const int v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        if (visit(e0, before, lo, hi, tiles, upto)) return -1;
        before += __builtin_amdgcn_readlane(upto, WAVE - 1);
    }
    return before;
}
// All row tiles there are.
template <int BM> __device__ __forceinline__ int count_tiles(const ProductArgs &a) {
    if (!a.offsets) return a.m / BM + (a.m % BM != 0);
    return visit_tiles<BM>(a, [](int, int, int, int, int, int) { return false; });
}
// The expert that has row tile t; tiles = 0 if none has.
template <int BM> __device__ __forceinline__ ExpertTiles find_expert(const ProductArgs &a, int t) {
    if (!a.offsets) return {0, 0, a.m / BM + (a.m % BM != 0), 0, a.m};
    ExpertTiles found = {0, 0, 0, 0, 0};
    visit_tiles<BM>(a, [&](int e0, int before, int lo, int hi, int tiles, int upto) {
        const unsigned long long past = __ballot(before + upto > t);
        if (!past) return false;
        const int l = __ffsll((long long)past) - 1;
        found = {e0 + l, before + __builtin_amdgcn_readlane(upto - tiles, l), __builtin_amdgcn_readlane(tiles, l),
                 __builtin_amdgcn_readlane(lo, l), __builtin_amdgcn_readlane(hi, l)};
        return true;
    });
    return found;
}
template <int BM> __device__ __forceinline__ RowTile find_tile(const ProductArgs &a, int t) {
    const ExpertTiles e = find_expert<BM>(a, t);
    if (t - e.first >= e.tiles) return {0, 0, 0};
    const int row0 = e.start + (t - e.first) * BM;
    return {e.expert, row0, min(BM, e.end - row0)};
}

// Most row tiles that there can be.
inline int64_t most_row_tiles(const Product &p, int bm) {
    const int64_t m = p.m;
    return p.offsets ? m / bm + (m < p.n_experts ? m : p.n_experts) : (m + bm - 1) / bm;
}

// The largest of a wave's values, in every lane: within 16 lanes by DPP, then over the four of them.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));    // lane ^ 1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));    // lane ^ 2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false));   // the other four of eight
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false));   // the other eight of sixteen
    const uint32_t a = __builtin_amdgcn_readlane((int)v, 0), b = __builtin_amdgcn_readlane((int)v, 16);
    const uint32_t c = __builtin_amdgcn_readlane((int)v, 32), d = __builtin_amdgcn_readlane((int)v, 48);
    return max(max(a, b), max(c, d));
}

// Eight neighbours of a row as they are read, and as fp32.
template <int DTYPE> struct Eight;
template <> struct Eight<0> {
    pr_i32x4_t a, b;
    template <typename R> __device__ __forceinline__ void load(R from, uint32_t at) {       // a buffer, a byte offset
        a = __builtin_bit_cast(pr_i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from, (int)at, 0, 0));
        b = __builtin_bit_cast(pr_i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from, (int)at, 16, 0));
    }
    __device__ __forceinline__ float value(int i) const { return __int_as_float(i < 4 ? a[i & 3] : b[i & 3]); }
};
template <> struct Eight<1> {
    pr_i32x4_t a;
    template <typename R> __device__ __forceinline__ void load(R from, uint32_t at) {
        a = __builtin_bit_cast(pr_i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from, (int)at, 0, 0));
    }
    __device__ __forceinline__ float value(int i) const {
        return __int_as_float(i & 1 ? (int)((uint32_t)a[i >> 1] & 0xFFFF0000u) : a[i >> 1] << 16);
    }
};

// Steps of the quantisation to 8 bits: the scale and the factor from the largest |v| (its bits order finite values, infinity, NaNs).
struct Quantiser {
    float inv, scale;                     // inv = 0: all codes are 0
    __device__ __forceinline__ explicit Quantiser(uint32_t most) {
        const float a = __uint_as_float(most);
        const bool finite = most < 0x7F800000u, some = finite && a >= 0x1p-110f;
        inv = some ? 127.0f / a : 0.0f;
        scale = some ? a / 127.0f : finite ? 0.0f : __uint_as_float(0x7FC00000u);
    }
    __device__ __forceinline__ uint32_t code(float v) const { return inv != 0.0f ? (uint32_t)(int)rintf(v * inv) & 255u : 0u; }
};

// g / (1 + exp(-g)) with the hardware's exponential and reciprocal, for a fifth of the instructions.  Relative error, measured from -110 to
// 110: under 1.1 (|g| + 8) 2^-24 for g < 0, since the exponential's argument is rounded and its size multiplies that, 2.4 * 2^-24 for g >= 0.  From
// g = -87.34 down the reciprocal would be subnormal and is 0, where silu is under 1.1e-36 in size; exp overflows to infinity, whose reciprocal is 0.
__device__ __forceinline__ float silu(float g) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

// Two values rounded to bf16 (nearest, ties to even).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{lo, hi}), b2));
}

// Four neighbours of a row of Y, or of the scales of W, wherever they lie: the memory instructions take any address.
template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Unaligned {
    T v[N];
};

template <bool BF16> __device__ __forceinline__ void store_y4(void *Y, int64_t at, const float (&v)[4], int n) {
    if (n >= 4) {
        if (BF16) {
            const uint2 two = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            *reinterpret_cast<Unaligned<uint16_t, 4> *>(reinterpret_cast<uint16_t *>(Y) + at) = __builtin_bit_cast(Unaligned<uint16_t, 4>, two);
        } else {
            *reinterpret_cast<Unaligned<float, 4> *>(reinterpret_cast<float *>(Y) + at) = Unaligned<float, 4>{{v[0], v[1], v[2], v[3]}};
        }
        return;
    }
    for (int q = 0; q < 3; ++q)
        if (q < n) {
            if (BF16) reinterpret_cast<uint16_t *>(Y)[at + q] = (uint16_t)bf16_rne_bits(v[q]);
            else reinterpret_cast<float *>(Y)[at + q] = v[q];
        }
}

template <bool BF16> __device__ __forceinline__ void store_y(void *Y, int64_t at, float v) {
    if (BF16)
        reinterpret_cast<uint16_t *>(Y)[at] = (uint16_t)bf16_rne_bits(v);
    else
        reinterpret_cast<float *>(Y)[at] = v;
}

}  // namespace qamw
