// Rows in 4-bit floating point with a scale for every 32 columns: their layout and their quantisation.
#pragma once
#include "qamw_product_tile.hpp"

namespace qamw {

// Where the scale of block b is: the matrix instruction takes the scales of four neighbouring blocks from four groups of lanes, and one of the four bytes
// of a register, so that a lane's blocks b % 4 of four such instructions are one dword.
inline __host__ __device__ int mx4_scale_at(int b) { return b / 16 * 16 + b % 4 * 4 + b % 16 / 4; }

// A block's exponent from its largest |v| (the bits; infinities and NaNs are the largest of all): 2^e times 6 is the largest value, so that one of
// 2^(floor(log2 |v|) + 1) is rounded down to it.
struct Mx4Scale {
    uint32_t byte;                       // e + 127; 255: not a number
    float inv;                           // 2^-e, or 0 where all codes are 0
    __device__ __forceinline__ explicit Mx4Scale(uint32_t most) {
        const uint32_t p = most >> 23;                     // floor(log2) + 127, or 0 below the smallest normal number, where e is -127 in any case
        byte = p >= 255 ? 255 : p > 2 ? p - 2 : 0;
        inv = p >= 255 ? 0.0f : __uint_as_float((254 - byte) << 23);
    }
};
// Eight neighbours to codes, the first in the lowest bits.  The conversion rounds to nearest, ties to even, and what is beyond 6 to 6.
__device__ __forceinline__ uint32_t mx4_codes(const float (&v)[8], const Mx4Scale &s) {
    if (s.byte == 255) return 0;
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0] * s.inv, v[1] * s.inv, 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2] * s.inv, v[3] * s.inv, 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4] * s.inv, v[5] * s.inv, 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6] * s.inv, v[7] * s.inv, 1.0f, 3);
    return c;
}
// The largest of four neighbouring lanes' values.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));
}
// 2^(byte - 127)
__device__ __forceinline__ float mx4_power(uint32_t byte) {
    return __uint_as_float(byte == 255 ? 0x7FC00000u : byte ? byte << 23 : 0x00400000u);
}

// Eight neighbours of a row of d >= 8, as they are read, wherever they begin: of a row's last ones, or where none are left, the eight that end with the row.
// Loads under a condition would be waited for one after the other.
template <int DTYPE> struct Raw {
    using E = typename Elem<DTYPE>::type;
    Unaligned<E, 8> e;
    __device__ __forceinline__ void load(const void *row, int j, int d) { e = *reinterpret_cast<const Unaligned<E, 8> *>(static_cast<const E *>(row) + min(j, d - 8)); }
    __device__ __forceinline__ float value(int k) const { return DTYPE == 1 ? __uint_as_float((uint32_t)e.v[k] << 16) : (float)e.v[k]; }
};
// As values: the first `there` of them, after the last 8 - there of what was read; zeros behind.
template <int DTYPE, bool RAGGED> __device__ __forceinline__ void values_of(const Raw<DTYPE> &raw, int there, float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = there > 0 ? raw.value(k) : 0.0f;
    if (!RAGGED) return;                                                       // rows of whole eights
    const int by = there >= 8 || there <= 0 ? 0 : 8 - there;
#pragma unroll
    for (int bit = 1; bit < 8; bit <<= 1)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = by & bit ? (k + bit < 8 ? v[(k + bit) & 7] : 0.0f) : v[k];
}

}  // namespace qamw
