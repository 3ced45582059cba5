// Rows to 4-bit floating point with a scale for every 32 columns, and back.
//   v_j = x_j c_j;  a = max |v| of the block;  e = max(floor(log2 a) - 2, -127);  code_j = the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to v_j 2^-e.
// A wave has 16 blocks of a row, a lane 8 neighbours, four lanes a block.  Memory bounds it: 4 or 2 bytes a value on one side, 17 / 32 on the other.
// 11008 x 4096 bf16 17.9 us and back 18.1, fp32 30 and 45; with stores of 4 bytes, and loads under conditions, it was a third more.
#include "qamw_mx4.hpp"

namespace qamw {
namespace {

constexpr int MQ_THREADS = 256, MQ_WAVES = MQ_THREADS / WAVE, MQ_SPAN = WAVE * 8;

// Group `id` of 512 columns: its row, and the column where the lane's eight begin.
struct Group {
    int64_t row;
    int g, j;
    __device__ __forceinline__ Group(uint32_t id, uint32_t groups) : row(id / groups), g((int)(id % groups)), j(g * MQ_SPAN + (int)(threadIdx.x % WAVE) * 8) {}
};

// EACH groups a wave, all asked for together.  ROWS: 0 of whole eights, 1 of eight columns and more, 2 of fewer.
template <int DTYPE, bool SCALED, int EACH, int ROWS>
__global__ __launch_bounds__(MQ_THREADS) void k_mx4_quantize(const void *X, uint32_t all, uint32_t groups, int d, int64_t ldx, const float *col_scale,
                                                             uint8_t *codes, int64_t ldc, uint8_t *scales, int64_t lds) {
    using E = typename Elem<DTYPE>::type;
    const int lane = threadIdx.x % WAVE;
    const uint32_t id0 = (blockIdx.x * MQ_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE)) * EACH;
    Raw<DTYPE> raw[EACH];
    Raw<0> col[EACH];
    if (ROWS != 2)
#pragma unroll
        for (int n = 0; n < EACH; ++n) {
            const Group a(min(id0 + n, all - 1), groups);
            raw[n].load(static_cast<const E *>(X) + a.row * ldx, a.j, d);
            if (SCALED) col[n].load(col_scale, a.j, d);
        }
    uint32_t code[EACH], byte[EACH];
#pragma unroll
    for (int n = 0; n < EACH; ++n) {
        const Group a(min(id0 + n, all - 1), groups);
        float v[8], c[8];
        if (ROWS == 2) {
            for (int i = 0; i < 8; ++i) {
                const bool is = a.j + i < d;
                v[i] = is ? Elem<DTYPE>::load(X, a.row * ldx + a.j + i) : 0.0f;
                if (SCALED) c[i] = is ? col_scale[a.j + i] : 0.0f;
            }
        } else {
            values_of<DTYPE, ROWS == 1>(raw[n], d - a.j, v);
            if (SCALED) values_of<0, ROWS == 1>(col[n], d - a.j, c);
        }
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (SCALED) v[i] *= c[i];
            most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        }
        const Mx4Scale s(quad_max(most));
        code[n] = mx4_codes(v, s);
        byte[n] = s.byte;                                   // 0 where no column is
    }
    if constexpr (EACH == 4) {
        // Four lanes have a block of each of four groups, and exchange them: each gets a whole block of one, which is a store of 16 bytes for four of 4.
        auto swap = [](uint32_t &lo, uint32_t &hi, bool up, auto move) {
            const uint32_t got = (uint32_t)move((int)(up ? lo : hi));
            lo = up ? got : lo;
            hi = up ? hi : got;
        };
        const int q = lane % 4;
        auto one = [](int v) { return dpp_move<DPP_XOR1>(v); };
        auto two = [](int v) { return dpp_move<DPP_XOR2>(v); };
        swap(code[0], code[1], q & 1, one);
        swap(code[2], code[3], q & 1, one);
        swap(code[0], code[2], q & 2, two);
        swap(code[1], code[3], q & 2, two);
        const uint32_t mine = q & 2 ? (q & 1 ? byte[3] : byte[2]) : q & 1 ? byte[1] : byte[0];
        const uint32_t id = id0 + q;
        if (id >= all) return;
        const int64_t row = id / groups;
        const int g = (int)(id % groups), block = g * 16 + lane / 4;
        if (block * 32 < d) *reinterpret_cast<uint4 *>(codes + row * ldc + block * 16) = {code[0], code[1], code[2], code[3]};
        scales[row * lds + g * 16 + mx4_scale_at(lane / 4)] = (uint8_t)mine;
    } else {
        const Group a(min(id0, all - 1), groups);
        if (id0 >= all) return;
        if (a.j / 32 * 32 < d) *reinterpret_cast<uint32_t *>(codes + a.row * ldc + a.j / 2) = code[0];
        if (lane % 4 == 0) scales[a.row * lds + a.g * 16 + mx4_scale_at(lane / 4)] = (uint8_t)byte[0];
    }
}

// Back, a lane 16 bytes of the result at a time: 8 values of bf16, or 4 of fp32 from each half of the group.  With all eight its own, and so half of every 32
// bytes a store, fp32 took 16.2 us for 2000 x 5120, now 13.5.  Four groups a wave, as above, brought nothing.
template <bool OBF16>
__global__ __launch_bounds__(MQ_THREADS) void k_mx4_dequantize(const uint8_t *codes, int64_t ldc, const uint8_t *scales, int64_t lds, uint32_t all,
                                                               uint32_t groups, int d, void *out, int64_t ldo) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const int lane = threadIdx.x % WAVE;
    for (uint32_t id = blockIdx.x * MQ_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE); id < all; id += gridDim.x * MQ_WAVES) {
        const Group a(id, groups);
        const uint8_t *from = codes + a.row * ldc, *scale = scales + a.row * lds + a.g * 16;
        if constexpr (OBF16) {
            const uint32_t c = *reinterpret_cast<const uint32_t *>(from + min((int64_t)a.j / 2, ldc - 4));   // past the end: the row's last ones
            const float p = mx4_power(scale[mx4_scale_at(lane / 4)]);
            const f2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
            const f2 v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
            const float lo[4] = {v0[0] * p, v0[1] * p, v1[0] * p, v1[1] * p}, hi[4] = {v2[0] * p, v2[1] * p, v3[0] * p, v3[1] * p};
            const int64_t at = a.row * ldo + a.j;
            const int there = d - a.j;
            if (there >= 8) {
                const uint4 eight = {pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3])};
                *reinterpret_cast<Unaligned<uint16_t, 8> *>(static_cast<uint16_t *>(out) + at) = __builtin_bit_cast(Unaligned<uint16_t, 8>, eight);
            } else if (there > 0) {
                store_y4<true>(out, at, lo, there);
                if (there > 4) store_y4<true>(out, at + 4, hi, there - 4);
            }
        } else {
            uint32_t c[2], byte[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = a.g * MQ_SPAN + h * 256 + lane * 4;
                c[h] = *reinterpret_cast<const uint16_t *>(from + min((int64_t)j / 2, ldc - 2));
                byte[h] = scale[mx4_scale_at(h * 8 + lane / 8)];
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = a.g * MQ_SPAN + h * 256 + lane * 4;
                const float p = mx4_power(byte[h]);
                const f2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[h], 1.0f, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[h], 1.0f, 1);
                const float v[4] = {v0[0] * p, v0[1] * p, v1[0] * p, v1[1] * p};
                if (j < d) store_y4<false>(out, a.row * ldo + j, v, d - j);
            }
        }
    }
}

// Four groups a wave where that leaves enough waves to fill half of the chip: bf16 4001 x 4096 6.9 us (8.1 with one), 2000 4.2 (4.3), 1000 3.05 (2.95).
constexpr int64_t MQ_MANY = 4 * 4096;
constexpr int64_t MQ_BLOCKS = 0xFFFFFF;                    // threads of a launch are counted in 32 bits
int64_t groups_of(int d) { return ((int64_t)d + MQ_SPAN - 1) / MQ_SPAN; }   // at most 2^22 rows of 2^8

}  // namespace

hipError_t launch_mx4_quantize(const void *X, int dtype, int64_t m, int d, int64_t ldx, const float *col_scale, uint8_t *codes, uint8_t *scales,
                               hipStream_t stream) {
    if (m == 0) return hipSuccess;
    const int64_t ldc = mx4_code_bytes(d), lds = mx4_scale_bytes(d);
    const int64_t groups = groups_of(d), all = m * groups, each = all >= MQ_MANY ? 4 : 1, blocks = (all + MQ_WAVES * each - 1) / (MQ_WAVES * each);
    if (blocks > MQ_BLOCKS) return hipErrorNotSupported;
    auto go = [&](auto kernel) {
        kernel<<<(uint32_t)blocks, MQ_THREADS, 0, stream>>>(X, (uint32_t)all, (uint32_t)groups, d, ldx, col_scale, codes, ldc, scales, lds);
    };
    auto by_rows = [&](auto type, auto scaled) {
        constexpr int T = decltype(type)::value;
        constexpr bool S = decltype(scaled)::value;
        if (d < 8) each == 4 ? go(k_mx4_quantize<T, S, 4, 2>) : go(k_mx4_quantize<T, S, 1, 2>);
        else if (d % 8) each == 4 ? go(k_mx4_quantize<T, S, 4, 1>) : go(k_mx4_quantize<T, S, 1, 1>);
        else each == 4 ? go(k_mx4_quantize<T, S, 4, 0>) : go(k_mx4_quantize<T, S, 1, 0>);
    };
    auto by_scale = [&](auto type) { col_scale ? by_rows(type, std::true_type{}) : by_rows(type, std::false_type{}); };
    dtype == 0 ? by_scale(std::integral_constant<int, 0>{}) : by_scale(std::integral_constant<int, 1>{});
    return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t m, int d, void *out, int out_dtype, int64_t ldo,
                                 hipStream_t stream) {
    if (m == 0) return hipSuccess;
    const int64_t ldc = mx4_code_bytes(d), lds = mx4_scale_bytes(d);
    const int64_t groups = groups_of(d), all = m * groups, need = (all + MQ_WAVES - 1) / MQ_WAVES, blocks = need < MQ_BLOCKS ? need : MQ_BLOCKS;
    auto go = [&](auto kernel) { kernel<<<(uint32_t)blocks, MQ_THREADS, 0, stream>>>(codes, ldc, scales, lds, (uint32_t)all, (uint32_t)groups, d, out, ldo); };
    out_dtype == 1 ? go(k_mx4_dequantize<true>) : go(k_mx4_dequantize<false>);
    return hipGetLastError();
}

}  // namespace qamw
