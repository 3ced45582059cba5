// Products of served layers: Y = X W^T with W in 8-bit integers or bf16, one matrix or one for each expert.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "qamw_common.hpp"

namespace qamw {

// What the operands are.  Rows in 4 bits are rows of bytes: their d_in and leading dimensions are those of their codes.
enum { PRODUCT_BF16 = 0, PRODUCT_I8 = 1, PRODUCT_MX4 = 2 };

// One call.  Without offsets: one group of m rows.  With offsets: rows offsets[e] .. offsets[e + 1] belong to expert e.
struct Product {
    const void *X = nullptr;             // int8 codes, bf16 or codes of 4 bits
    const float *x_scales = nullptr;     // int8: one for each row of X
    const int32_t *rows = nullptr;       // row of X for each row of the product, nullable
    const void *W = nullptr;             // gated: the gate's d_out rows, then the up projection's
    const float *w_scales = nullptr;     // int8: one for each row of W, expert after expert
    const int32_t *offsets = nullptr;    // device, n_experts + 1, nullable
    void *Y = nullptr;
    int64_t ldx = 0, ldw = 0, expert_stride = 0, ldy = 0;
    int m = 0, x_rows = 0, n_experts = 1, d_out = 0, d_in = 0;
    int kind = PRODUCT_BF16;
    bool gated = false, y_bf16 = false;
    const uint8_t *x_blocks = nullptr, *w_blocks = nullptr;   // 4 bits: the scales of blocks, as the rows of X and W
    int block_bytes = 0;                 // of a row
    int64_t elem() const { return kind == PRODUCT_BF16 ? 2 : 1; }
    void *scratch = nullptr;             // product_scratch_bytes(), nullable: the product is not parted then
    hipStream_t stream = nullptr;
};

hipError_t launch_product(const Product &p);
int product_tile_rows();                                                // set by qamw_set_kernel_path(): products of many rows by such tiles; 0: as estimated
// What launch_product() would take for operands that product_wide_supported(); may_part: with scratch.
void product_plan(int m, int n_experts, bool grouped, int d_out, int d_in, bool gated, int kind, bool may_part, int (&out)[3]);
size_t product_scratch_bytes(int m, int d_out, int d_in, bool gated, int kind);   // of an int8 product of one group, or one in 4 bits
// Row of the sums of a part of the columns, in 32-bit words: whole 16 bytes; where the up projection's follow the gate's, four of them
// are read together from anywhere.
inline int64_t parts_row(int64_t d_out, bool gated) { return (d_out * (gated ? 2 : 1) + 3 + (gated ? 3 : 0)) / 4 * 4; }
// More LDS than the 64 KB that a workgroup has without asking, asked for once on a device.
struct MoreLds {
    std::atomic<uint64_t> done{0};
    hipError_t ask(const void *kernel, int bytes) {
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorNotSupported;
        if (!(done.load(std::memory_order_acquire) & (1ull << dev))) {
            const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
            if (e != hipSuccess) return e;
            done.fetch_or(1ull << dev, std::memory_order_release);
        }
        return hipSuccess;
    }
};
// The kernels by what they are for.  wide and few: products that product_wide_supported(), tile_rows of 16 / 32 / 64 and 64 / 128 / 256.
bool product_wide_supported(const Product &p);
hipError_t launch_product_wide(const Product &p, int tile_rows, int parts);
hipError_t launch_product_few(const Product &p, int tile_rows, bool pair);   // pair: 4 bits, tiles of 16 or 32 rows, not gated: 32 rows of W a wave
// Waves that share a tile of outputs: enough for all of memory's bandwidth, about 8 on every CU, while a share has four units.
inline int few_split(int64_t tiles, int units, int waves) {
    int split = 1;
    while (split < waves && tiles * split < 2048 && units >= split * 4) split *= 2;
    return split;
}
// The product of rows that are quantised in the same launch; W as launch_product_few() needs it.
bool product_from_floats_supported(const Product &p, const void *X, int dtype, int columns, int64_t ldx, const float *col_scale);
hipError_t launch_product_from_floats(const Product &p, const void *X, int dtype, int columns, int64_t ldx, const float *col_scale);
hipError_t launch_int8_quantize(const void *X, int dtype, int64_t m, int d, int64_t ldx, const float *col_scale, int8_t *codes,
                                int64_t ldc, float *scales, hipStream_t stream);

// Rows in 4-bit floating point with a scale for every 32 columns.
// A row's codes are whole 16 bytes, a block of 32 columns each; its scales whole 16 bytes, 16 blocks each.
inline __host__ __device__ int64_t mx4_code_bytes(int64_t d) { return (d + 31) / 32 * 16; }
inline __host__ __device__ int64_t mx4_scale_bytes(int64_t d) { return (d + 511) / 512 * 16; }
hipError_t launch_mx4_quantize(const void *X, int dtype, int64_t m, int d, int64_t ldx, const float *col_scale, uint8_t *codes, uint8_t *scales,
                               hipStream_t stream);
hipError_t launch_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t m, int d, void *out, int out_dtype, int64_t ldo, hipStream_t stream);
// Norms around a block.  Null: without block, block_weight, gate, weight.
struct BlockNorm {
    const void *h = nullptr, *block = nullptr, *gate = nullptr;
    const float *block_weight = nullptr, *weight = nullptr;
    void *h_out = nullptr, *x = nullptr, *x_scales = nullptr;
    int64_t ldh = 0, ldb = 0, ldg = 0, ldho = 0, ldx = 0;
    int dtype = 0, x_dtype = 0, m = 0, d = 0;     // x_dtype: 0 fp32, 1 bf16, 2 int8, 3 4 bits
    float scale = 1.0f, eps = 0.0f;
    hipStream_t stream = nullptr;
};
hipError_t launch_block_norm(const BlockNorm &p);

// Routed experts.
struct RouteProblem {
    const void *logits = nullptr;
    int dtype = 0, m = 0, n_experts = 0, k = 0;
    int64_t ld = 0;
    bool renormalise = false;
    int32_t *experts = nullptr, *offsets = nullptr, *rows = nullptr, *positions = nullptr;
    float *weights = nullptr;
    uint8_t *counts = nullptr;           // scratch
    hipStream_t stream = nullptr;
    // by scores: choices by the logits alone where it is not set
    bool scored = false, softmax = false;
    const float *bias = nullptr;
    int groups = 1, top_groups = 1, group_top = 1;
    float scale = 1.0f;
};
size_t route_workspace_bytes(int m, int n_experts, int k);
hipError_t launch_route(const RouteProblem &p);
hipError_t launch_combine(const void *Y, int dtype, int64_t y_rows, int64_t ldy, const int32_t *positions, const float *weights, int m,
                          int k, int d, void *out, int out_dtype, int64_t ldo, hipStream_t stream);

}  // namespace qamw
