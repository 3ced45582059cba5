// Products of served layers: Y = X W^T with W in 8-bit integers or bf16, one matrix or one for each expert.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "qamw_common.hpp"

namespace qamw {

// One call.  Without offsets: one group of m rows.  With offsets: rows offsets[e] .. offsets[e + 1] belong to expert e.
struct Product {
    const void *X = nullptr;             // int8 codes or bf16
    const float *x_scales = nullptr;     // int8: one for each row of X
    const int32_t *rows = nullptr;       // row of X for each row of the product, nullable
    const void *W = nullptr;             // gated: the gate's d_out rows, then the up projection's
    const float *w_scales = nullptr;     // int8: one for each row of W, expert after expert
    const int32_t *offsets = nullptr;    // device, n_experts + 1, nullable
    void *Y = nullptr;
    int64_t ldx = 0, ldw = 0, expert_stride = 0, ldy = 0;
    int m = 0, x_rows = 0, n_experts = 1, d_out = 0, d_in = 0;
    bool i8 = false, gated = false, y_bf16 = false;
    void *scratch = nullptr;             // product_scratch_bytes(), nullable: the product is not parted then
    hipStream_t stream = nullptr;
};

hipError_t launch_product(const Product &p);
int product_tile_rows();                                                // set by qamw_set_kernel_path(): products of many rows by such tiles; 0: as estimated
// What launch_product() would take for operands that product_wide_supported(); may_part: with scratch.
void product_plan(int m, int n_experts, bool grouped, int d_out, int d_in, bool gated, bool i8, bool may_part, int (&out)[3]);
size_t product_scratch_bytes(int m, int d_out, int d_in, bool gated);   // of an int8 product of one group
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
hipError_t launch_product_few(const Product &p, int tile_rows);
// Waves that share a tile of outputs: enough for all of memory's bandwidth, about 8 on every CU, while a share has four units.
inline int few_split(int64_t tiles, int units, int waves) {
    int split = 1;
    while (split < waves && tiles * split < 2048 && units >= split * 4) split *= 2;
    return split;
}
// The product of rows that are quantised in the same launch; W as launch_product_few() needs it.
bool product_from_floats_supported(const Product &p, const void *X, int dtype, int64_t ldx, const float *col_scale);
hipError_t launch_product_from_floats(const Product &p, const void *X, int dtype, int64_t ldx, const float *col_scale);
hipError_t launch_int8_quantize(const void *X, int dtype, int64_t m, int d, int64_t ldx, const float *col_scale, int8_t *codes,
                                int64_t ldc, float *scales, hipStream_t stream);

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
};
size_t route_workspace_bytes(int m, int n_experts, int k);
hipError_t launch_route(const RouteProblem &p);
hipError_t launch_combine(const void *Y, int dtype, int64_t y_rows, int64_t ldy, const int32_t *positions, const float *weights, int m,
                          int k, int d, void *out, int out_dtype, int64_t ldo, hipStream_t stream);

}  // namespace qamw
