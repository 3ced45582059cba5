// Y = X W^T with both in 4-bit floating point, one matrix or one for each expert.
//
// A workgroup has 64 rows of W and 64 of X, a wave 32 of each, and steps over 512 columns at a time, which is a dword of scales a lane.  Operands come
// from memory to registers: a lane's 16 bytes of codes are a block of 32 columns.
#include "qamw_mx4.hpp"

namespace qamw {
namespace {

constexpr int MP_TILE = 64, MP_THREADS = 256;

template <bool GATED, bool YBF16>
__global__ __launch_bounds__(MP_THREADS) void k_mx4_product(ProductArgs a, int col_tiles) {
    const int t = (int)(blockIdx.x / (uint32_t)col_tiles), ct = (int)(blockIdx.x % (uint32_t)col_tiles);
    const RowTile rt = find_tile<MP_TILE>(a, t);
    if (rt.n <= 0) return;
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, wn = wave & 1, wm = wave >> 1, fr = lane & 15, block = lane >> 4;
    // row r of the tile's 64 rows of W; gated: 16 of the gate, then the same 16 of the up projection
    auto out_of = [&](int r) { return GATED ? ct * 32 + (r >> 5) * 16 + (r & 15) : ct * 64 + r; };
    const char *w[2], *x[2];
    const uint8_t *ws[2], *xs[2];
    bool has_w[2], has_x[2];
    for (int i = 0; i < 2; ++i) {
        const int r = wn * 32 + i * 16 + fr, o = out_of(r);
        has_w[i] = o < a.d_out;
        const int64_t row = has_w[i] ? (GATED && i ? a.d_out + (int64_t)o : o) : 0;
        w[i] = a.W + rt.expert * a.expert_stride + row * a.ldw + block * 16;
        ws[i] = a.w_blocks + (rt.expert * (int64_t)a.d_out * (GATED ? 2 : 1) + row) * a.block_bytes + block * 4;
        const int n = wm * 32 + i * 16 + fr;
        has_x[i] = n < rt.n;
        int64_t from = has_x[i] ? rt.row0 + n : 0;
        if (a.rows && has_x[i]) from = min(max(a.rows[from], 0), a.x_rows - 1);
        x[i] = a.X + from * a.ldx + block * 16;
        xs[i] = a.x_blocks + from * a.block_bytes + block * 4;
    }
    pr_f32x4_t acc[2][2] = {};
    const int blocks = a.d_in / 16;
    auto some = [](bool has, const void *from) { return has ? *static_cast<const pr_i32x4_t *>(from) : pr_i32x4_t{0, 0, 0, 0}; };
    for (int b0 = 0; b0 < blocks; b0 += 16) {
        int sw[2], sx[2];
        for (int i = 0; i < 2; ++i) {
            sw[i] = has_w[i] ? *reinterpret_cast<const int *>(ws[i] + b0) : 0;
            sx[i] = has_x[i] ? *reinterpret_cast<const int *>(xs[i] + b0) : 0;
        }
        auto step = [&](auto T) {
            constexpr int t4 = decltype(T)::value;
            const bool is = b0 + t4 * 4 + block < blocks;
            pr_i32x4_t fw[2], fx[2];
            for (int i = 0; i < 2; ++i) {
                fw[i] = some(has_w[i] && is, w[i] + (int64_t)(b0 + t4 * 4) * 16);
                fx[i] = some(has_x[i] && is, x[i] + (int64_t)(b0 + t4 * 4) * 16);
            }
            for (int i = 0; i < 2; ++i)
                for (int j = 0; j < 2; ++j) acc[i][j] = mx4_mul<t4>(fw[i], fx[j], acc[i][j], sw[i], sx[j]);
        };
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
    }
    for (int j = 0; j < 2; ++j) {
        const int r = wm * 32 + j * 16 + fr;
        if (r >= rt.n) continue;
        for (int i = 0; i < (GATED ? 1 : 2); ++i) {
            const int o = out_of(wn * 32 + i * 16 + block * 4);
            float y[4];
            for (int n = 0; n < 4; ++n) y[n] = GATED ? silu(acc[0][j][n]) * acc[1][j][n] : acc[i][j][n];
            if (o < a.d_out) store_y4<YBF16>(a.Y, (int64_t)(rt.row0 + r) * a.ldy + o, y, a.d_out - o);
        }
    }
}

}  // namespace

hipError_t launch_mx4_product(const Product &p) {
    const ProductArgs a = args_of(p);
    const int outs = p.gated ? 32 : 64;
    const int64_t cols = ((int64_t)p.d_out + outs - 1) / outs, n = most_row_tiles(p, MP_TILE) * cols;
    if (n * MP_THREADS > 0xFFFFFFFFll) return hipErrorNotSupported;
    const dim3 g((uint32_t)n);
    if (p.gated) {
        if (p.y_bf16) k_mx4_product<true, true><<<g, MP_THREADS, 0, p.stream>>>(a, (int)cols);
        else k_mx4_product<true, false><<<g, MP_THREADS, 0, p.stream>>>(a, (int)cols);
    } else {
        if (p.y_bf16) k_mx4_product<false, true><<<g, MP_THREADS, 0, p.stream>>>(a, (int)cols);
        else k_mx4_product<false, false><<<g, MP_THREADS, 0, p.stream>>>(a, (int)cols);
    }
    return hipGetLastError();
}

}  // namespace qamw
