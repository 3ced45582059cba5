// Y = X W^T for 8-bit integers with scales or bf16, one matrix or one for each expert.
#include <cmath>

#include "qamw_product_tile.hpp"

namespace qamw {
namespace {

// ---- every shape, alignment and extent ------------------------------------------------------------------------------------
//
// A workgroup has 64 rows of W and 64 of X and steps over 128 bytes of both at a time, two steps in LDS and the next one on its way to
// registers.  Loads are 16 bytes wherever they begin, which the memory instructions allow, with 64-bit addresses; zeros stand
// where there is nothing: rows past the end, and columns past the last one, up to which a row's last piece is loaded by elements.
// Loads bound it, in latency and number.  4096 rows by 4096 x 4096: int8 207 us, bf16 388 us (60 and 105 us by whole lines and 256 rows);
// 16 rows 27 and 54 us (11 and 13 by the kernel for few rows, the call's own cost), 512 rows 35 and 69 us (29 and 51).
constexpr int PA_TILE = 64, PA_THREADS = 256, PA_K = 128, PA_PITCH = PA_K + 16;   // bytes: 16 more, or rows of a fragment share their banks

template <bool I8, bool GATED, bool YBF16>
__global__ __launch_bounds__(PA_THREADS) void k_product_any(ProductArgs a, int col_tiles) {
    using M = Mfma<I8>;
    using Piece = Unaligned<typename M::elem_t, 16 / M::ELEM>;
    __shared__ __align__(16) char lds[2][2][PA_TILE * PA_PITCH];
    const int t = (int)(blockIdx.x / (uint32_t)col_tiles), ct = (int)(blockIdx.x % (uint32_t)col_tiles);
    const RowTile rt = find_tile<PA_TILE>(a, t);
    if (rt.n <= 0) return;
    const int tid = threadIdx.x, lane = tid % WAVE, wave = tid / WAVE, wn = wave & 1, wm = wave >> 1;
    // row r of the tile's 64 rows of W; gated: 16 of the gate, then the same 16 of the up projection
    auto out_of = [&](int r) { return GATED ? ct * 32 + (r >> 5) * 16 + (r & 15) : ct * 64 + r; };
    const char *W = a.W + (int64_t)rt.expert * a.expert_stride;
    // what this thread loads: 32 bytes of one row of each operand
    const int lr = tid >> 2, lc = (tid & 3) * 32;
    const int out = out_of(lr);
    const bool has_w = out < a.d_out, has_x = lr < rt.n;
    const char *src_w = W + (has_w ? (int64_t)(GATED && ((lr >> 4) & 1) ? a.d_out + (int64_t)out : out) * a.ldw : 0);
    int64_t x_row = has_x ? rt.row0 + lr : 0;
    if (a.rows && has_x) x_row = min(max(a.rows[x_row], 0), a.x_rows - 1);
    const char *src_x = a.X + x_row * a.ldx;

    const int64_t bytes = (int64_t)a.d_in * M::ELEM;
    Piece w[2], x[2];
    auto load = [&](const char *src, bool has, int64_t at, Piece &to) {
        to = {};
        if (!has) return;
        if (at + 16 <= bytes) to = *reinterpret_cast<const Piece *>(src + at);
        else
            for (int i = 0; i < 16 / M::ELEM; ++i)
                if (at + i * M::ELEM < bytes) to.v[i] = *reinterpret_cast<const typename M::elem_t *>(src + at + i * M::ELEM);
    };
    auto request = [&](int64_t k0) {
        for (int i = 0; i < 2; ++i) {
            load(src_w, has_w, k0 + lc + i * 16, w[i]);
            load(src_x, has_x, k0 + lc + i * 16, x[i]);
        }
    };
    request(0);
    typename M::acc_t acc[2][2] = {};
    int half = 0;
    for (int64_t k0 = 0; k0 < bytes; k0 += PA_K, half ^= 1) {
        char(&to)[2][PA_TILE * PA_PITCH] = lds[half];
        for (int i = 0; i < 2; ++i) {
            *reinterpret_cast<pr_i32x4_t *>(&to[0][lr * PA_PITCH + lc + i * 16]) = __builtin_bit_cast(pr_i32x4_t, w[i]);
            *reinterpret_cast<pr_i32x4_t *>(&to[1][lr * PA_PITCH + lc + i * 16]) = __builtin_bit_cast(pr_i32x4_t, x[i]);
        }
        __syncthreads();           // of the step before, all have read the other half when they come here again
        request(k0 + PA_K);
        for (int h = 0; h < PA_K; h += 64) {
            pr_i32x4_t fw[2], fx[2];
            for (int i = 0; i < 2; ++i) {
                fw[i] = *reinterpret_cast<const pr_i32x4_t *>(&to[0][(wn * 32 + i * 16 + lane % 16) * PA_PITCH + h + lane / 16 * 16]);
                fx[i] = *reinterpret_cast<const pr_i32x4_t *>(&to[1][(wm * 32 + i * 16 + lane % 16) * PA_PITCH + h + lane / 16 * 16]);
            }
            for (int i = 0; i < 2; ++i)
                for (int j = 0; j < 2; ++j) acc[i][j] = M::mul(fw[i], fx[j], acc[i][j]);
        }
    }

    const float *ws = I8 ? a.w_scales + (int64_t)rt.expert * a.d_out * (GATED ? 2 : 1) : nullptr;
    for (int j = 0; j < 2; ++j) {
        const int r = wm * 32 + j * 16 + lane % 16;
        if (r >= rt.n) continue;
        const int64_t row = rt.row0 + r;
        const float xs = I8 ? a.x_scales[a.rows ? min(max(a.rows[row], 0), a.x_rows - 1) : row] : 1.0f;
        for (int i = 0; i < (GATED ? 1 : 2); ++i)
            for (int q = 0; q < 4; ++q) {
                const int o = out_of(wn * 32 + i * 16 + lane / 16 * 4 + q);
                if (o >= a.d_out) continue;
                float v = (float)acc[i][j][q];
                if (I8) v = v * xs * ws[o];
                if (GATED) {
                    float u = (float)acc[1][j][q];
                    if (I8) u = u * xs * ws[a.d_out + o];
                    v = silu(v) * u;
                }
                store_y<YBF16>(a.Y, row * a.ldy + o, v);
            }
    }
}

template <bool I8> hipError_t launch_any(const Product &p) {
    const ProductArgs a = args_of(p);
    const int outs = p.gated ? 32 : 64;
    const int64_t cols = ((int64_t)p.d_out + outs - 1) / outs, n = most_row_tiles(p, PA_TILE) * cols;
    if (n * PA_THREADS > 0xFFFFFFFFll) return hipErrorNotSupported;
    const dim3 g((uint32_t)n);
    if (p.gated) {
        if (p.y_bf16) k_product_any<I8, true, true><<<g, PA_THREADS, 0, p.stream>>>(a, (int)cols);
        else k_product_any<I8, true, false><<<g, PA_THREADS, 0, p.stream>>>(a, (int)cols);
    } else {
        if (p.y_bf16) k_product_any<I8, false, true><<<g, PA_THREADS, 0, p.stream>>>(a, (int)cols);
        else k_product_any<I8, false, false><<<g, PA_THREADS, 0, p.stream>>>(a, (int)cols);
    }
    return hipGetLastError();
}

}  // namespace

namespace {

// ---- which kernel ----------------------------------------------------------------------------------------------------------
//
// The choice is by an estimate of the time, in us, of weights that come from memory: a launch, and the root of the squares of what the
// busiest CU has to do and of what memory and the caches have to give: W, X once more for each of up to 8 XCDs that read it, in part, and for few
// rows W again for each tile of rows, in part.  The figures are fitted to measurements of 1 to 9000 rows, 1 to 128 experts, 48 to 27648
// outputs and 256 to 13824 columns in int8 and bf16 (a tenth off, in the mean): what a tile's begin and end and 128 bytes of columns cost, by rows of a
// tile; the bytes a us that a CU of the kernel for few rows takes in; how much more either is where rows are not whole 128-byte lines.
//   Both sides, int8 and us, few rows by 16 / 32 / 64 against wide ones by 64 / 128 / 256 in so many parts of the columns:
//     outputs x columns   rows   few                  wide, whole columns    wide, parts
//     1024 x 1024          64    3.5 / 4.0 / 5.1      10.9 / 12.8 / 18.1     (2) 10.9
//                          300   7.0 / 7.8 / 6.9      11.3 / 13.6 / 19.5     (2) 12.0
//     4096 x 4096            8   6.4 / 6.6 / 8.5      28.3 / 30.4 / 41.4     (4) 14.3 / 15.6 / 19.5
//                          100   17.2 / 13.9 / 13.9   28.5 / 33.4 / 42.7     (4) 17.8 / 19.7 / 23.3
//                          300   31.4 / 27.9 / 26.1   28.2 / 31.9 / 45.0     (2) 23.8 / 25.7 / 32.2
//                         1000                        30.2 / 34.2 / 48.4     (2) 46.8 / 35.4 / 41.3
//                         4000                        106 / 71.9 / 62.0
//     5120 x 13824          16   21.3 / 22.8 / 29.6   80.2 / 83.7 / 114      (4) 29.1 / 30.6 / 38.4
//                           64   39.6 / 35.0 / 39.6   86.5 / 89.6 / 114      (4) 31.7 / 33.1 / 39.7; (8) 27.8 by 64
//                          300   118 / 112 / 95.6     81.3 / 88.0 / 127      (4) 57.6 / 40.0 / 50.4
//                         1000                        161 / 96.6 / 133       (2) 146 / 120 / 89.3; (3) 83.8 by 256
//     27648 x 12800         34   179 / 148 / 109      92.1 / 95.0 / 111      (2) 70.5 / 71.7 / 77.1
//     27648 x 12720, off the lines: 34   253 / 179 / 148    132 / 135 / 143      (2) 86.5 / 88.0 / 92.1
// Of 428 measured shapes the choice was within 15 % of the fastest in all but 15 (one matrix, or experts with as many rows each), a third off at
// worst (3 rows by 1339 x 448, 5.3 us by tiles of 16, 3.9 by 32).
struct Plan {
    bool few;
    int tile_rows, parts;
    double us;
};
struct Off {
    double work, memory;                                   // times as much for rows off the 128-byte lines
};
struct Cost {
    int rows;
    double tile, stage;                                    // us, and bytes a us / us for 128 bytes of columns
};
constexpr double LAUNCH = 3.3, MEMORY = 7.3e6, PARTS = 2.2, PARTS_RATE = 6.5e6, FEW_X = 0.45, FEW_W = 0.15, WIDE_X = 0.12;
constexpr Off FEW_OFF = {1.3, 1.45}, WIDE_OFF = {1.23, 1.23};
constexpr Cost FEW[3] = {{16, 0.4, 9.4e4}, {32, 0.4, 9.9e4}, {64, 0.4, 8.0e4}}, WIDE[3] = {{64, 2.9, 0.72}, {128, 3.8, 0.83}, {256, 5.9, 1.12}};
constexpr double FEW_GATED_64 = 0.75;                      // of the rate: the ring is two units then

// groups: how many have rows, at most; row tiles are expected to be half a tile short.
Plan plan(int64_t m, int64_t groups, bool grouped, int64_t d_out, int64_t d_in, bool gated, bool i8, bool may_part) {
    const int64_t outs = d_out * (gated ? 2 : 1), bytes = d_in * (i8 ? 1 : 2), units = (bytes + 127) / 128;
    const double each = (double)m / groups, w_bytes = (double)groups * outs * bytes, x_bytes = (double)m * bytes;
    auto time = [&](double work, double memory, const Off &off) {
        if (bytes % 128) {
            work *= off.work;
            memory *= off.memory;
        }
        memory /= MEMORY;
        return LAUNCH + std::sqrt(work * work + memory * memory);
    };
    auto row_tiles = [&](int rows) {                        // of a group
        if (!grouped) return (double)((m + rows - 1) / rows);
        const double t = each / rows + 0.5;
        return t < 1 ? 1 : t;
    };
    auto rounds = [](double blocks) { return blocks <= 256 ? 1.0 : blocks <= 1024 ? (double)(((int64_t)blocks + 255) / 256) : blocks / 256 + 0.5; };
    auto xcds = [](double readers) { return readers < 1 ? 1 : readers > 8 ? 8 : readers; };
    Plan best = {true, 64, 1, 1e30};
    auto offer = [&](bool few, int rows, int parts, double us) {
        if (us < best.us) best = {few, rows, parts, us};
    };
    for (const Cost &c : FEW) {
        const double mine = row_tiles(c.rows), cols = (double)((d_out + 15) / 16), tiles = groups * mine * cols;
        const int split = few_split((int64_t)tiles, (int)units, 4);
        const double slot = 2048.0 * ((gated ? 2 : 1) + c.rows / 16), rate = gated && c.rows == 64 ? c.stage * FEW_GATED_64 : c.stage;
        const double work = rounds(tiles * split / 4) * (c.tile + units * 4 / split * slot / rate);
        offer(true, c.rows, 1, time(work, w_bytes * (1 + FEW_W * (mine - 1)) + x_bytes * FEW_X * xcds(cols * split / 4), FEW_OFF));
    }
    const double cols = (double)((outs + 255) / 256);
    for (const Cost &c : WIDE)
        for (int parts : {1, 2, 3, 4, 6, 8}) {
            if (parts > 1 && (!may_part || units < parts * 4)) break;
            const double work = rounds(groups * row_tiles(c.rows) * cols * parts) * (c.tile + (double)units / parts * c.stage);
            double us = time(work, w_bytes + x_bytes * WIDE_X * xcds(cols), WIDE_OFF);
            if (parts > 1) us += PARTS + 8.0 * parts * m * outs / PARTS_RATE;
            offer(false, c.rows, parts, us);
        }
    return best;
}
Plan plan_of(int m, int n_experts, bool grouped, int d_out, int d_in, bool gated, bool i8, bool may_part) {
    if (const int rows = product_tile_rows()) return {false, rows, 1, 0.0};
    return plan(m, !grouped ? 1 : m < n_experts ? m : n_experts, grouped, d_out, d_in, gated, i8, may_part);
}

}  // namespace

void product_plan(int m, int n_experts, bool grouped, int d_out, int d_in, bool gated, bool i8, bool may_part, int (&out)[3]) {
    const Plan c = plan_of(m, n_experts, grouped, d_out, d_in, gated, i8, may_part);
    out[0] = c.few ? 0 : 1;
    out[1] = c.tile_rows;
    out[2] = c.parts;
}

// The sums of all parts, whatever qamw_set_kernel_path() says: a workspace of this size serves the call before and after.
size_t product_scratch_bytes(int m, int d_out, int d_in, bool gated) {
    if (m == 0) return 0;
    const int parts = plan(m, 1, false, d_out, d_in, gated, true, true).parts;
    return parts == 1 ? 0 : (size_t)parts * m * (size_t)parts_row(d_out, gated) * 4;
}

hipError_t launch_product(const Product &p) {
    if (p.m == 0) return hipSuccess;
    if (!product_wide_supported(p)) return p.i8 ? launch_any<true>(p) : launch_any<false>(p);
    const Plan c = plan_of(p.m, p.n_experts, p.offsets != nullptr, p.d_out, p.d_in, p.gated, p.i8, p.scratch != nullptr);
    return c.few ? launch_product_few(p, c.tile_rows) : launch_product_wide(p, c.tile_rows, c.parts);
}

}  // namespace qamw
