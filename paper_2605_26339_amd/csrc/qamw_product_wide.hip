// Y = X W^T on the matrix cores for many rows: 8-bit integers with scales or bf16, one matrix or one for each expert.
//
// A workgroup of eight waves has a tile of BN rows of W and BM of X and steps over 64 bytes of both at a time (a stage: 64
// columns of int8, 32 of bf16).  16 rows of a stage are a fragment, 1 KB in LDS, filled by one buffer load of a wave that goes
// to LDS directly and read by one 16-byte LDS read of a wave: the operand of a 16x16 matrix instruction.
//   In LDS the four 16-byte pieces of a row are exchanged by (row / 2) mod 4, or the lanes of a read would meet in half of
//   the banks; the loading lanes ask for their piece accordingly, from the same 64 bytes.
//   Four stages are in LDS: one is read, the next ones are on their way while two others' products run, which covers the latency of memory.
//   The waves form two groups of four, one wave of each group on every SIMD.  While one group reads its fragments the other
//   multiplies, then they change places; a barrier is all that they need to keep in step.
// What is not there (rows past the end, columns past d_in, stages past the last) is loaded as zeros: such a lane asks for an
// address beyond its buffer's end.
#include "qamw_product_tile.hpp"

namespace qamw {
namespace {

constexpr int PW_WAVES = 8, PW_THREADS = PW_WAVES * WAVE, PW_STAGES = 4, PW_FRAG = 1024, PW_KB = 64;
constexpr uint32_t PW_NOWHERE = 0x80000000u;       // added to an offset: beyond the end of any buffer here

// Tiles: WN x WM waves, each of FN fragments of W and FM of X.
template <int WN_, int FN_, int WM_, int FM_> struct Shape {
    static constexpr int WN = WN_, FN = FN_, WM = WM_, FM = FM_, BN = WN * FN * 16, BM = WM * FM * 16;
    static constexpr int NW = WN * FN, NX = WM * FM;                          // fragments of a stage
    static constexpr int LW = NW / PW_WAVES, LX = (NX + PW_WAVES - 1) / PW_WAVES;   // loads of a wave: fragments wave, wave + 8, ...
    static constexpr int STAGE = (NW + (LX * PW_WAVES)) * PW_FRAG;            // where NX < 8, room for what some waves load for nothing
    static_assert(WN * WM == PW_WAVES && NW % PW_WAVES == 0, "");
};

// FN + FM fragments of one stage, complete when this returns.
template <int FN, int FM>
__device__ __forceinline__ void read_fragments(uint32_t at_w, uint32_t at_x, pr_i32x4_t (&w)[FN], pr_i32x4_t (&x)[FM]) {
    static_assert(FM == 4, "");
    if constexpr (FN == 8) {
        asm volatile(
            "ds_read_b128 %8, %13\n\tds_read_b128 %9, %13 offset:1024\n\tds_read_b128 %10, %13 offset:2048\n\tds_read_b128 %11, %13 offset:3072\n\t"
            "ds_read_b128 %0, %12\n\tds_read_b128 %1, %12 offset:1024\n\tds_read_b128 %2, %12 offset:2048\n\tds_read_b128 %3, %12 offset:3072\n\t"
            "ds_read_b128 %4, %12 offset:4096\n\tds_read_b128 %5, %12 offset:5120\n\tds_read_b128 %6, %12 offset:6144\n\tds_read_b128 %7, %12 offset:7168\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]), "=&v"(w[4]), "=&v"(w[5]), "=&v"(w[6]), "=&v"(w[7]), "=&v"(x[0]),
              "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
            : "v"(at_w), "v"(at_x)
            : "memory");
    } else if constexpr (FN == 4) {
        asm volatile(
            "ds_read_b128 %4, %9\n\tds_read_b128 %5, %9 offset:1024\n\tds_read_b128 %6, %9 offset:2048\n\tds_read_b128 %7, %9 offset:3072\n\t"
            "ds_read_b128 %0, %8\n\tds_read_b128 %1, %8 offset:1024\n\tds_read_b128 %2, %8 offset:2048\n\tds_read_b128 %3, %8 offset:3072\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]), "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
            : "v"(at_w), "v"(at_x)
            : "memory");
    } else {
        static_assert(FN == 2, "");
        asm volatile(
            "ds_read_b128 %2, %7\n\tds_read_b128 %3, %7 offset:1024\n\tds_read_b128 %4, %7 offset:2048\n\tds_read_b128 %5, %7 offset:3072\n\t"
            "ds_read_b128 %0, %6\n\tds_read_b128 %1, %6 offset:1024\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(w[0]), "=&v"(w[1]), "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
            : "v"(at_w), "v"(at_x)
            : "memory");
    }
}

template <int N> __device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void meet() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

template <bool I8, bool GATED, bool YBF16, typename S>
__global__ __launch_bounds__(PW_THREADS, 2) void k_product_wide(ProductArgs a, int col_tiles, int group) {
    using M = Mfma<I8>;
    extern __shared__ __align__(16) char pw_lds[];
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);

    // Workgroups go to the 8 XCDs in turn: an XCD gets tiles that follow one another, and these are ordered such that `group` row
    // tiles share their W while it is in the XCD's cache.
    const int row_tiles = count_tiles<S::BM>(a);
    const uint32_t all = (uint32_t)row_tiles * (uint32_t)col_tiles, share = (all + 7) / 8;
    const uint32_t nth = blockIdx.x / 8;
    const uint32_t t = (blockIdx.x % 8) * share + nth;
    if (nth >= share || t >= all) return;
    const ExpertTiles et = find_expert<S::BM>(a, (int)(t / (uint32_t)col_tiles));
    if (et.tiles == 0) return;
    const uint32_t v = t - (uint32_t)et.first * (uint32_t)col_tiles, per = (uint32_t)(group * col_tiles);
    const int g0 = (int)(v / per) * group, rows_in = min(group, et.tiles - g0), in = (int)(v % per);
    const int ct = in / rows_in, rt = g0 + in % rows_in;
    const int row0 = et.start + rt * S::BM, n = min(S::BM, et.end - row0);

    // fragment f, row r of the tile's W: the output it makes, and the row that it is (gated: 16 of the gate, then the same 16 of up)
    auto out_of = [&](int f, int r) { return GATED ? ct * (S::BN / 2) + (f >> 1) * 16 + r : ct * S::BN + f * 16 + r; };
    const int bytes = a.d_in * M::ELEM, stages = (bytes + PW_KB - 1) / PW_KB;
    const char *wp = a.W + (int64_t)et.expert * a.expert_stride;
    const char *xp = a.rows ? a.X : a.X + (int64_t)row0 * a.ldx;
    const int lr = lane >> 2, piece = ((lane ^ (lane >> 3)) & 3) * 16;
    const bool past = (stages - 1) * PW_KB + piece >= bytes;                  // nothing there in the last stage
    uint32_t off_w[S::LW], off_x[S::LX];
#pragma unroll
    for (int i = 0; i < S::LW; ++i) {
        const int f = wave + i * PW_WAVES, o = out_of(f, lr);
        const int64_t row = GATED && (f & 1) ? a.d_out + (int64_t)o : o;
        off_w[i] = o < a.d_out ? (uint32_t)(row * a.ldw) + piece : PW_NOWHERE;
    }
#pragma unroll
    for (int i = 0; i < S::LX; ++i) {
        const int r = (wave + i * PW_WAVES) * 16 + lr;
        const bool is = r < n;                                                // r < BM with it
        int row = is ? r : 0;
        if (a.rows && is) row = min(max(a.rows[row0 + r], 0), a.x_rows - 1);
        off_x[i] = is ? (uint32_t)((int64_t)row * a.ldx) + piece : PW_NOWHERE;
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)pw_lds;
    auto request = [&](int s) {
        const int records = s < stages ? 0x7FFFFFFF : 0;
        const auto wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(wp), 0, records, 0x00020000);
        const auto xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(xp), 0, records, 0x00020000);
        const uint32_t to = lds0 + (uint32_t)(s % PW_STAGES) * S::STAGE + wave * PW_FRAG, gone = s == stages - 1 && past ? PW_NOWHERE : 0;
#pragma unroll
        for (int i = 0; i < S::LW; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (__attribute__((address_space(3))) void *)(uintptr_t)(to + i * PW_WAVES * PW_FRAG), 16,
                                                     (int)(off_w[i] | gone), s * PW_KB, 0, 0);
#pragma unroll
        for (int i = 0; i < S::LX; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (__attribute__((address_space(3))) void *)(uintptr_t)(to + (S::NW + i * PW_WAVES) * PW_FRAG), 16,
                                                     (int)(off_x[i] | gone), s * PW_KB, 0, 0);
    };

    const int wn = wave % S::WN, wm = wave / S::WN;
    const uint32_t mine = (uint32_t)((lane & 15) * 64 + (((lane >> 4) ^ ((lane >> 1) & 3)) * 16));
    const uint32_t read_w = lds0 + mine + wn * S::FN * PW_FRAG, read_x = lds0 + mine + (S::NW + wm * S::FM) * PW_FRAG;
    typename M::acc_t acc[S::FN][S::FM] = {};
    constexpr int L = S::LW + S::LX;

    request(0);
    request(1);
    request(2);
    wait_loads<2 * L>();
    meet();
    if (wave >= PW_WAVES / 2) meet();                                         // the second group is half a step behind
    for (int s = 0; s < stages; ++s) {
        pr_i32x4_t fw[S::FN], fx[S::FM];
        request(s + 3);                                                       // over the stage that both groups have read
        const uint32_t at = (uint32_t)(s % PW_STAGES) * S::STAGE;
        read_fragments<S::FN, S::FM>(read_w + at, read_x + at, fw, fx);
        wait_loads<2 * L>();                                                  // stage s + 1 is there
        meet();
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < S::FM; ++j)
#pragma unroll
            for (int i = 0; i < S::FN; ++i) acc[i][j] = M::mul(fw[i], fx[j], acc[i][j]);
        __builtin_amdgcn_s_setprio(0);
        meet();
    }
    if (wave < PW_WAVES / 2) meet();

    const float *ws = I8 ? a.w_scales + (int64_t)et.expert * a.d_out * (GATED ? 2 : 1) : nullptr;
    const int q0 = (lane >> 4) * 4;
    float xs[S::FM];
#pragma unroll
    for (int j = 0; j < S::FM; ++j) {
        const int r = (wm * S::FM + j) * 16 + (lane & 15);
        xs[j] = 1.0f;
        if (I8 && r < n) xs[j] = a.x_scales[a.rows ? min(max(a.rows[row0 + r], 0), a.x_rows - 1) : row0 + r];
    }
#pragma unroll
    for (int i = 0; i < S::FN; i += GATED ? 2 : 1) {
        const int o = out_of(wn * S::FN + i, q0), there = a.d_out - o;        // of the four outputs from o
        if (there <= 0) continue;
        float sg[4] = {1, 1, 1, 1}, su[4] = {1, 1, 1, 1};
        if (I8)
            for (int q = 0; q < 4; ++q)
                if (q < there) {
                    sg[q] = ws[o + q];
                    if (GATED) su[q] = ws[a.d_out + o + q];
                }
#pragma unroll
        for (int j = 0; j < S::FM; ++j) {
            const int r = (wm * S::FM + j) * 16 + (lane & 15);
            if (r >= n) continue;
            float y[4];
            for (int q = 0; q < 4; ++q) {
                y[q] = (float)acc[i][j][q];
                if (I8) y[q] = y[q] * xs[j] * sg[q];
                if (GATED) {
                    float u = (float)acc[i + 1][j][q];
                    if (I8) u = u * xs[j] * su[q];
                    y[q] = silu(y[q]) * u;
                }
            }
            store_y4<YBF16>(a.Y, (int64_t)(row0 + r) * a.ldy + o, y, there);
        }
    }
}

template <bool I8, bool GATED, bool YBF16, typename S> hipError_t launch(const Product &p) {
    const int outs = GATED ? S::BN / 2 : S::BN;
    const int64_t cols = ((int64_t)p.d_out + outs - 1) / outs, tiles = most_row_tiles(p, S::BM) * cols, blocks = (tiles + 7) / 8 * 8;
    if (blocks * PW_THREADS > 0xFFFFFFFFll) return hipErrorNotSupported;
    const auto kernel = &k_product_wide<I8, GATED, YBF16, S>;
    constexpr int lds = PW_STAGES * S::STAGE;
    static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (once != hipSuccess) return once;
    kernel<<<dim3((uint32_t)blocks), PW_THREADS, lds, p.stream>>>(args_of(p), (int)cols, 8);
    return hipGetLastError();
}

template <bool I8, typename S> hipError_t launch_shape(const Product &p) {
    if (p.gated) return p.y_bf16 ? launch<I8, true, true, S>(p) : launch<I8, true, false, S>(p);
    return p.y_bf16 ? launch<I8, false, true, S>(p) : launch<I8, false, false, S>(p);
}

using Shape256 = Shape<2, 8, 4, 4>;
using Shape128 = Shape<4, 4, 2, 4>;
using Shape64 = Shape<8, 2, 1, 4>;

template <bool I8> hipError_t launch_type(const Product &p) {
    const int64_t rows = p.m / (p.offsets ? p.n_experts : 1);                  // of a group, on average
    if (rows > 128) return launch_shape<I8, Shape256>(p);
    if (rows > 64) return launch_shape<I8, Shape128>(p);
    return launch_shape<I8, Shape64>(p);
}

}  // namespace

// Whole 16 bytes everywhere, and offsets from a tile's or an expert's first row that 31 bits hold (with a stage's 64 bytes).
bool product_wide_supported(const Product &p) {
    const int64_t e = p.i8 ? 1 : 2, most = 0x7FFFFFFF - 2 * PW_KB;
    auto whole = [](int64_t v) { return v % 16 == 0; };
    if (!whole(p.d_in * e) || !whole(p.ldx * e) || !whole(p.ldw * e) || !whole(p.expert_stride * e) || (reinterpret_cast<uintptr_t>(p.X) & 15) ||
        (reinterpret_cast<uintptr_t>(p.W) & 15))
        return false;
    const int64_t outs = (int64_t)p.d_out * (p.gated ? 2 : 1), x_rows = p.rows ? p.x_rows : p.m < 256 ? p.m : 256;
    return p.ldw * e <= most / outs && p.ldx * e <= most / x_rows;
}

hipError_t launch_product_wide(const Product &p) { return p.i8 ? launch_type<true>(p) : launch_type<false>(p); }

}  // namespace qamw
