// Y = X W^T on the matrix cores for many rows: 8-bit integers with scales or bf16, one matrix or one for each expert.
//
// A workgroup of eight waves has a tile of BN rows of W and BM of X and steps over 128 bytes of both at a time (a stage: 128
// columns of int8, 64 of bf16).  16 rows of a stage are a fragment, 2 KB in LDS, filled by two buffer loads of a wave that go
// to LDS directly, eight whole lines each, and read by two 16-byte LDS reads of a wave: the operands of 16x16 matrix instructions.
//   In LDS the eight 16-byte pieces of a row are exchanged by row mod 8, or the lanes of a read would meet in some of the
//   banks; the loading lanes ask for their piece accordingly, from the same 128 bytes.
//   A stage has two steps: X and half of each wave's W, then the other half of W with X in registers.  Two stages are in
//   LDS; what a step has read is free for the stage after the next one, whose loads have a whole stage's time to come.
//   The waves form two groups of four, one wave of each group on every SIMD.  While one group reads its fragments the other
//   multiplies, then they change places; a barrier is all that they need to keep in step.
// What is not there (rows past the end, columns past d_in, stages past the last) is loaded as zeros: such a lane asks for an
// address beyond its buffer's end.
// What bounds it: power, and what a stage does beside its products.  8192 x 8192 x 8192 in int8 runs at 2200 TOPS with random operands and at
// 3185 with zeros, at 1.3 and 1.9 GHz and in the same clocks a stage, bf16 at 1270 and 1747 TFLOP/s; matrix instructions alone reach 3527 and 1981
// with random operands.  Of a wave's 1500 clocks a stage 585 are products, 428 reads, 490 waits and barriers; the matrix cores are busy for three
// fifths.  The library's product of the same card reaches 2140 to 2175 TOPS and 1435 to 1550 TFLOP/s: for bf16 power is not all.  256 rows of W and
// 256 of X, the most that accumulators have room for, read least for each product.  Smaller row tiles where there are too few to fill
// the CUs: 1000 rows by 4096 x 4096 in 30.2 us by 64, 34.2 by 128, 48.4 by 256; 4000 rows 106, 71.9, 62.0.
// Tried and slower: four waves of 128 x 128, one barrier a stage for all eight waves, five stages of 64 bytes, loads issued among the matrix
// instructions, and the barrier before the last of a step's products (3 to 12 %).
#include "qamw_product_tile.hpp"

namespace qamw {
namespace {

constexpr int PW_WAVES = 8, PW_THREADS = PW_WAVES * WAVE, PW_FRAG = 2048, PW_KB = 128, PW_CUS = 256, PW_TURN = 2048, PW_SLOTS = 3;
constexpr uint32_t PW_NOWHERE = 0x80000000u;       // added to an offset: beyond the end of any buffer here

// Tiles: WN x WM waves, each of FN fragments of W and FM of X.  A stage in LDS: the first halves of the waves' fragments of W, the second
// halves, X.
template <int WN_, int FN_, int WM_, int FM_> struct Shape {
    static constexpr int WN = WN_, FN = FN_, WM = WM_, FM = FM_, BN = WN * FN * 16, BM = WM * FM * 16;
    static constexpr int HN = FN / 2, NW = WN * FN, NX = WM * FM;             // fragments of a step, and of a stage
    static constexpr int LW = NW / PW_WAVES, LX = NX * 2 / PW_WAVES;          // loads of a wave, 8 rows each: of half of W, of X
    static constexpr int SECOND = NW / 2 * PW_FRAG, X = NW * PW_FRAG, STAGE = (NW + NX) * PW_FRAG;
    static_assert(WN * WM == PW_WAVES && NW % PW_WAVES == 0 && NX * 2 % PW_WAVES == 0 && BN == 256 && BM <= 256, "");
};

typedef uint32_t pw_u32x4_t __attribute__((ext_vector_type(4)));

// The two steps of a stage: what they read, and the loads that they issue while that comes.  Complete when they return, but for the loads.
// Both 64-byte halves of a row: their pieces are 64 bytes apart, exchanged by bit 6.  The loads go to LDS from `to` on, 8 KB apart.
template <int HN, int FM, int LW>
__device__ __forceinline__ void read_first(uint32_t at_w, uint32_t at_x, pr_i32x4_t (&w)[2][HN], pr_i32x4_t (&x)[2][FM], const uint32_t (&off_w)[LW],
                                           pw_u32x4_t wr, uint32_t so, uint32_t to) {
    static_assert(FM == 4 && LW == 2 && (HN == 4 || HN == 2 || HN == 1), "");
    if constexpr (HN == 4) {
        asm volatile(
            "ds_read_b128 %0, %18\n\tds_read_b128 %1, %18 offset:2048\n\tds_read_b128 %2, %18 offset:4096\n\t"
            "ds_read_b128 %3, %18 offset:6144\n\tds_read_b128 %8, %16\n\tds_read_b128 %9, %16 offset:2048\n\t"
            "ds_read_b128 %10, %16 offset:4096\n\tds_read_b128 %11, %16 offset:6144\n\tds_read_b128 %4, %19\n\t"
            "ds_read_b128 %5, %19 offset:2048\n\tds_read_b128 %6, %19 offset:4096\n\t"
            "ds_read_b128 %7, %19 offset:6144\n\tds_read_b128 %12, %17\n\tds_read_b128 %13, %17 offset:2048\n\t"
            "ds_read_b128 %14, %17 offset:4096\n\tds_read_b128 %15, %17 offset:6144\n\ts_mov_b32 m0, %24\n\t"
            "s_nop 0\n\tbuffer_load_dwordx4 %20, %22, %23 offen lds\n\ts_add_u32 m0, m0, 0x2000\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %21, %22, %23 offen lds\n\ts_waitcnt lgkmcnt(0)"
            : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[0][3]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[1][2]),
              "=&v"(x[1][3]), "=&v"(w[0][0]), "=&v"(w[0][1]), "=&v"(w[0][2]), "=&v"(w[0][3]), "=&v"(w[1][0]), "=&v"(w[1][1]),
              "=&v"(w[1][2]), "=&v"(w[1][3])
            : "v"(at_w), "v"(at_w ^ 64u), "v"(at_x), "v"(at_x ^ 64u), "v"(off_w[0]), "v"(off_w[1]), "s"(wr), "s"(so), "s"(to)
            : "memory", "scc");
    } else if constexpr (HN == 2) {
        asm volatile(
            "ds_read_b128 %0, %14\n\tds_read_b128 %1, %14 offset:2048\n\tds_read_b128 %2, %14 offset:4096\n\t"
            "ds_read_b128 %3, %14 offset:6144\n\tds_read_b128 %8, %12\n\tds_read_b128 %9, %12 offset:2048\n\t"
            "ds_read_b128 %4, %15\n\tds_read_b128 %5, %15 offset:2048\n\tds_read_b128 %6, %15 offset:4096\n\t"
            "ds_read_b128 %7, %15 offset:6144\n\tds_read_b128 %10, %13\n\tds_read_b128 %11, %13 offset:2048\n\t"
            "s_mov_b32 m0, %20\n\ts_nop 0\n\tbuffer_load_dwordx4 %16, %18, %19 offen lds\n\t"
            "s_add_u32 m0, m0, 0x2000\n\ts_nop 0\n\tbuffer_load_dwordx4 %17, %18, %19 offen lds\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[0][3]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[1][2]),
              "=&v"(x[1][3]), "=&v"(w[0][0]), "=&v"(w[0][1]), "=&v"(w[1][0]), "=&v"(w[1][1])
            : "v"(at_w), "v"(at_w ^ 64u), "v"(at_x), "v"(at_x ^ 64u), "v"(off_w[0]), "v"(off_w[1]), "s"(wr), "s"(so), "s"(to)
            : "memory", "scc");
    } else {
        asm volatile(
            "ds_read_b128 %0, %12\n\tds_read_b128 %1, %12 offset:2048\n\tds_read_b128 %2, %12 offset:4096\n\t"
            "ds_read_b128 %3, %12 offset:6144\n\tds_read_b128 %8, %10\n\tds_read_b128 %4, %13\n\t"
            "ds_read_b128 %5, %13 offset:2048\n\tds_read_b128 %6, %13 offset:4096\n\t"
            "ds_read_b128 %7, %13 offset:6144\n\tds_read_b128 %9, %11\n\ts_mov_b32 m0, %18\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %14, %16, %17 offen lds\n\ts_add_u32 m0, m0, 0x2000\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %15, %16, %17 offen lds\n\ts_waitcnt lgkmcnt(0)"
            : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[0][3]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[1][2]),
              "=&v"(x[1][3]), "=&v"(w[0][0]), "=&v"(w[1][0])
            : "v"(at_w), "v"(at_w ^ 64u), "v"(at_x), "v"(at_x ^ 64u), "v"(off_w[0]), "v"(off_w[1]), "s"(wr), "s"(so), "s"(to)
            : "memory", "scc");
    }
}
template <int HN, int LW, int LX>
__device__ __forceinline__ void read_second(uint32_t at_w, pr_i32x4_t (&w)[2][HN], const uint32_t (&off_w)[LW], const uint32_t (&off_x)[LX], pw_u32x4_t wr,
                                            pw_u32x4_t xr, uint32_t so, uint32_t to_w, uint32_t to_x) {
    static_assert(LW == 2 && LX == HN && (HN == 4 || HN == 2 || HN == 1), "");
    if constexpr (LX == 4) {
        asm volatile(
            "ds_read_b128 %0, %8\n\tds_read_b128 %1, %8 offset:2048\n\tds_read_b128 %2, %8 offset:4096\n\t"
            "ds_read_b128 %3, %8 offset:6144\n\tds_read_b128 %4, %9\n\tds_read_b128 %5, %9 offset:2048\n\t"
            "ds_read_b128 %6, %9 offset:4096\n\tds_read_b128 %7, %9 offset:6144\n\ts_mov_b32 m0, %20\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %12, %17, %18 offen lds\n\ts_add_u32 m0, m0, 0x2000\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %13, %17, %18 offen lds\n\ts_add_u32 m0, m0, 0x2000\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %14, %17, %18 offen lds\n\ts_add_u32 m0, m0, 0x2000\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %15, %17, %18 offen lds\n\ts_mov_b32 m0, %19\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %10, %16, %18 offen lds\n\ts_add_u32 m0, m0, 0x2000\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %11, %16, %18 offen lds\n\ts_waitcnt lgkmcnt(0)"
            : "=&v"(w[0][0]), "=&v"(w[0][1]), "=&v"(w[0][2]), "=&v"(w[0][3]), "=&v"(w[1][0]), "=&v"(w[1][1]), "=&v"(w[1][2]),
              "=&v"(w[1][3])
            : "v"(at_w), "v"(at_w ^ 64u), "v"(off_w[0]), "v"(off_w[1]), "v"(off_x[0]), "v"(off_x[1]), "v"(off_x[2]), "v"(off_x[3]),
              "s"(wr), "s"(xr), "s"(so), "s"(to_w), "s"(to_x)
            : "memory", "scc");
    } else if constexpr (LX == 2) {
        asm volatile(
            "ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:2048\n\tds_read_b128 %2, %5\n\t"
            "ds_read_b128 %3, %5 offset:2048\n\ts_mov_b32 m0, %14\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %8, %11, %12 offen lds\n\ts_add_u32 m0, m0, 0x2000\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %9, %11, %12 offen lds\n\ts_mov_b32 m0, %13\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %6, %10, %12 offen lds\n\ts_add_u32 m0, m0, 0x2000\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %7, %10, %12 offen lds\n\ts_waitcnt lgkmcnt(0)"
            : "=&v"(w[0][0]), "=&v"(w[0][1]), "=&v"(w[1][0]), "=&v"(w[1][1])
            : "v"(at_w), "v"(at_w ^ 64u), "v"(off_w[0]), "v"(off_w[1]), "v"(off_x[0]), "v"(off_x[1]), "s"(wr), "s"(xr), "s"(so), "s"(to_w),
              "s"(to_x)
            : "memory", "scc");
    } else {
        asm volatile(
            "ds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_mov_b32 m0, %11\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %6, %8, %9 offen lds\n\ts_mov_b32 m0, %10\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %4, %7, %9 offen lds\n\ts_add_u32 m0, m0, 0x2000\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %5, %7, %9 offen lds\n\ts_waitcnt lgkmcnt(0)"
            : "=&v"(w[0][0]), "=&v"(w[1][0])
            : "v"(at_w), "v"(at_w ^ 64u), "v"(off_w[0]), "v"(off_w[1]), "v"(off_x[0]), "s"(wr), "s"(xr), "s"(so), "s"(to_w), "s"(to_x)
            : "memory", "scc");
    }
}
// A load alone, of 16 bytes a lane or 4.
__device__ __forceinline__ void request(uint32_t off, pw_u32x4_t from, uint32_t so, uint32_t to) {
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(off), "s"(from), "s"(so), "s"(to) : "memory");
}
__device__ __forceinline__ void request_dword(uint32_t off, pw_u32x4_t from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(off), "s"(from), "s"(to) : "memory");
}

template <int N> __device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void meet() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ pw_u32x4_t resource(const void *p, uint32_t records = 0x7FFFFFFF) {
    return {(uint32_t)(uintptr_t)p, (uint32_t)((uintptr_t)p >> 32) & 0xFFFFu, records, 0x00020000u};
}

template <bool BF16> struct Store {
    using type = float;
};
template <> struct Store<true> {
    using type = uint16_t;
};

template <int V> struct Half {
    static constexpr int value = V;
};
using First = Half<0>;
using Second = Half<1>;

// A tile: where its rows are, and what this lane asks for of them.
template <typename S> struct Tile {
    int expert, row0, n, ct;                         // rows row0 .. row0 + n, the ct-th outputs; n = 0: no tile
    int part, full;                                  // the part of the columns, its stages
    const char *w, *x;
    uint32_t off_w[2][S::LW], off_x[S::LX], off_scale;
};

// OUT: what is stored: 0 fp32, 1 bf16, 2 the sums of a part of the columns as they are (int32 or fp32), one array of `part_stride`
// elements a part.
template <bool I8, bool GATED, int OUT, typename S>
__global__ __launch_bounds__(PW_THREADS, 2) void k_product_wide(ProductArgs a, int most_tiles, int col_tiles, int group, int whole, int parts, int64_t part_stride) {
    constexpr bool YBF16 = OUT == 1, SCALED = I8 && OUT != 2;
    using M = Mfma<I8>;
    extern __shared__ __align__(16) char pw_lds[];
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)pw_lds;
    const uint32_t turn = lds0 + 2 * S::STAGE + wave * PW_TURN, scales0 = lds0 + 2 * S::STAGE + PW_WAVES * PW_TURN;

    // Workgroups go to the 8 XCDs in turn: an XCD gets tiles that follow one another, and these are ordered such that `group` row
    // tiles share their W while it is in the XCD's cache.  8 of them: gated int8, 8192 rows by 2 x 11008 x 4096, by groups of 1, 2, 4, 8, 16, 32:
    // 651, 636, 622, 618, 643, 654 us; 8002 rows of 8 such experts 807, 735, 703, 695, 681, 689.
    //   Offsets that do not ascend can make more row tiles than rows have room for: no more than the host has counted on are done, or the number of all
    // tiles could pass 32 bits and a workgroup's turn with it.
    const uint32_t one = (uint32_t)min(count_tiles<S::BM>(a), most_tiles) * (uint32_t)col_tiles, all = one * parts, share = (all + 7) / 8;
    const uint32_t begin = blockIdx.x % 8 * share, end = min(begin + share, all), step = gridDim.x / 8;
    // fragment f, row r of a tile's W: the output it makes (gated: 16 of the gate, then the same 16 of up)
    auto out_of = [&](int ct, int f, int r) { return GATED ? ct * (S::BN / 2) + (f >> 1) * 16 + r : ct * S::BN + f * 16 + r; };
    auto w_row = [&](int ct, int f, int r) { return (int64_t)(GATED && (f & 1) ? a.d_out : 0) + out_of(ct, f, r); };
    const int bytes = a.d_in * M::ELEM, every = (bytes + PW_KB - 1) / PW_KB;
    const int lr = lane >> 3, piece = ((lane & 7) ^ lr) * 16;
    const bool past = (every - 1) * PW_KB + piece >= bytes;                   // nothing there in the last stage of all

    ExpertTiles et = {0, 0, 0, 0, 0};
    auto tile_at = [&](uint32_t t) {
        Tile<S> z;
        z.n = 0;
        z.w = z.x = nullptr;
        z.expert = z.row0 = z.ct = z.part = z.full = 0;
        z.off_scale = PW_NOWHERE;
        for (int i = 0; i < S::LW; ++i) z.off_w[0][i] = z.off_w[1][i] = PW_NOWHERE;
        for (int i = 0; i < S::LX; ++i) z.off_x[i] = PW_NOWHERE;
        if (t >= end) return z;
        z.part = (int)(t / one);
        t -= z.part * one;
        const int row_tile = (int)(t / (uint32_t)col_tiles);
        if (row_tile < et.first || row_tile - et.first >= et.tiles) et = find_expert<S::BM>(a, row_tile);
        if (et.tiles == 0) return z;
        const uint32_t v = t - (uint32_t)et.first * (uint32_t)col_tiles, per = (uint32_t)(group * col_tiles);
        const int g0 = (int)(v / per) * group, rows_in = min(group, et.tiles - g0), in = (int)(v % per);
        z.expert = et.expert;
        z.ct = in / rows_in;
        z.row0 = et.start + (g0 + in % rows_in) * S::BM;
        z.n = min(S::BM, et.end - z.row0);
        const int s0 = (int)((int64_t)every * z.part / parts);
        z.full = (int)((int64_t)every * (z.part + 1) / parts) - s0;
        z.w = a.W + (int64_t)et.expert * a.expert_stride + s0 * PW_KB;
        z.x = (a.rows ? a.X : a.X + (int64_t)z.row0 * a.ldx) + s0 * PW_KB;
#pragma unroll
        for (int i = 0; i < 2 * S::LW; ++i) {
            const int unit = wave + i % S::LW * PW_WAVES, in_half = unit / 2;  // 8 rows of a fragment of the first or the second halves
            const int f = in_half / S::HN * S::FN + in_half % S::HN + i / S::LW * S::HN, r = unit % 2 * 8 + lr;
            z.off_w[i / S::LW][i % S::LW] = out_of(z.ct, f, r) < a.d_out ? (uint32_t)(w_row(z.ct, f, r) * a.ldw) + piece : PW_NOWHERE;
        }
#pragma unroll
        for (int i = 0; i < S::LX; ++i) {
            const int r = (wave + i * PW_WAVES) * 8 + lr;
            const bool is = r < z.n;                                          // r < BM with it
            int row = is ? r : 0;
            if (a.rows && is) row = min(max(a.rows[z.row0 + r], 0), a.x_rows - 1);
            z.off_x[i] = is ? (uint32_t)((int64_t)row * a.ldx) + piece : PW_NOWHERE;
        }
        if (SCALED) {                                                         // one scale a thread: 256 of rows, 256 of outputs
            const int r = threadIdx.x % 256;
            if (threadIdx.x < 256) {
                if (r < z.n) z.off_scale = 4 * (uint32_t)(a.rows ? min(max(a.rows[z.row0 + r], 0), a.x_rows - 1) : r);
            } else if (out_of(z.ct, r >> 4, r & 15) < a.d_out) {
                z.off_scale = 4 * (uint32_t)w_row(z.ct, r >> 4, r & 15);
            }
        }
        return z;
    };
    // Three slots: a tile of one or two stages asks for the next one's scales before its first barrier, when the second group may still have the
    // scales of the tile before it to read; in the third are its own.
    auto request_scales = [&](const Tile<S> &z, uint32_t slot) {
        if (!SCALED) return;
        const float *from = wave < PW_WAVES / 2 ? a.x_scales + (a.rows ? 0 : z.row0) : a.w_scales + (int64_t)z.expert * a.d_out * (GATED ? 2 : 1);
        request_dword(z.off_scale, resource(from), scales0 + slot + wave * 256);
    };

    const int wn = wave % S::WN, wm = wave / S::WN;
    const uint32_t mine = (uint32_t)((lane & 15) * PW_KB + (((lane >> 4) ^ (lane & 7)) * 16));
    const uint32_t read_w = lds0 + mine + wn * S::HN * PW_FRAG, read_x = lds0 + mine + S::X + wm * S::FM * PW_FRAG;
    constexpr int L = 2 * S::LW + S::LX;
    constexpr int YB = YBF16 ? 2 : 4, OUTS = S::FN * 16 / (GATED ? 2 : 1), PASS = 128 / YB < OUTS ? 128 / YB : OUTS;   // outputs of a wave's row, of a pass
    constexpr int PIECES = PASS * YB / 16, AT_ONCE = WAVE / PIECES, TIMES = AT_ONCE < 16 ? 16 / AT_ONCE : 1;   // 16-byte pieces of a pass' row, rows stored at once
    constexpr int STORES = S::FM * (OUTS / PASS) * TIMES;

    uint32_t t = begin + blockIdx.x / 8;
    Tile<S> now = tile_at(t);
    if (now.n == 0) return;
    uint32_t at = 0, slot = 0;                                                // the stage that is read, the scales that are
    // which lanes have nothing in stage s of a tile
    auto nothing = [&](const Tile<S> &z, int s) { return s >= z.full || (s == z.full - 1 && z.part == parts - 1 && past) ? PW_NOWHERE : 0; };
    auto offsets = [&](auto &to, const auto &from, uint32_t gone) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(to) / sizeof(to[0])); ++i) to[i] = from[i] | gone;
    };
    request_scales(now, 0);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const uint32_t gone = nothing(now, s), to = lds0 + s * S::STAGE + wave * 1024;
#pragma unroll
        for (int i = 0; i < S::LX; ++i) request(now.off_x[i] | gone, resource(now.x), s * PW_KB, to + S::X + i * 8192);
#pragma unroll
        for (int i = 0; i < S::LW; ++i) request(now.off_w[0][i] | gone, resource(now.w), s * PW_KB, to + i * 8192);
        if (s == 0)
#pragma unroll
            for (int i = 0; i < S::LW; ++i) request(now.off_w[1][i] | gone, resource(now.w), 0, to + S::SECOND + i * 8192);
    }
    wait_loads<L>();
    meet();
    if (wave >= PW_WAVES / 2) meet();                                         // the second group is half a step behind

    typename M::acc_t acc[S::FN][S::FM];
    pr_i32x4_t fw[2][S::HN], fx[2][S::FM];                                    // [halves of a row]
    auto multiply = [&](auto second, bool busy) {
        constexpr int I0 = decltype(second)::value * S::HN;
        __builtin_amdgcn_s_setprio(1);
        if (busy)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < S::FM; ++j)
#pragma unroll
                    for (int n = 0; n < S::HN; ++n) {
                        const int i = j & 1 ? S::HN - 1 - n : n;              // to and fro: one operand changes at a time, 1 % less time for random ones
                        acc[I0 + i][j] = M::mul(fw[h][i], fx[h][j], acc[I0 + i][j]);
                    }
        __builtin_amdgcn_s_setprio(0);
    };
    // A stage.  First step: X and half of W; the second half of W of stage s1 of tile z1, the next one, is asked for.  Second step: the
    // second half of W; X and the first half of W of stage s2 of tile z2, the one after, are asked for.  Either goes over what
    // both groups have read a step before, and is waited for a stage later.  `stored`: the stores of the tile before may still be on
    // their way, between the loads that are waited for and the newer ones.
    auto stage = [&](const Tile<S> &z1, int s1, const Tile<S> &z2, int s2, bool stored, bool busy) {
        const uint32_t other = S::STAGE - at;
        auto wait = [&] {
            if (stored) wait_loads<L + STORES>();
            else wait_loads<L>();
        };
        uint32_t ow[S::LW], ox[S::LX];
        offsets(ow, z1.off_w[1], nothing(z1, s1));
        read_first<S::HN, S::FM, S::LW>(read_w + at, read_x + at, fw, fx, ow, resource(z1.w), (uint32_t)s1 * PW_KB, lds0 + other + S::SECOND + wave * 1024);
        wait();                                                               // the second half of this stage's W is there
        meet();
        multiply(First{}, busy);
        meet();
        const uint32_t gone = nothing(z2, s2);
        offsets(ow, z2.off_w[0], gone);
        offsets(ox, z2.off_x, gone);
        read_second<S::HN, S::LW, S::LX>(read_w + at + S::SECOND, fw, ow, ox, resource(z2.w), resource(z2.x), (uint32_t)s2 * PW_KB,
                                         lds0 + at + wave * 1024, lds0 + at + S::X + wave * 1024);
        wait();                                                               // the rest of the next stage is there
        meet();
        multiply(Second{}, busy);
        meet();
        at = other;
    };

    bool stored = false;
    for (;;) {
#pragma unroll
        for (int i = 0; i < S::FN; ++i)
#pragma unroll
            for (int j = 0; j < S::FM; ++j) acc[i][j] = typename M::acc_t{};
        const bool busy = wm * S::FM * 16 < now.n && out_of(now.ct, wn * S::FN, 0) < a.d_out;   // some of the wave's rows and outputs are there
        const int stages = max(now.full, 2);
        for (int s = 0; s < stages - 2; ++s) stage(now, s + 1, now, s + 2, stored && s == 0, busy);
        // the last two stages ask for the first ones of the next tile
        t += step;
        const Tile<S> next = tile_at(t);
        const uint32_t slot_next = slot == (PW_SLOTS - 1) * 2048 ? 0 : slot + 2048;
        request_scales(next, slot_next);
        stage(now, stages - 1, next, 0, stored && stages == 2, busy);
        stage(next, 0, next, 1, false, busy);

        const int q0 = (lane >> 4) * 4;
        // four outputs of fragment i (gated: and i + 1) in row j * 16 + lane % 16
        auto four = [&](int i, int j, float (&y)[4]) {
            const uint32_t sc = scales0 + slot;
            float xs = 1.0f;
            pr_f32x4_t sg = {1, 1, 1, 1}, su = {1, 1, 1, 1};
            if (SCALED) {
                xs = lds_read<float>(sc + ((wm * S::FM + j) * 16 + (lane & 15)) * 4);
                sg = lds_read<pr_f32x4_t>(sc + 1024 + ((wn * S::FN + i) * 16 + q0) * 4);
                if (GATED) su = lds_read<pr_f32x4_t>(sc + 1024 + ((wn * S::FN + i + 1) * 16 + q0) * 4);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                y[q] = (float)acc[i][j][q];
                if (SCALED) y[q] = y[q] * xs * sg[q];
                if (GATED) {
                    float u = (float)acc[i + 1][j][q];
                    if (SCALED) u = u * xs * su[q];
                    y[q] = silu(y[q]) * u;
                }
            }
        };
        // 16 rows of PASS outputs at a time are turned in the wave's own 2 KB of LDS, so that 16 bytes a lane and whole lines are stored.  The
        // eight 16-byte pieces of a row are exchanged by row mod 8.  Where Y's rows are whole pieces every wave makes the same number
        // of stores: what is not there goes beyond the buffer's end.
        constexpr int FRAGS = PASS / 16, STEP = GATED ? 2 : 1, EACH = 16 / YB;
        const int col0 = out_of(now.ct, wn * S::FN, 0);
        char *const yp = static_cast<char *>(a.Y) + (now.part * part_stride + (int64_t)now.row0 * a.ldy) * YB;
        const auto yr = __builtin_amdgcn_make_buffer_rsrc(yp, 0, 0x7FFFFFFF, 0x00020000);
#pragma unroll
        for (int j = 0; j < S::FM; ++j)
#pragma unroll
            for (int h = 0; h < OUTS / PASS; ++h) {
#pragma unroll
                for (int f = 0; f < FRAGS; ++f) {
                    float y[4];
                    if constexpr (OUT != 2) four((h * FRAGS + f) * STEP, j, y);
                    const int r = lane & 15, b = (f * 16 + q0) * YB;
                    const uint32_t to = turn + r * 128 + (((b >> 4) ^ (r & 7)) << 4) + (b & 15);
                    if constexpr (YBF16) lds_write<uint64_t>(to, (uint64_t)pack_bf16(y[2], y[3]) << 32 | pack_bf16(y[0], y[1]));
                    else if constexpr (OUT == 2) lds_write<pr_i32x4_t>(to, __builtin_bit_cast(pr_i32x4_t, acc[h * FRAGS + f][j]));
                    else lds_write<pr_f32x4_t>(to, pr_f32x4_t{y[0], y[1], y[2], y[3]});
                }
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int k = 0; k < TIMES; ++k) {
                    const int nth = k * AT_ONCE + lane / PIECES, r = nth & 15, p = lane % PIECES;
                    const pr_i32x4_t v = lds_read<pr_i32x4_t>(turn + r * 128 + ((p ^ (r & 7)) << 4));
                    const int row = (wm * S::FM + j) * 16 + r, col = col0 + h * PASS + p * EACH;
                    const bool is = nth < 16 && row < now.n && col < a.d_out;
                    if (whole) {
                        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(pw_u32x4_t, v), yr, (int)(is ? (uint32_t)(row * a.ldy + col) * YB : PW_NOWHERE), 0, 0);
                    } else if (is) {
                        using E = typename Store<YBF16>::type;
                        E *to = reinterpret_cast<E *>(yp) + row * a.ldy + col;
                        const auto e = __builtin_bit_cast(Unaligned<E, EACH>, v);
                        if (col + EACH <= a.d_out) {
                            *reinterpret_cast<Unaligned<E, EACH> *>(to) = e;
                        } else {
#pragma unroll
                            for (int i = 0; i < EACH - 1; ++i)
                                if (col + i < a.d_out) to[i] = e.v[i];
                        }
                    }
                }
                __builtin_amdgcn_wave_barrier();
            }
        if (next.n == 0) break;
        now = next;
        slot = slot_next;
        stored = whole != 0;
    }
    if (wave < PW_WAVES / 2) meet();
}

// The sums of the parts, in their order, and what is done with them: four outputs a thread.  Memory bounds it: 4 bytes a part and output
// are read, and all parts' are asked for together, which is why their number is known here: 509 rows of 5120 outputs in 3 parts 7.1 us, 5.2 TB/s
// with what is written (10.4 with a loop over any number).
//   Parts pay where the tiles of whole columns leave CUs without one: 300 rows by 5120 x 13824 take 40.0 us in 4 parts of tiles of 128
// rows, sums included, and 88 in one.  int8 only: its sums are whole numbers, and in any order the same.
constexpr int PS_THREADS = 256;
template <bool GATED, bool YBF16, int PARTS>
__global__ __launch_bounds__(PS_THREADS) void k_product_parts(ProductArgs a, const char *sums, int64_t part_stride, int64_t ld, int fours) {
    const uint32_t id = blockIdx.x * PS_THREADS + threadIdx.x;
    const int64_t row = id / (uint32_t)fours;
    const int o = (int)(id % (uint32_t)fours) * 4;
    if (row >= a.m) return;
    const char *at = sums + (row * ld + o) * 4, *up = at + (int64_t)a.d_out * 4;
    pr_i32x4_t g = {0, 0, 0, 0}, u = {0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        g += *reinterpret_cast<const pr_i32x4_t *>(at + p * part_stride * 4);
        if (GATED) u += __builtin_bit_cast(pr_i32x4_t, *reinterpret_cast<const Unaligned<int, 4> *>(up + p * part_stride * 4));
    }
    const float xs = a.x_scales[row];
    float y[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int i = min(o + q, a.d_out - 1);
        y[q] = (float)g[q] * xs * a.w_scales[i];
        if (GATED) y[q] = silu(y[q]) * ((float)u[q] * xs * a.w_scales[a.d_out + i]);
    }
    store_y4<YBF16>(a.Y, row * a.ldy + o, y, a.d_out - o);
}

template <bool I8, bool GATED, int OUT, typename S> hipError_t launch(const Product &p, int parts, int64_t part_stride) {
    const int outs = GATED ? S::BN / 2 : S::BN;
    const int64_t cols = ((int64_t)p.d_out + outs - 1) / outs, rows = most_row_tiles(p, S::BM), tiles = rows * cols * parts;
    if (tiles > 0x7FFFFFFF / 2) return hipErrorNotSupported;
    const int64_t blocks = tiles < PW_CUS ? (tiles + 7) / 8 * 8 : PW_CUS;       // one a CU, which goes from tile to tile
    const int64_t y_bytes = OUT == 1 ? 2 : 4;
    const bool whole = (reinterpret_cast<uintptr_t>(p.Y) & 15) == 0 && p.ldy * y_bytes % 16 == 0 && (p.d_out * y_bytes % 16 == 0 || OUT == 2) &&
                       p.ldy <= 0x7FFFFFFF / (S::BM * y_bytes);
    const auto kernel = &k_product_wide<I8, GATED, OUT, S>;
    constexpr int lds = 2 * S::STAGE + PW_WAVES * PW_TURN + PW_SLOTS * 2048;
    static MoreLds more;
    const hipError_t e = more.ask(reinterpret_cast<const void *>(kernel), lds);
    if (e != hipSuccess) return e;
    kernel<<<dim3((uint32_t)blocks), PW_THREADS, lds, p.stream>>>(args_of(p), (int)rows, (int)cols, 8, whole, parts, part_stride);
    return hipGetLastError();
}

template <bool I8, typename S> hipError_t launch_shape(const Product &p) {
    if (p.gated) return p.y_bf16 ? launch<I8, true, 1, S>(p, 1, 0) : launch<I8, true, 0, S>(p, 1, 0);
    return p.y_bf16 ? launch<I8, false, 1, S>(p, 1, 0) : launch<I8, false, 0, S>(p, 1, 0);
}

template <int PARTS> void launch_sums(const Product &p, int64_t stride, int64_t ld) {
    const int64_t fours = ((int64_t)p.d_out + 3) / 4;
    const dim3 g((uint32_t)((fours * p.m + PS_THREADS - 1) / PS_THREADS));
    const ProductArgs a = args_of(p);
    const char *sums = static_cast<const char *>(p.scratch);
    if (p.gated) {
        if (p.y_bf16) k_product_parts<true, true, PARTS><<<g, PS_THREADS, 0, p.stream>>>(a, sums, stride, ld, (int)fours);
        else k_product_parts<true, false, PARTS><<<g, PS_THREADS, 0, p.stream>>>(a, sums, stride, ld, (int)fours);
    } else {
        if (p.y_bf16) k_product_parts<false, true, PARTS><<<g, PS_THREADS, 0, p.stream>>>(a, sums, stride, ld, (int)fours);
        else k_product_parts<false, false, PARTS><<<g, PS_THREADS, 0, p.stream>>>(a, sums, stride, ld, (int)fours);
    }
}

// In `parts` parts of the columns (2, 3, 4, 6 or 8), whose sums lie in p.scratch.
template <typename S> hipError_t launch_parts(const Product &p, int parts) {
    Product q = p;
    q.d_out = p.d_out * (p.gated ? 2 : 1);
    q.gated = false;
    q.Y = p.scratch;
    q.ldy = parts_row(p.d_out, p.gated);
    const int64_t stride = q.ldy * p.m;
    if (((int64_t)p.d_out + 3) / 4 * p.m + PS_THREADS > 0xFFFFFFFFll) return hipErrorNotSupported;
    const hipError_t e = launch<true, false, 2, S>(q, parts, stride);
    if (e != hipSuccess) return e;
    switch (parts) {
    case 2: launch_sums<2>(p, stride, q.ldy); break;
    case 3: launch_sums<3>(p, stride, q.ldy); break;
    case 4: launch_sums<4>(p, stride, q.ldy); break;
    case 6: launch_sums<6>(p, stride, q.ldy); break;
    case 8: launch_sums<8>(p, stride, q.ldy); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

using Shape256 = Shape<2, 8, 4, 4>;
using Shape128 = Shape<4, 4, 2, 4>;
using Shape64 = Shape<8, 2, 1, 4>;

template <typename S> hipError_t launch_either(const Product &p, int parts) {
    if (parts > 1) return launch_parts<S>(p, parts);
    return p.i8 ? launch_shape<true, S>(p) : launch_shape<false, S>(p);
}

}  // namespace

// Whole 16 bytes everywhere, and offsets from a tile's or an expert's first row that 31 bits hold (with what a stage goes past a row); rows that
// are gathered come from anywhere, so that all of X has to lie within.
bool product_wide_supported(const Product &p) {
    const int64_t e = p.i8 ? 1 : 2, most = 0x7FFFFFFF - 2 * PW_KB;
    auto whole = [](int64_t v) { return v % 16 == 0; };
    if (!whole(p.d_in * e) || !whole(p.ldx * e) || !whole(p.ldw * e) || !whole(p.expert_stride * e) || (reinterpret_cast<uintptr_t>(p.X) & 15) ||
        (reinterpret_cast<uintptr_t>(p.W) & 15))
        return false;
    const int64_t outs = (int64_t)p.d_out * (p.gated ? 2 : 1), x_rows = p.rows ? p.x_rows : p.m < 256 ? p.m : 256;
    return p.ldw * e <= most / outs && p.ldx * e <= most / x_rows;
}

hipError_t launch_product_wide(const Product &p, int tile_rows, int parts) {
    if (tile_rows <= 64) return launch_either<Shape64>(p, parts);
    if (tile_rows <= 128) return launch_either<Shape128>(p, parts);
    return launch_either<Shape256>(p, parts);
}

}  // namespace qamw
