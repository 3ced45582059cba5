// Y = X W^T for few rows: what is read of W is what it costs.  8-bit integers with scales or bf16, one matrix or one for each expert.
//
// A wave has 16 rows of W (gated: 16 of the gate and the same 16 of the up projection), up to 64 rows of X and a share of the columns, in
// units of 128 bytes.  Units come to the wave's own ring in LDS by buffer loads that go there directly, whole 128-byte lines of
// eight rows at a time; no barrier is needed until the waves that share rows of W add up what they have.
//   In LDS the eight 16-byte pieces of a row are exchanged by row mod 8, against bank conflicts of the 16 lanes that read a column.
// What bounds it: one CU gets 45 to 58 GB/s of weights that come from memory, however many it asks for at once, so tiles share their
// columns among waves until there are about 8 on every CU; with enough of them, memory.  Launches included: 4096 x 4096 int8 for 8 rows 6.4 us,
// 11008 x 4096 12.1, 5120 x 13824 19.1 (3.7 TB/s); gated int8 of 8 experts of 2 x 5632 x 2048 for 10 rows 27 us; bf16 of 64 experts of
// 1408 x 2048 with 8 rows each 70.6 us (5.2 TB/s).
//   Rows of X are read again for every 16 outputs, from the caches, so that many rows are dearer here than in tiles of 256 outputs; the
// estimate that chooses has both sides.
// Few values, quantised in the call: the workgroup's waves quantise the rows while their first weights are on their way.  Every
// workgroup does so again.  Against a launch for it, in a graph: one row by 4096 x 4096 6.9 us (8.1), of 11008 columns 13.1 (15.2), 4 rows
// of 4096 columns 9.9 (8.3); called one by one, a launch less is 4 us less of the host's time.  13 rows of 5632 took 18.6 us, in two launches
// 8.5: so no more values than the threads hold in four groups of 8.
#include "qamw_product_tile.hpp"

namespace qamw {
namespace {

constexpr int PF_UNIT = 128, PF_SLOT = 16 * PF_UNIT;            // 16 rows of a unit
constexpr int PF_ONCE = 2;                                     // cache policy of a load: not kept (nt)
constexpr uint32_t PF_NOWHERE = 0x80000000u;                    // added to an offset: beyond the end of any buffer here
// FROM: where X comes from: -1 as the product takes it, from memory; 0 fp32 and 1 bf16 to be quantised here, EIGHTS groups of 8
// values by a thread.
template <int T_, int FN_, int FROM_ = -1, int EIGHTS_ = 1> struct FewShape {
    static constexpr int T = T_, FN = FN_, FROM = FROM_, EIGHTS = EIGHTS_, XT = FROM >= 0 ? 0 : T;   // XT: fragments of X in the ring
    static constexpr int SLOT = (FN + XT) * PF_SLOT;
    // Workgroups of 4 waves, two or more on a CU, share the CUs more evenly than ones of 8 (288 rows routed to those 64 experts 58 us a call
    // and 10 to the 8 21 us, 71 and 27 with ones of 8); one that quantises has 8 for it.
    static constexpr int WAVES = FROM >= 0 ? 8 : 4;
    static constexpr int FIT = 80 * 1024 / (WAVES * SLOT), RING = FROM >= 0 || FIT > 4 ? 4 : FIT < 2 ? 2 : FIT;   // units on their way or being read
    static constexpr int THREADS = WAVES * WAVE, BM = T * 16;
    static constexpr int LDS = WAVES * RING * SLOT;
};

struct FewArgs {
    ProductArgs p;
    int col_tiles, split;                                       // waves that share a tile of columns
    const void *xf;                                             // rows to be quantised here
    const float *col_scale;
    int64_t ldxf;
};

// N fragments from `at` on, complete when this returns: rows are 128 bytes apart, `piece` is where the lane's 16 bytes are.
template <int N> __device__ __forceinline__ void read_unit(uint32_t at, pr_i32x4_t (&v)[N]) {
    static_assert(N >= 1 && N <= 6, "");
    if constexpr (N == 1)
        asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v[0]) : "v"(at) : "memory");
    else if constexpr (N == 2)
        asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:2048\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v[0]), "=&v"(v[1]) : "v"(at) : "memory");
    else if constexpr (N == 3)
        asm volatile("ds_read_b128 %0, %3\n\tds_read_b128 %1, %3 offset:2048\n\tds_read_b128 %2, %3 offset:4096\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2])
                     : "v"(at)
                     : "memory");
    else if constexpr (N == 4)
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:2048\n\tds_read_b128 %2, %4 offset:4096\n\tds_read_b128 %3, %4 offset:6144\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
                     : "v"(at)
                     : "memory");
    else if constexpr (N == 5)
        asm volatile("ds_read_b128 %0, %5\n\tds_read_b128 %1, %5 offset:2048\n\tds_read_b128 %2, %5 offset:4096\n\tds_read_b128 %3, %5 offset:6144\n\t"
                     "ds_read_b128 %4, %5 offset:8192\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4])
                     : "v"(at)
                     : "memory");
    else
        asm volatile("ds_read_b128 %0, %6\n\tds_read_b128 %1, %6 offset:2048\n\tds_read_b128 %2, %6 offset:4096\n\tds_read_b128 %3, %6 offset:6144\n\t"
                     "ds_read_b128 %4, %6 offset:8192\n\tds_read_b128 %5, %6 offset:10240\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5])
                     : "v"(at)
                     : "memory");
}

template <bool I8, bool GATED, bool YBF16, bool ONCE, typename S>
__global__ __launch_bounds__(S::THREADS) void k_product_few(FewArgs q) {
    using M = Mfma<I8>;
    const ProductArgs &a = q.p;
    extern __shared__ __align__(16) char pf_lds[];
    const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
    const int per = S::WAVES / q.split;                                        // tiles of columns of a workgroup
    const int groups = (q.col_tiles + per - 1) / per;
    const RowTile rt = find_tile<S::BM>(a, (int)(blockIdx.x / (uint32_t)groups));
    if (rt.n <= 0) return;
    const int ct = (int)(blockIdx.x % (uint32_t)groups) * per + wave / q.split, part = wave % q.split;
    const int bytes = a.d_in * M::ELEM, units = (bytes + PF_UNIT - 1) / PF_UNIT;
    const int u0 = (int)((int64_t)units * part / q.split), u1 = ct < q.col_tiles ? (int)((int64_t)units * (part + 1) / q.split) : u0;

    // fragment f, row r of W: its output (gated: fragments in pairs, 16 of the gate and the same 16 of up)
    auto out_of = [&](int f, int r) { return (GATED ? ct * (S::FN / 2) + f / 2 : ct * S::FN + f) * 16 + r; };
    const char *wp = a.W + (int64_t)rt.expert * a.expert_stride;
    const char *xp = a.rows ? a.X : a.X + (int64_t)rt.row0 * a.ldx;
    const int lr = lane >> 3, piece = ((lane & 7) ^ lr) * 16;
    const bool past = (units - 1) * PF_UNIT + piece >= bytes;
    uint32_t off_w[S::FN][2], off_x[S::XT ? S::XT : 1][2];
#pragma unroll
    for (int f = 0; f < S::FN; ++f)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int o = out_of(f, h * 8 + lr);
            const int64_t row = GATED && (f & 1) ? a.d_out + (int64_t)o : o;
            off_w[f][h] = o < a.d_out ? (uint32_t)(row * a.ldw) + piece : PF_NOWHERE;
        }
#pragma unroll
    for (int t = 0; t < S::XT; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = t * 16 + h * 8 + lr;
            const bool is = r < rt.n;
            int row = is ? r : 0;
            if (a.rows && is) row = min(max(a.rows[rt.row0 + r], 0), a.x_rows - 1);
            off_x[t][h] = is ? (uint32_t)((int64_t)row * a.ldx) + piece : PF_NOWHERE;
        }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)pf_lds, ring = lds0 + wave * (S::RING * S::SLOT);
    constexpr int L = 2 * (S::FN + S::XT);
    auto request = [&](int u) {
        const int records = u < u1 ? 0x7FFFFFFF : 0;
        const auto wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(wp), 0, records, 0x00020000);
        const auto xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(xp), 0, records, 0x00020000);
        const uint32_t to = ring + (uint32_t)((u - u0) % S::RING) * S::SLOT, gone = u == units - 1 && past ? PF_NOWHERE : 0;
#pragma unroll
        for (int f = 0; f < S::FN; ++f)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (__attribute__((address_space(3))) void *)(uintptr_t)(to + f * PF_SLOT + h * 1024), 16,
                                                         (int)(off_w[f][h] | gone), u * PF_UNIT, 0, ONCE ? PF_ONCE : 0);
#pragma unroll
        for (int t = 0; t < S::XT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (__attribute__((address_space(3))) void *)(uintptr_t)(to + (S::FN + t) * PF_SLOT + h * 1024),
                                                         16, (int)(off_x[t][h] | gone), u * PF_UNIT, 0, 0);
    };
    // what the last step needs, asked for first
    const int fr = lane & 15, q0 = (lane >> 4) * 4;
    float xs[S::T], ws[S::FN][4];
    if (I8) {
        const float *from = a.w_scales + (int64_t)rt.expert * a.d_out * (GATED ? 2 : 1);
#pragma unroll
        for (int f = 0; f < S::FN; ++f)
            for (int k = 0; k < 4; ++k) ws[f][k] = from[min(out_of(f, q0 + k), a.d_out - 1) + (GATED && (f & 1) ? a.d_out : 0)];
        if (S::FROM < 0)
#pragma unroll
            for (int t = 0; t < S::T; ++t) {
                const int r = rt.row0 + min(t * 16 + fr, rt.n - 1);
                xs[t] = a.x_scales[a.rows ? min(max(a.rows[r], 0), a.x_rows - 1) : r];
            }
    }
    // the rows to be quantised are asked for before the weights, or they would be waited for together
    constexpr int SPAN = S::THREADS * 8;
    const int spans = (a.d_in + SPAN - 1) / SPAN;                              // m * spans <= EIGHTS
    Eight<(S::FROM == 1)> raw[S::EIGHTS];
    Eight<0> col[S::EIGHTS];
    if constexpr (S::FROM >= 0) {
        const auto xf = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(q.xf), 0, 0x7FFFFFFF, 0x00020000);
        const auto cs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(q.col_scale), 0, q.col_scale ? 0x7FFFFFFF : 0, 0x00020000);
#pragma unroll
        for (int i = 0; i < S::EIGHTS; ++i) {
            const int r = i / spans, j = (i % spans) * SPAN + tid * 8;
            const uint32_t gone = r < a.m && j < a.d_in ? 0 : PF_NOWHERE;
            raw[i].load(xf, (uint32_t)((r * (uint32_t)q.ldxf + j) * (S::FROM ? 2 : 4)) | gone);
            col[i].load(cs, (uint32_t)(j * 4) | gone);
        }
    }
#pragma unroll
    for (int i = 0; i < S::RING; ++i) request(u0 + i);

    // the rows of X as codes, a pitch of units * 128 + 16 bytes apart, behind the rings
    const uint32_t x_pitch = units * PF_UNIT + 16, x_at = lds0 + S::LDS;
    if constexpr (S::FROM >= 0) {
        const uint32_t most_of = x_at + a.m * x_pitch;                        // [EIGHTS][WAVES], behind the codes
        float v[S::EIGHTS][8];
#pragma unroll
        for (int i = 0; i < S::EIGHTS; ++i) {
            uint32_t most = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[i][k] = raw[i].value(k);
                if (q.col_scale) v[i][k] *= col[i].value(k);
                most = max(most, __float_as_uint(v[i][k]) & 0x7FFFFFFFu);
            }
            most = wave_max(most);
            if (lane == 0) lds_write<uint32_t>(most_of + (i * S::WAVES + wave) * 4, most);
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int i = 0; i < S::EIGHTS; ++i) {
            const int r = i / spans, j = (i % spans) * SPAN + tid * 8;
            if (r >= a.m) continue;
            uint32_t most = 0;
            for (int s = 0; s < spans; ++s)
                most = max(most, lds_read<uint32_t>(most_of + ((S::EIGHTS == 1 ? 0 : r * spans + s) * S::WAVES + lane % S::WAVES) * 4));
            const Quantiser z(wave_max(most));
            if (fr == r) xs[0] = z.scale;
            if (j < units * PF_UNIT) {                                        // beyond d_in: zeros, which v holds there
                uint32_t c[2] = {0, 0};
#pragma unroll
                for (int k = 0; k < 8; ++k) c[k / 4] |= z.code(v[i][k]) << (k % 4 * 8);
                lds_write<uint64_t>(x_at + r * x_pitch + j, (uint64_t)c[1] << 32 | c[0]);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }

    const uint32_t mine = (uint32_t)(fr * PF_UNIT);
    const uint32_t x_mine = x_at + min(fr, a.m - 1) * x_pitch + (lane >> 4) * 16;
    typename M::acc_t acc[S::FN][S::T] = {};
    for (int u = u0; u < u1; ++u) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S::RING - 1) * L) : "memory");
        const uint32_t slot = ring + (uint32_t)((u - u0) % S::RING) * S::SLOT + mine;
        pr_i32x4_t f0[S::FN + S::XT], f1[S::FN + S::XT], x0[1], x1[1];
        read_unit<S::FN + S::XT>(slot + (((lane >> 4) ^ (fr & 7)) * 16), f0);
        read_unit<S::FN + S::XT>(slot + (((4 + (lane >> 4)) ^ (fr & 7)) * 16), f1);
        if constexpr (S::FROM >= 0) {
            read_unit<1>(x_mine + u * PF_UNIT, x0);
            read_unit<1>(x_mine + u * PF_UNIT + 64, x1);
        }
        request(u + S::RING);
#pragma unroll
        for (int f = 0; f < S::FN; ++f)
#pragma unroll
            for (int t = 0; t < S::T; ++t) {
                acc[f][t] = M::mul(f0[f], S::FROM >= 0 ? x0[0] : f0[S::FROM >= 0 ? 0 : S::FN + t], acc[f][t]);
                acc[f][t] = M::mul(f1[f], S::FROM >= 0 ? x1[0] : f1[S::FROM >= 0 ? 0 : S::FN + t], acc[f][t]);
            }
    }

    // the shares of the columns are added in their order, in LDS, where the ring was
    if (q.split > 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int f = 0; f < S::FN; ++f)
#pragma unroll
            for (int t = 0; t < S::T; ++t)
                *reinterpret_cast<__attribute__((address_space(3))) pr_i32x4_t *>((uintptr_t)(ring + (f * S::T + t) * 1024 + lane * 16)) =
                    __builtin_bit_cast(pr_i32x4_t, acc[f][t]);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (part != 0) return;
#pragma unroll
        for (int f = 0; f < S::FN; ++f)
#pragma unroll
            for (int t = 0; t < S::T; ++t)
                for (int s = 1; s < q.split; ++s)
                    acc[f][t] += __builtin_bit_cast(typename M::acc_t, *reinterpret_cast<__attribute__((address_space(3))) pr_i32x4_t *>(
                                                                           (uintptr_t)(ring + s * (S::RING * S::SLOT) + (f * S::T + t) * 1024 + lane * 16)));
    }

#pragma unroll
    for (int f = 0; f < S::FN; f += GATED ? 2 : 1) {
        const int o = out_of(f, q0), there = ct < q.col_tiles ? a.d_out - o : 0;
        if (there <= 0) continue;
#pragma unroll
        for (int t = 0; t < S::T; ++t) {
            const int r = t * 16 + fr;
            if (r >= rt.n) continue;
            float y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                y[k] = (float)acc[f][t][k];
                if (I8) y[k] = y[k] * xs[t] * ws[f][k];
                if (GATED) {
                    float u = (float)acc[GATED ? f + 1 : f][t][k];
                    if (I8) u = u * xs[t] * ws[GATED ? f + 1 : f][k];
                    y[k] = silu(y[k]) * u;
                }
            }
            store_y4<YBF16>(a.Y, (int64_t)(rt.row0 + r) * a.ldy + o, y, there);
        }
    }
}

template <bool I8, bool GATED, bool YBF16, bool ONCE, typename S> hipError_t launch_once(const Product &p, const FewArgs &given, size_t more_lds) {
    FewArgs q = given;
    const int outs = (GATED ? S::FN / 2 : S::FN) * 16;
    const int64_t cols = ((int64_t)p.d_out + outs - 1) / outs, rows = most_row_tiles(p, S::BM);
    const int units = (int)((p.d_in * (I8 ? 1 : 2) + PF_UNIT - 1) / PF_UNIT);
    const int split = few_split((p.offsets && p.m < p.n_experts ? p.m : rows) * cols, units, S::WAVES);
    const int per = S::WAVES / split;
    const int64_t blocks = rows * ((cols + per - 1) / per);
    if (cols > 0x7FFFFFFF || blocks * S::THREADS > 0xFFFFFFFFll) return hipErrorNotSupported;
    q.p = args_of(p);
    q.col_tiles = (int)cols;
    q.split = split;
    const auto kernel = &k_product_few<I8, GATED, YBF16, ONCE, S>;
    static MoreLds more;
    const hipError_t e = more.ask(reinterpret_cast<const void *>(kernel), 160 * 1024);
    if (e != hipSuccess) return e;
    kernel<<<dim3((uint32_t)blocks), S::THREADS, S::LDS + more_lds, p.stream>>>(q);
    return hipGetLastError();
}

// Weights of which half the Infinity Cache would be full are read as what is not read again, where an expert's rows are a tile or so: 64 experts
// of 1408 x 2048 bf16 with 8 rows each 70.6 us, 75.6 by ordinary loads, 8 of 11008 x 4096 134 and 147; with 20 rows each 91.2 and 91.4, with
// 40 99.6 and 96.3.  Not where rows are off the 128-byte lines, whose other part the next unit asks for: 64 of 1408 x 2064 92.9 and 85.9, 8 of
// 11008 x 4112 197 and 180.  Smaller weights may be found there again: 13824 x 5120 int8, over and over, 24.1 and 19.4.
constexpr int64_t PF_KEPT = 128ll << 20;
template <bool I8, bool GATED, bool YBF16, typename S> hipError_t launch(const Product &p, const FewArgs &q, size_t more_lds) {
    const int64_t bytes = (int64_t)p.n_experts * p.d_out * (p.gated ? 2 : 1) * p.d_in * (I8 ? 1 : 2);
    constexpr bool MAY = S::FROM < 0 && S::T == 1;
    const bool on_lines = (p.ldw * (I8 ? 1 : 2) % 128 | p.expert_stride * (I8 ? 1 : 2) % 128 | (int64_t)(reinterpret_cast<uintptr_t>(p.W) % 128)) == 0;
    return MAY && on_lines && bytes > PF_KEPT ? launch_once<I8, GATED, YBF16, MAY, S>(p, q, more_lds) : launch_once<I8, GATED, YBF16, false, S>(p, q, more_lds);
}

template <bool I8, int T, int FROM, int EIGHTS> hipError_t launch_shape(const Product &p, const FewArgs &q, size_t more_lds) {
    using Gated = FewShape<T, 2, FROM, EIGHTS>;
    using Plain = FewShape<T, 1, FROM, EIGHTS>;
    if (p.gated) return p.y_bf16 ? launch<I8, true, true, Gated>(p, q, more_lds) : launch<I8, true, false, Gated>(p, q, more_lds);
    return p.y_bf16 ? launch<I8, false, true, Plain>(p, q, more_lds) : launch<I8, false, false, Plain>(p, q, more_lds);
}

template <bool I8> hipError_t launch_type(const Product &p, int tile_rows) {
    const FewArgs q = {};
    if (tile_rows <= 16) return launch_shape<I8, 1, -1, 1>(p, q, 0);
    if (tile_rows <= 32) return launch_shape<I8, 2, -1, 1>(p, q, 0);
    return launch_shape<I8, 4, -1, 1>(p, q, 0);
}

}  // namespace

hipError_t launch_product_few(const Product &p, int tile_rows) { return p.i8 ? launch_type<true>(p, tile_rows) : launch_type<false>(p, tile_rows); }

// As many values as the threads of a workgroup hold, and rows that are read in whole 16 bytes, with offsets that 31 bits hold.
constexpr int PF_MOST_EIGHTS = 4, PF_SPAN = 8 * 8 * WAVE;

bool product_from_floats_supported(const Product &p, const void *X, int dtype, int64_t ldx, const float *col_scale) {
    const int64_t spans = ((int64_t)p.d_in + PF_SPAN - 1) / PF_SPAN, e = dtype == 0 ? 4 : 2;
    return p.m * spans <= PF_MOST_EIGHTS && (reinterpret_cast<uintptr_t>(X) & 15) == 0 && (reinterpret_cast<uintptr_t>(col_scale) & 15) == 0 &&
           ldx * e % 16 == 0 && ldx * e <= 0x7FFFFFFF / PF_MOST_EIGHTS;
}

template <int EIGHTS> static hipError_t from_floats(const Product &p, const FewArgs &q, int dtype, size_t codes) {
    return dtype == 0 ? launch_shape<true, 1, 0, EIGHTS>(p, q, codes) : launch_shape<true, 1, 1, EIGHTS>(p, q, codes);
}

hipError_t launch_product_from_floats(const Product &p, const void *X, int dtype, int64_t ldx, const float *col_scale) {
    FewArgs q = {};
    q.xf = X;
    q.ldxf = ldx;
    q.col_scale = col_scale;
    const size_t codes = (size_t)p.m * (((size_t)p.d_in + PF_UNIT - 1) / PF_UNIT * PF_UNIT + 16) + PF_MOST_EIGHTS * 8 * 4;   // and the waves' maxima
    return p.m == 1 && p.d_in <= PF_SPAN ? from_floats<1>(p, q, dtype, codes) : from_floats<PF_MOST_EIGHTS>(p, q, dtype, codes);
}

}  // namespace qamw
