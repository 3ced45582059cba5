// Routed experts: the choice of experts, the order of the rows, and the way back.
#include "qamw_product_tile.hpp"

namespace qamw {
namespace {

constexpr int RT_WAVES = 16, RT_THREADS = RT_WAVES * WAVE;

// ---- choice ---------------------------------------------------------------------------------------------------------------
//
// Sixteen lanes have a token, so that the largest of its logits is found by DPP within a row of lanes, for four tokens of a wave at a
// time; a lane has PER experts that follow one another.  A logit becomes an unsigned number that orders as it does.
// bf16 leaves room for the expert below it, the lowest one as the largest number, so that one maximum finds both, and the next one is the
// largest that is smaller: of numbers below 2^31 it has the largest difference to the last one as an unsigned number.  fp32 takes the lowest lane that has the maximum, and the lowest of its experts, and strikes it out.
//   Arithmetic bounds it, and the way through memory next: 16384 tokens over 256 experts, 8 of them chosen, 10.2 us, of which some 5 are
// instructions, 2 the logits' 8.4 MB, the rest a launch and the steps between (12.4 where a choice was struck out, and values were made of numbers
// again for the sum).  With 64 lanes for a token the whole routing took 31.6 us, with sixteen 16.4.
constexpr int RT_LANES = 16, RT_GROUPS = WAVE / RT_LANES;
// Tokens of a workgroup of the first launch, and so the most that it can count for an expert: 8 bits hold it.  A workgroup's counts lie in
// sectors of 32 bytes of their own, so that no two write to one.
constexpr int RT_TOKENS = RT_GROUPS * RT_WAVES;
__host__ __device__ constexpr int counts_row(int n_experts) { return (n_experts + 31) / 32 * 32; }

__device__ __forceinline__ uint32_t row_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));    // lane ^ 1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));    // lane ^ 2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false));   // the other four of eight
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false));   // the other eight of sixteen
    return v;
}
__device__ __forceinline__ float row_sum(float v) {
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xF, 0xF, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xF, 0xF, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xF, 0xF, false));
    return v;
}
// NaN as -inf, -0 as 0; -inf and what lies below it are never chosen
__device__ __forceinline__ float clean(float f) { return fmaxf(f + 0.0f, -__builtin_inff()); }
constexpr uint32_t RT_LEAST = 0x00800000u;                  // the key of the lowest finite value
__device__ __forceinline__ uint32_t key_of(float f) {
    const uint32_t u = __float_as_uint(f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
// exp(x - top), x <= top; infinities of one sign are equal: their difference is no number, and 0 the smaller of the two
__device__ __forceinline__ float share_of(float x, float top) { return __expf(fminf(x - top, 0.0f)); }

// Lane j of a token's sixteen gets its choices j and j + 16: the experts (-1: none) and weights.  t >= m: none.
template <int DTYPE, int PER>
__device__ __forceinline__ void pick(const RouteProblem &q, int64_t t, int (&expert)[2], float (&weight)[2]) {
    constexpr bool PACKED = DTYPE == 1;
    const int lane = threadIdx.x % RT_LANES, n = q.n_experts, e0 = lane * PER;
    using E = typename Elem<DTYPE>::type;
    uint32_t key[PER];
    Unaligned<E, PER> row;                                  // wherever it lies: the memory instructions take any address
    const bool whole = t < q.m && e0 + PER <= n;
    if (whole) row = *reinterpret_cast<const Unaligned<E, PER> *>(static_cast<const E *>(q.logits) + t * q.ld + e0);
    else
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (DTYPE == 1) row.v[i] = (E)0xFF80u;          // -inf
            else row.v[i] = (E)-__builtin_inff();
            if (t < q.m && e0 + i < n) row.v[i] = static_cast<const E *>(q.logits)[t * q.ld + e0 + i];
        }
    auto logit = [&](int i) { return clean(DTYPE == 1 ? __uint_as_float((uint32_t)row.v[i] << 16) : (float)row.v[i]); };
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        key[i] = key_of(logit(i));
        if (PACKED) key[i] = (key[i] >> 16 << 10 | (1023u - (uint32_t)e0)) - i;   // e0 + i <= 1023: no borrow
    }
    constexpr uint32_t LEAST = PACKED ? RT_LEAST >> 16 << 10 : RT_LEAST;
    // of a packed key all that a negative value lacks are ones
    auto value = [](uint32_t k) { return value_of(PACKED ? (k >> 10 << 16) | (k & 0x2000000u ? 0u : 0xFFFFu) : k); };
    float total = 0.0f, top = 0.0f, mine[2] = {0.0f, 0.0f};
    expert[0] = expert[1] = -1;
    uint32_t best = 0;
    bool some = true;
    for (int j = 0; j < q.k; ++j) {
        const uint32_t last = PACKED ? best : 0;
        uint32_t own = key[0] - last;
#pragma unroll
        for (int i = 1; i < PER; ++i) own = max(own, key[i] - last);
        best = last + row_max(own);
        some = some && best >= LEAST;                       // a token that has run out of experts stays so
        if (!__any(some)) break;
        const float v = value(best);
        if (j == 0) {
            top = v;
            if (!q.renormalise) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < PER; ++i) sum += share_of(PER > 32 ? value(key[i]) : logit(i), top);   // no registers for both
                total = row_sum(sum);
            }
        }
        int who;
        if (PACKED) {
            who = (int)(1023u - (best & 1023u));
        } else {
            const uint32_t has = (uint32_t)(__ballot(own == best) >> (threadIdx.x % WAVE / RT_LANES * RT_LANES)) & 0xFFFFu;
            const int winner = __ffs((int)has) - 1;
            int at = 0;
#pragma unroll
            for (int i = PER - 1; i >= 0; --i) at = key[i] == best ? i : at;
            who = __shfl(e0 + at, winner, RT_LANES);
            at = lane == winner ? at : -1;
#pragma unroll
            for (int i = 0; i < PER; ++i) key[i] = i == at ? 0 : key[i];
        }
        const float p = some ? share_of(v, top) : 0.0f;
        if (q.renormalise) total += p;
        if (some && lane == j % RT_LANES) {
            expert[j / RT_LANES] = who;
            mine[j / RT_LANES] = p;
        }
    }
    for (int h = 0; h < 2; ++h) weight[h] = expert[h] >= 0 ? mine[h] / total : 0.0f;
}

// ---- order ----------------------------------------------------------------------------------------------------------------
//
// A stable counting sort of the slots (token after token, choice after choice).  A wave has the slots of the tokens that follow one
// another and finds equal experts among 64 slots by the bits of the expert; a workgroup's counts are those of its waves in their
// order, a launch's those of its workgroups.  What is written as a slot's position is first the slot's rank among those of its
// expert in the workgroup; when all counts are known, what comes before is added: what comes before an expert, and before the
// workgroup within the expert.  A single workgroup knows all counts by itself: up to 64 tokens are one launch (5 tokens, 8 experts 3.4 us),
// more are two: a workgroup of the second sums the counts of all and of those before it, so none waits for another.  What it reads of
// them bounds that: 16384 tokens over 256 experts 6.1 us with counts of 8 bits, four experts' to a load, 8.5 with ones of 32 bits.
//   Every workgroup reads all workgroups' counts, (m / 64)^2 bytes an expert, so that the second launch's time grows with the square of the tokens and
// is most of a large call: over 256 experts, 8 of them chosen, both launches take 27 us for 32768 tokens, 128 for 131072, 381 for 262144 and 4.7 ms
// for 1048576.

// Exclusive sums of the counts in `total` (LDS), by one wave; their sum.
__device__ __forceinline__ uint32_t exclusive(uint32_t *total, int n) {
    const int lane = threadIdx.x % WAVE;
    uint32_t before = 0;
    for (int e0 = 0; e0 < n; e0 += WAVE) {
        const int e = e0 + lane;
        const uint32_t c = e < n ? total[e] : 0;
        uint32_t upto = c;
        for (int d = 1; d < WAVE; d <<= 1) {
            const uint32_t v = (uint32_t)__shfl_up((int)upto, d);
            if (lane >= d) upto += v;
        }
        if (e < n) total[e] = before + upto - c;
        before += (uint32_t)__builtin_amdgcn_readlane((int)upto, WAVE - 1);
    }
    return before;
}

template <int DTYPE, int PER, bool ALONE>
__global__ __launch_bounds__(RT_THREADS) void k_route_pick(RouteProblem q) {
    extern __shared__ uint32_t rt_lds[];                    // [RT_WAVES][n_experts]: counts, then what comes before them
    __shared__ uint32_t all;
    const int n = q.n_experts, k = q.k, lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    uint32_t *mine = rt_lds + wave * n, *total = rt_lds + RT_WAVES * n;
    for (int i = threadIdx.x; i < RT_WAVES * n; i += RT_THREADS) rt_lds[i] = 0;
    __syncthreads();
    const int t0 = (blockIdx.x * RT_WAVES + wave) * RT_GROUPS, t1 = min(t0 + RT_GROUPS, q.m);
    // lane's slots, of the tokens that are ranked together: token g0 + lane / k, choice lane % k
    const int at_once = k <= RT_LANES ? RT_GROUPS : 2, token = lane / k, choice = lane % k;
    int slot_expert[2] = {-1, -1}, slot_rank[2] = {-1, -1};
    if (t0 < t1) {
        int expert[2];
        float weight[2];
        pick<DTYPE, PER>(q, t0 + lane / RT_LANES, expert, weight);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int g0 = t0 + h * at_once;
            if (g0 >= t0 + RT_GROUPS || g0 >= t1) break;
            const int from = ((h * at_once + token) % RT_GROUPS) * RT_LANES + choice % RT_LANES;
            const bool is = token < at_once && g0 + token < t1;
            const int lo = __shfl(expert[0], from), hi = __shfl(expert[1], from);
            const float wlo = __shfl(weight[0], from), whi = __shfl(weight[1], from);
            const int e = !is ? -1 : choice < RT_LANES ? lo : hi;
            asm volatile("" ::: "memory");                   // the counts of the tokens before are other lanes' work: read no earlier than here
            unsigned long long same = __ballot(e >= 0);
            for (int b = 0; b < 10; ++b) {
                const unsigned long long has = __ballot((e >> b) & 1);
                same &= (e >> b) & 1 ? has : ~has;
            }
            if (is) {
                const int64_t at = (int64_t)g0 * k + lane;
                if (e >= 0) {
                    const int rank = (int)mine[e] + __popcll(same & ((1ull << lane) - 1));
                    // the wave's LDS accesses are made in order: all ranks are read before the last slot of an expert counts them
                    if ((same >> lane) == 1) mine[e] = (uint32_t)rank + 1;
                    slot_rank[h] = rank;
                    slot_expert[h] = e;
                } else
                    q.positions[at] = -1;
                q.experts[at] = e;
                q.weights[at] = choice < RT_LANES ? wlo : whi;
            }
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < n; e += RT_THREADS) {
        uint32_t before = 0;
        for (int w = 0; w < RT_WAVES; ++w) {
            const uint32_t c = rt_lds[w * n + e];
            rt_lds[w * n + e] = before;
            before += c;
        }
        if (ALONE) total[e] = before;
        else q.counts[(int64_t)blockIdx.x * counts_row(n) + e] = (uint8_t)before;
    }
    __syncthreads();
    if (ALONE) {
        if (wave == 0) {
            const uint32_t sum = exclusive(total, n);
            if (lane == 0) all = sum;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < n; e += RT_THREADS) q.offsets[e] = (int32_t)total[e];
        if (threadIdx.x == 0) q.offsets[n] = (int32_t)all;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int e = slot_expert[h];
        if (e < 0) continue;
        const uint32_t place = (ALONE ? total[e] : 0) + mine[e] + (uint32_t)slot_rank[h];
        q.positions[(int64_t)(t0 + h * at_once) * k + lane] = (int32_t)place;
        if (ALONE) q.rows[place] = t0 + h * at_once + token;
    }
    if (ALONE)
        for (int p = (int)all + threadIdx.x; p < q.m * k; p += RT_THREADS) q.rows[p] = -1;
}

// `lanes` threads, a power of two, have four experts each; RT_THREADS / lanes of them share the sums of the experts' counts.
__global__ __launch_bounds__(RT_THREADS) void k_route_order(RouteProblem q, int tokens, int blocks, int lanes) {
    extern __shared__ uint32_t rt_lds[];
    uint32_t *before = rt_lds, *total = rt_lds + q.n_experts;   // [n_experts] each: of the workgroups before, of all
    __shared__ uint32_t all;
    const int n = q.n_experts, k = q.k;
    for (int i = threadIdx.x; i < 2 * n; i += RT_THREADS) rt_lds[i] = 0;
    __syncthreads();
    const int e0 = threadIdx.x % lanes * 4, segment = threadIdx.x / lanes, segments = RT_THREADS / lanes, row = counts_row(n);
    if (e0 < n) {
        constexpr int MOST = 0xFFFF / RT_TOKENS;            // counts that 16 bits hold the sum of
        for (int i0 = segment; i0 < blocks; i0 += segments * MOST) {
            uint32_t b[2] = {0, 0}, t[2] = {0, 0};          // experts e0 and e0 + 2, e0 + 1 and e0 + 3
            const int i1 = min((int64_t)blocks, i0 + (int64_t)segments * MOST);
#pragma unroll 8
            for (int i = i0; i < i1; i += segments) {
                const uint32_t c = *reinterpret_cast<const uint32_t *>(q.counts + (int64_t)i * row + e0), even = c & 0xFF00FF, odd = c >> 8 & 0xFF00FF;
                const bool is = i < (int)blockIdx.x;
                t[0] += even;
                t[1] += odd;
                b[0] += is ? even : 0;
                b[1] += is ? odd : 0;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e0 + j < n) {                           // whole numbers: their order changes nothing
                    atomicAdd(&before[e0 + j], b[j & 1] >> (j / 2 * 16) & 0xFFFF);
                    atomicAdd(&total[e0 + j], t[j & 1] >> (j / 2 * 16) & 0xFFFF);
                }
        }
    }
    __syncthreads();
    if (threadIdx.x < WAVE) {
        const uint32_t sum = exclusive(total, n);
        if (threadIdx.x == 0) all = sum;
    }
    __syncthreads();
    if (blockIdx.x == 0) {
        for (int e = threadIdx.x; e < n; e += RT_THREADS) q.offsets[e] = (int32_t)total[e];
        if (threadIdx.x == 0) q.offsets[n] = (int32_t)all;
    }
    const int64_t slots = (int64_t)q.m * k, s0 = (int64_t)blockIdx.x * tokens * k, s1 = min(s0 + (int64_t)tokens * k, slots);
    for (int64_t s = s0 + threadIdx.x; s < s1; s += RT_THREADS) {
        const int e = q.experts[s];
        if (e >= 0) {
            const uint32_t place = total[e] + before[e] + (uint32_t)q.positions[s];
            q.positions[s] = (int32_t)place;
            q.rows[place] = (int32_t)(s / k);
        }
    }
    // places that no slot has
    for (int64_t p = (int64_t)all + (int64_t)blockIdx.x * RT_THREADS + threadIdx.x; p < slots; p += (int64_t)blocks * RT_THREADS)
        q.rows[p] = -1;
}

// ---- the way back ---------------------------------------------------------------------------------------------------------

constexpr int CB_THREADS = 256;

// A thread has eight neighbours of a token's row, wherever they lie: the memory instructions take any address.  What it reads of
// the experts' rows it asks for eight rows at a time.  Memory bounds it: 8192 tokens of 8 rows of 4096 bf16 in 104 us, 5.8 TB/s; one value a
// thread, one row at a time took 312.  5 tokens of 2 rows 3.4 us, a launch.
//   The last d % 8 columns are one thread's, which asks for one value at a time and waits for it: 8192 tokens of 8 rows of 4097 take 128 us, of 4095
// 212 (fp32: 262 and 344, 237 of 4096), 100 tokens of 4095 14.5 against 7.2.
// Rows that are read once, and a layer's are many: what passes them by is kept in the caches instead (132 us with ordinary loads).
typedef uint32_t cb_u32x4_t __attribute__((ext_vector_type(4)));
template <int DTYPE> struct EightOf;
template <> struct EightOf<0> {
    cb_u32x4_t a, b;
    __device__ __forceinline__ void load(const void *from) {
        typedef cb_u32x4_t Anywhere __attribute__((aligned(4)));
        a = __builtin_nontemporal_load(static_cast<const Anywhere *>(from));
        b = __builtin_nontemporal_load(static_cast<const Anywhere *>(from) + 1);
    }
    __device__ __forceinline__ float value(int i) const { return __uint_as_float(i < 4 ? a[i & 3] : b[i & 3]); }
};
template <> struct EightOf<1> {
    cb_u32x4_t a;
    __device__ __forceinline__ void load(const void *from) {
        typedef cb_u32x4_t Anywhere __attribute__((aligned(2)));
        a = __builtin_nontemporal_load(static_cast<const Anywhere *>(from));
    }
    __device__ __forceinline__ float value(int i) const { return __uint_as_float(i & 1 ? a[i / 2] & 0xFFFF0000u : a[i / 2] << 16); }
};

template <int DTYPE, bool OBF16>
__global__ __launch_bounds__(CB_THREADS) void k_combine(const void *Y, int64_t y_rows, int64_t ldy, const int32_t *positions,
                                                        const float *weights, int m, int k, int d, int chunks, void *out, int64_t ldo) {
    const uint32_t id = blockIdx.x * CB_THREADS + threadIdx.x;
    const int t = (int)(id / (uint32_t)chunks), c = (int)(id % (uint32_t)chunks) * 8;
    if (t >= m) return;
    constexpr int AT_ONCE = 8;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const int64_t s = (int64_t)t * k;
    if (d - c >= 8) {                                       // c + 8 need not fit
        for (int j0 = 0; j0 < k; j0 += AT_ONCE) {
            int at[AT_ONCE];
            float w[AT_ONCE];
            EightOf<DTYPE> y[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                const bool is = j0 + j < k;
                at[j] = is ? positions[s + j0 + j] : -1;
                w[j] = is ? weights[s + j0 + j] : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j)
                if (at[j] >= 0 && at[j] < y_rows)
                    y[j].load(static_cast<const char *>(Y) + ((int64_t)at[j] * ldy + c) * (DTYPE ? 2 : 4));
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j)
                if (at[j] >= 0 && at[j] < y_rows)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i] = fmaf(w[j], y[j].value(i), sum[i]);
        }
        const float lo[4] = {sum[0], sum[1], sum[2], sum[3]}, hi[4] = {sum[4], sum[5], sum[6], sum[7]};
        if (OBF16) {
            Unaligned<uint32_t, 4> four;
            for (int i = 0; i < 4; ++i) four.v[i] = bf16_rne_bits(sum[2 * i]) | bf16_rne_bits(sum[2 * i + 1]) << 16;
            *reinterpret_cast<Unaligned<uint16_t, 8> *>(reinterpret_cast<uint16_t *>(out) + t * ldo + c) = __builtin_bit_cast(Unaligned<uint16_t, 8>, four);
        } else {
            store_y4<false>(out, t * ldo + c, lo, 4);
            store_y4<false>(out, t * ldo + c + 4, hi, 4);
        }
        return;
    }
    for (int i = 0; c + i < d; ++i) {
        float one = 0.0f;
        for (int j = 0; j < k; ++j) {
            const int32_t at = positions[s + j];
            if (at >= 0 && at < y_rows) one = fmaf(weights[s + j], Elem<DTYPE>::load(Y, at * ldy + c + i), one);
        }
        store_y<OBF16>(out, t * ldo + c + i, one);
    }
}

template <int DTYPE, int PER> hipError_t launch_pick(const RouteProblem &q, int blocks) {
    const size_t lds = ((size_t)RT_WAVES + 1) * q.n_experts * 4;
    static MoreLds alone, together;
    const hipError_t e = blocks == 1 ? alone.ask(reinterpret_cast<const void *>(&k_route_pick<DTYPE, PER, true>), 80 * 1024)
                                     : together.ask(reinterpret_cast<const void *>(&k_route_pick<DTYPE, PER, false>), 80 * 1024);
    if (e != hipSuccess) return e;
    if (blocks == 1) k_route_pick<DTYPE, PER, true><<<1, RT_THREADS, lds, q.stream>>>(q);
    else k_route_pick<DTYPE, PER, false><<<blocks, RT_THREADS, lds, q.stream>>>(q);
    return hipGetLastError();
}
template <int DTYPE> hipError_t launch_pick(const RouteProblem &q, int blocks) {
    if (q.n_experts <= 16) return launch_pick<DTYPE, 1>(q, blocks);
    if (q.n_experts <= 64) return launch_pick<DTYPE, 4>(q, blocks);
    if (q.n_experts <= 128) return launch_pick<DTYPE, 8>(q, blocks);
    if (q.n_experts <= 256) return launch_pick<DTYPE, 16>(q, blocks);
    if (q.n_experts <= 512) return launch_pick<DTYPE, 32>(q, blocks);
    return launch_pick<DTYPE, 64>(q, blocks);
}

template <int DTYPE, bool OBF16>
hipError_t launch_combine_type(const void *Y, int64_t y_rows, int64_t ldy, const int32_t *positions, const float *weights, int m, int k, int d,
                               void *out, int64_t ldo, hipStream_t stream) {
    const int64_t chunks = ((int64_t)d + 7) / 8, blocks = (chunks * m + CB_THREADS - 1) / CB_THREADS;
    if (blocks * CB_THREADS > 0xFFFFFFFFll) return hipErrorNotSupported;
    k_combine<DTYPE, OBF16><<<dim3((uint32_t)blocks), CB_THREADS, 0, stream>>>(Y, y_rows, ldy, positions, weights, m, k, d, (int)chunks, out, ldo);
    return hipGetLastError();
}

}  // namespace

// Counts by workgroup and expert; a single workgroup keeps them.
size_t route_workspace_bytes(int m, int n_experts, int) {
    return m <= RT_TOKENS ? 0 : (size_t)((m + RT_TOKENS - 1) / RT_TOKENS) * counts_row(n_experts);
}

hipError_t launch_route(const RouteProblem &q) {
    const int blocks = q.m <= RT_TOKENS ? 1 : (q.m + RT_TOKENS - 1) / RT_TOKENS;
    const hipError_t e = q.dtype == 0 ? launch_pick<0>(q, blocks) : launch_pick<1>(q, blocks);
    if (e != hipSuccess || blocks == 1) return e;
    int lanes = WAVE;
    while (lanes * 4 < q.n_experts) lanes *= 2;
    k_route_order<<<blocks, RT_THREADS, 2 * (size_t)q.n_experts * 4, q.stream>>>(q, RT_TOKENS, blocks, lanes);
    return hipGetLastError();
}

hipError_t launch_combine(const void *Y, int dtype, int64_t y_rows, int64_t ldy, const int32_t *positions, const float *weights, int m,
                          int k, int d, void *out, int out_dtype, int64_t ldo, hipStream_t stream) {
    if (m == 0) return hipSuccess;
    if (dtype == 0)
        return out_dtype == 0 ? launch_combine_type<0, false>(Y, y_rows, ldy, positions, weights, m, k, d, out, ldo, stream)
                              : launch_combine_type<0, true>(Y, y_rows, ldy, positions, weights, m, k, d, out, ldo, stream);
    return out_dtype == 0 ? launch_combine_type<1, false>(Y, y_rows, ldy, positions, weights, m, k, d, out, ldo, stream)
                          : launch_combine_type<1, true>(Y, y_rows, ldy, positions, weights, m, k, d, out, ldo, stream);
}

}  // namespace qamw
