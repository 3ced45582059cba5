// Routed experts: the choice of experts, the order of the rows, and the way back.
#include "qamw_product.hpp"

namespace qamw {
namespace {

constexpr int RT_WAVES = 16, RT_THREADS = RT_WAVES * WAVE;

// ---- choice ---------------------------------------------------------------------------------------------------------------
//
// A wave has a token, a lane the experts lane, lane + 64, ...  A logit becomes an unsigned number that orders as it does, 0 for
// what is never chosen (-inf, NaN); the largest of the wave wins, of equals the lowest expert.
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
    for (int d = 32; d; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ uint32_t key_of(float f) {
    if (!(f > -__builtin_inff())) return 0;
    f += 0.0f;                                             // -0 is 0
    const uint32_t u = __float_as_uint(f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// Lane j < k gets the j-th choice: its expert (-1: none) and weight.
template <int DTYPE, int NPL>
__device__ __forceinline__ void pick(const void *logits, int64_t at, int n, int k, bool renormalise, int &expert, float &weight) {
    const int lane = threadIdx.x % WAVE;
    uint32_t key[NPL];
    for (int i = 0; i < NPL; ++i) {
        const int e = lane + i * WAVE;
        key[i] = e < n ? key_of(Elem<DTYPE>::load(logits, at + e)) : 0;
    }
    float total = 0.0f, top = 0.0f, mine = 0.0f;
    expert = -1;
    weight = 0.0f;
    for (int j = 0; j < k; ++j) {
        uint32_t best = 0;
        for (int i = 0; i < NPL; ++i) best = max(best, key[i]);
        best = wave_umax(best);
        if (best == 0) break;
        // the lowest expert that has it: its complement is the largest
        uint32_t who = 0;
        for (int i = 0; i < NPL; ++i)
            if (key[i] == best) who = max(who, ~(uint32_t)(lane + i * WAVE));
        who = ~wave_umax(who);
        const float v = value_of(best);
        if (j == 0) {
            top = v;
            if (!renormalise) {
                float sum = 0.0f;
                for (int i = 0; i < NPL; ++i)
                    if (key[i]) {
                        const float x = value_of(key[i]);
                        sum += x == top ? 1.0f : expf(x - top);
                    }
                total = wave_sum(sum);
            }
        }
        const float p = v == top ? 1.0f : expf(v - top);
        if (renormalise) total += p;
        if (lane == j) {
            expert = (int)who;
            mine = p;
        }
        for (int i = 0; i < NPL; ++i)
            if ((uint32_t)(lane + i * WAVE) == who) key[i] = 0;
    }
    if (expert >= 0) weight = mine / total;
}

// ---- order ----------------------------------------------------------------------------------------------------------------
//
// A stable counting sort of the slots (token after token, choice after choice).  Workgroup b has the tokens b * tokens .. and
// counts its slots by expert; what it writes as a slot's position is the slot's rank among those of its expert in the workgroup.
// The second launch knows all counts: what comes before an expert, and before the workgroup within the expert.
template <int DTYPE, int NPL>
__global__ __launch_bounds__(RT_THREADS) void k_route_pick(RouteProblem q, int tokens) {
    extern __shared__ int32_t rt_lds[];
    int32_t *chosen = rt_lds;                              // [tokens * k]
    uint32_t *counts = reinterpret_cast<uint32_t *>(rt_lds + tokens * q.k);   // [n_experts]
    const int t0 = blockIdx.x * tokens, nt = min(tokens, q.m - t0), n = q.n_experts, k = q.k;
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    for (int e = threadIdx.x; e < n; e += RT_THREADS) counts[e] = 0;
    for (int t = wave; t < nt; t += RT_WAVES) {
        int expert;
        float weight;
        pick<DTYPE, NPL>(q.logits, (int64_t)(t0 + t) * q.ld, n, k, q.renormalise, expert, weight);
        if (lane < k) {
            const int64_t at = (int64_t)(t0 + t) * k + lane;
            q.experts[at] = expert;
            q.weights[at] = weight;
            chosen[t * k + lane] = expert;
        }
    }
    __syncthreads();
    // one wave goes through the slots in order: 64 at a time, equal ones found by the bits of the expert
    if (wave == 0) {
        for (int s0 = 0; s0 < nt * k; s0 += WAVE) {
            const int s = s0 + lane;
            const int e = s < nt * k ? chosen[s] : -1;
            unsigned long long same = __ballot(e >= 0);
            for (int b = 0; b < 10; ++b) {
                const unsigned long long has = __ballot((e >> b) & 1);
                same &= (e >> b) & 1 ? has : ~has;
            }
            int rank = 0;
            if (e >= 0) {
                rank = (int)counts[e] + __popcll(same & ((1ull << lane) - 1));
            }
            __builtin_amdgcn_wave_barrier();
            if (e >= 0) {
                if ((same >> lane) == 1) counts[e] = (uint32_t)rank + 1;     // the last one of its expert
                q.positions[(int64_t)t0 * k + s] = rank;
            } else if (s < nt * k) {
                q.positions[(int64_t)t0 * k + s] = -1;
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < n; e += RT_THREADS) q.counts[(int64_t)blockIdx.x * n + e] = counts[e];
}

__global__ __launch_bounds__(RT_THREADS) void k_route_order(RouteProblem q, int tokens, int blocks) {
    extern __shared__ int32_t rt_lds[];
    uint32_t *base = reinterpret_cast<uint32_t *>(rt_lds);   // [n_experts]: where this workgroup's rows of an expert begin
    uint32_t *total = base + q.n_experts;                    // [n_experts + 1]
    const int n = q.n_experts, k = q.k;
    for (int e = threadIdx.x; e < n; e += RT_THREADS) {
        uint32_t before = 0, all = 0;
        for (int b = 0; b < blocks; ++b) {
            const uint32_t c = q.counts[(int64_t)b * n + e];
            all += c;
            if (b < (int)blockIdx.x) before += c;
        }
        base[e] = before;
        total[e] = all;
    }
    __syncthreads();
    if (threadIdx.x < WAVE) {                                // exclusive sums over the experts
        uint32_t before = 0;
        for (int e0 = 0; e0 < n; e0 += WAVE) {
            const int e = e0 + threadIdx.x;
            const uint32_t c = e < n ? total[e] : 0;
            uint32_t upto = c;
            for (int d = 1; d < WAVE; d <<= 1) {
                const uint32_t v = (uint32_t)__shfl_up((int)upto, d);
                if ((int)threadIdx.x >= d) upto += v;
            }
            if (e < n) {
                base[e] += before + upto - c;
                if (blockIdx.x == 0) q.offsets[e] = (int32_t)(before + upto - c);
            }
            before += (uint32_t)__shfl((int)upto, WAVE - 1);
        }
        if (threadIdx.x == 0) {
            total[n] = before;
            if (blockIdx.x == 0) q.offsets[n] = (int32_t)before;
        }
    }
    __syncthreads();
    const int64_t slots = (int64_t)q.m * k, s0 = (int64_t)blockIdx.x * tokens * k, s1 = min(s0 + (int64_t)tokens * k, slots);
    for (int64_t s = s0 + threadIdx.x; s < s1; s += RT_THREADS) {
        const int e = q.experts[s];
        if (e >= 0) {
            const int64_t place = (int64_t)base[e] + q.positions[s];
            q.positions[s] = (int32_t)place;
            q.rows[place] = (int32_t)(s / k);
        }
    }
    // places that no slot has
    for (int64_t p = (int64_t)total[n] + (int64_t)blockIdx.x * RT_THREADS + threadIdx.x; p < slots; p += (int64_t)blocks * RT_THREADS)
        q.rows[p] = -1;
}

// ---- the way back ---------------------------------------------------------------------------------------------------------

constexpr int CB_THREADS = 256;

template <int DTYPE, bool OBF16>
__global__ __launch_bounds__(CB_THREADS) void k_combine_any(const void *Y, int64_t y_rows, int64_t ldy, const int32_t *positions,
                                                            const float *weights, int k, int d, void *out, int64_t ldo) {
    const int64_t t = blockIdx.x;
    for (int c = threadIdx.x; c < d; c += CB_THREADS) {
        float sum = 0.0f;
        for (int j = 0; j < k; ++j) {
            const int32_t at = positions[t * k + j];
            if (at >= 0 && at < y_rows) sum = fmaf(weights[t * k + j], Elem<DTYPE>::load(Y, at * ldy + c), sum);
        }
        if (OBF16)
            reinterpret_cast<uint16_t *>(out)[t * ldo + c] = (uint16_t)bf16_rne_bits(sum);
        else
            reinterpret_cast<float *>(out)[t * ldo + c] = sum;
    }
}

// Tokens of a workgroup of the first launch.
int route_tokens(int m, int k) {
    (void)m;
    return k <= 8 ? 64 : 16;
}

template <int DTYPE> hipError_t launch_pick(const RouteProblem &q, int tokens, int blocks) {
    const size_t lds = ((size_t)tokens * q.k + q.n_experts) * 4;
    const int npl = (q.n_experts + WAVE - 1) / WAVE;
    if (npl <= 1) k_route_pick<DTYPE, 1><<<blocks, RT_THREADS, lds, q.stream>>>(q, tokens);
    else if (npl <= 2) k_route_pick<DTYPE, 2><<<blocks, RT_THREADS, lds, q.stream>>>(q, tokens);
    else if (npl <= 4) k_route_pick<DTYPE, 4><<<blocks, RT_THREADS, lds, q.stream>>>(q, tokens);
    else if (npl <= 8) k_route_pick<DTYPE, 8><<<blocks, RT_THREADS, lds, q.stream>>>(q, tokens);
    else k_route_pick<DTYPE, 16><<<blocks, RT_THREADS, lds, q.stream>>>(q, tokens);
    return hipGetLastError();
}

}  // namespace

size_t route_workspace_bytes(int m, int n_experts, int k) {
    const int tokens = route_tokens(m, k);
    return (size_t)((m + tokens - 1) / tokens) * n_experts * 4;
}

hipError_t launch_route(const RouteProblem &q) {
    const int tokens = route_tokens(q.m, q.k), blocks = q.m ? (q.m + tokens - 1) / tokens : 1;
    if (q.m) {
        const hipError_t e = q.dtype == 0 ? launch_pick<0>(q, tokens, blocks) : launch_pick<1>(q, tokens, blocks);
        if (e != hipSuccess) return e;
    }
    k_route_order<<<blocks, RT_THREADS, (2 * (size_t)q.n_experts + 1) * 4, q.stream>>>(q, tokens, q.m ? blocks : 0);
    return hipGetLastError();
}

hipError_t launch_combine(const void *Y, int dtype, int64_t y_rows, int64_t ldy, const int32_t *positions, const float *weights, int m,
                          int k, int d, void *out, int out_dtype, int64_t ldo, hipStream_t stream) {
    if (m == 0) return hipSuccess;
    const dim3 g((uint32_t)m);
    if (dtype == 0) {
        if (out_dtype == 0) k_combine_any<0, false><<<g, CB_THREADS, 0, stream>>>(Y, y_rows, ldy, positions, weights, k, d, out, ldo);
        else k_combine_any<0, true><<<g, CB_THREADS, 0, stream>>>(Y, y_rows, ldy, positions, weights, k, d, out, ldo);
    } else {
        if (out_dtype == 0) k_combine_any<1, false><<<g, CB_THREADS, 0, stream>>>(Y, y_rows, ldy, positions, weights, k, d, out, ldo);
        else k_combine_any<1, true><<<g, CB_THREADS, 0, stream>>>(Y, y_rows, ldy, positions, weights, k, d, out, ldo);
    }
    return hipGetLastError();
}

}  // namespace qamw
