// The rules that a request's logits go through before a token is taken from them: penalties for tokens that were there already,
// biases, and the tokens that a grammar allows.  For row r of sequence b and token v, with n = how often v stands in what the
// request has written and on the row's path through its block or tree, and "seen" = n > 0 or v stands in the prompt:
//   x = seen ? (x > 0 ? x / repetition : x * repetition) : x
//   x = x - frequency * n - (n > 0 ? presence : 0) + bias;     -inf where the row's mask does not allow v
//
// A workgroup owns a stretch of the vocabulary for some rows of one sequence, so that every logit has one owner, nothing is
// counted twice and no memory has to be cleared before the call:
//   - the stretch of every row is streamed to the output with the mask applied (in place: what the mask takes is struck out);
//   - the history is read once and counted into the stretch's counters in LDS, the few tokens that it touches are listed;
//   - those of every row are computed from the row's logits and written over what was streamed.
#include "orthrus_attn_dev.h"

namespace orthrus {

constexpr int kStretch = 8192;      // tokens of a workgroup
constexpr int kRulesThreads = 512;
constexpr uint32_t kInPrompt = 0x80000000u;

// 16 bytes of logits at the alignment of one
typedef __attribute__((ext_vector_type(4), aligned(4))) uint32_t vec_of_4;
typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t vec_of_8;
template <int DTYPE> struct Value;
template <> struct Value<0> { using T = uint32_t; using Vec = vec_of_4; static constexpr uint32_t kLow = 0xff800000u; };  // -inf
template <> struct Value<1> { using T = uint16_t; using Vec = vec_of_8; static constexpr uint32_t kLow = 0xff80ff80u; };
template <> struct Value<2> { using T = uint16_t; using Vec = vec_of_8; static constexpr uint32_t kLow = 0xfc00fc00u; };

template <int DTYPE>
__device__ __forceinline__ float value_of(uint32_t bits)
{
    if constexpr (DTYPE == 0) return __uint_as_float(bits);
    else if constexpr (DTYPE == 1) return __uint_as_float(bits << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}
template <int DTYPE>
__device__ __forceinline__ typename Value<DTYPE>::T bits_of(float x)
{
    if constexpr (DTYPE == 0) return __float_as_uint(x);
    else if constexpr (DTYPE == 1) return __builtin_bit_cast(uint16_t, (__bf16)x);
    else return __builtin_bit_cast(uint16_t, (_Float16)x);
}

struct Penalty {
    float rep, pres, freq;
    __device__ __forceinline__ Penalty(const RulesArgs &a, int b)
    {
        rep = a.repetition ? a.repetition[b] : 1.f;
        pres = a.presence ? a.presence[b] : 0.f;
        freq = a.frequency ? a.frequency[b] : 0.f;
        if (!(rep > 0.f) || rep == INFINITY) rep = 1.f;
        if (!(fabsf(pres) < INFINITY)) pres = 0.f;
        if (!(fabsf(freq) < INFINITY)) freq = 0.f;
    }
    __device__ __forceinline__ bool any() const { return rep != 1.f || pres != 0.f || freq != 0.f; }
    // 32 bits throughout, each step rounded once; the count is whole up to 2^24
    __device__ __forceinline__ float operator()(float x, uint32_t n, bool prompt) const
    {
        if (n > 0 || prompt) x = x > 0.f ? x / rep : x * rep;
        if (n > 0) x = __builtin_fmaf(-freq, (float)n, x) - pres;
        return x;
    }
};

// Whether row `row` of the masks allows token v.
__device__ __forceinline__ bool allowed(const uint32_t *mask, int v) { return mask[v >> 5] >> (v & 31) & 1u; }

template <int DTYPE>
__global__ void __launch_bounds__(kRulesThreads) logits_rules_kernel(const RulesArgs a)
{
    using T = typename Value<DTYPE>::T;
    constexpr int VEC = 16 / sizeof(T);
    using vec_t = typename Value<DTYPE>::Vec;
    extern __shared__ uint32_t smem[];
    uint32_t *counts = smem;                                     // [kStretch]
    uint32_t *biases = smem + kStretch;                          // [kStretch], only with biases: 1 + the entry's place in the list
    __shared__ uint16_t s_list[kStretch];
    __shared__ int s_listed;
    __shared__ int s_token[kMaxNodes];
    __shared__ unsigned long long s_path[kMaxNodes];             // the nodes on a row's path whose token lies in the stretch

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int stretches = (a.vocab + kStretch - 1) / kStretch, groups = (a.rows + a.rows_per_wg - 1) / a.rows_per_wg;
    const int stretch = (int)(blockIdx.x % (unsigned)stretches), group = (int)(blockIdx.x / (unsigned)stretches % (unsigned)groups);
    const int b = (int)(blockIdx.x / ((unsigned)stretches * (unsigned)groups));
    const int v0 = stretch * kStretch, v1 = min(a.vocab, v0 + kStretch);
    const int r0 = group * a.rows_per_wg, r1 = min(a.rows, r0 + a.rows_per_wg);
    const T *in = (const T *)a.logits + (int64_t)b * a.rows * a.stride_row;
    T *out = (T *)a.out + (int64_t)b * a.rows * a.out_stride_row;
    auto mask_of = [&](int r) __attribute__((always_inline)) -> const uint32_t * {
        if (!a.mask_rows) return nullptr;
        const int m = a.mask_rows[(int64_t)b * a.rows + r];
        return m < 0 || m >= a.num_masks ? nullptr : a.masks + (int64_t)m * a.mask_stride;
    };

    const Penalty penalty(a, b);
    const bool penalise = penalty.any();
    int64_t bias0 = 0, bias1 = 0;
    if (a.bias_starts) {
        bias0 = max((int64_t)a.bias_starts[b], (int64_t)0);
        bias1 = min((int64_t)a.bias_starts[b + 1], a.num_biases);
    }
    const bool biased = bias0 < bias1;

    // ---- the stretch of every row, with its mask
    constexpr int UNIT = 64 * VEC;
    const int units = (v1 - v0 + UNIT - 1) / UNIT;
    for (int x = wave; x < units * (r1 - r0); x += kRulesThreads / 64) {
        const int r = r0 + x / units, v = v0 + x % units * UNIT + lane * VEC;
        const uint32_t *mask = mask_of(r);
        if (a.in_place && !mask) continue;
        if (v >= v1) continue;
        const T *src = in + (int64_t)r * a.stride_row + v;
        T *dst = out + (int64_t)r * a.out_stride_row + v;
        constexpr uint32_t kAll = (1u << VEC) - 1u;
        const uint32_t bits = mask ? mask[v >> 5] >> (v & 31) & kAll : kAll;
        if (v + VEC <= v1) {
            if (a.in_place && bits == kAll) continue;
            vec_t y = {Value<DTYPE>::kLow, Value<DTYPE>::kLow, Value<DTYPE>::kLow, Value<DTYPE>::kLow};
            if (bits) {
                y = *(const vec_t *)src;
                if (bits != kAll) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        if constexpr (sizeof(T) == 4) {
                            y[e & 3] = bits >> e & 1u ? y[e & 3] : Value<DTYPE>::kLow;
                        } else {
                            const uint32_t keep = 0xffffu << 16 * (e & 1);
                            y[e / 2 & 3] = bits >> e & 1u ? y[e / 2 & 3] : (y[e / 2 & 3] & ~keep) | (Value<DTYPE>::kLow & keep);
                        }
                    }
                }
            }
            *(vec_t *)dst = y;
        } else {
            for (int e = 0; v + e < v1; ++e) {
                if (!(bits >> e & 1u)) dst[e] = (T)Value<DTYPE>::kLow;
                else if (!a.in_place) dst[e] = src[e];
            }
        }
    }
    if (!penalise && !biased) return;

    // ---- counters, biases and paths
    for (int i = tid; i < kStretch / 4; i += kRulesThreads) {
        ((uint4 *)counts)[i] = make_uint4(0, 0, 0, 0);
        if (biased) ((uint4 *)biases)[i] = make_uint4(0, 0, 0, 0);
    }
    if (tid == 0) s_listed = 0;
    if (wave == 0) {
        int token = -1;
        unsigned long long path = 0;
        if (penalise && a.tokens) {
            if (lane < a.rows) token = a.tokens[(int64_t)b * a.rows + lane];
            if (token < v0 || token >= v1) token = -1;
            if (a.parents) {
                const uint2 on = tree_path(a.parents + (int64_t)b * a.rows, a.rows);
                path = (unsigned long long)on.y << 32 | on.x;
            } else {
                path = ~0ull >> (63 - lane);  // a chain
            }
            path &= __ballot(token >= 0);
        }
        s_token[lane] = token;
        s_path[lane] = path;
    }
    __syncthreads();
    if (penalise && a.history) {
        const int64_t n = min(max((int64_t)a.history_lens[b], (int64_t)0), a.history_stride);
        const int64_t n0 = a.prompt_lens ? min(max((int64_t)a.prompt_lens[b], (int64_t)0), n) : 0;
        const int32_t *text = a.history + (int64_t)b * a.history_stride;
        for (int64_t i = tid; i < n; i += kRulesThreads) {
            const uint32_t at = (uint32_t)text[i] - (uint32_t)v0;
            if (at < (uint32_t)(v1 - v0)) {
                if (i < n0) atomicOr(&counts[at], kInPrompt);
                else atomicAdd(&counts[at], 1u);
            }
        }
    }
    if (biased) {
        for (int64_t i = bias0 + tid; i < bias1; i += kRulesThreads) {
            const uint32_t at = (uint32_t)a.bias_tokens[i] - (uint32_t)v0;
            if (at < (uint32_t)(v1 - v0)) atomicMax(&biases[at], (uint32_t)(i - bias0 + 1));  // the last entry of a token counts
        }
    }
    __syncthreads();
    for (int i = tid; i < kStretch; i += kRulesThreads) {
        const bool touched = counts[i] || (biased && biases[i]);
        const unsigned long long hit = __ballot(touched);
        int base = 0;
        if (lane == 0 && hit) base = atomicAdd(&s_listed, __popcll(hit));
        base = __shfl(base, 0);
        if (touched) s_list[base + __popcll(hit & ((1ull << lane) - 1))] = (uint16_t)i;
    }
    __syncthreads();  // (the streamed logits have left as well)

    // ---- the touched tokens of every row
    const int listed = s_listed;
    for (int x = tid; x < listed * (r1 - r0); x += kRulesThreads) {
        const int r = r0 + x / listed, at = s_list[x % listed], v = v0 + at;
        const uint32_t *mask = mask_of(r);
        if (mask && !allowed(mask, v)) continue;
        const uint32_t word = counts[at];
        uint32_t n = word & ~kInPrompt;
        for (unsigned long long p = s_path[r]; p; p &= p - 1) n += s_token[__builtin_ctzll(p)] == v ? 1u : 0u;
        float y = penalty(value_of<DTYPE>(in[(int64_t)r * a.stride_row + v]), n, word >> 31);
        if (biased && biases[at]) y += a.bias_values[bias0 + biases[at] - 1];
        out[(int64_t)r * a.out_stride_row + v] = bits_of<DTYPE>(y);
    }
    // those that stand on the row's path only
    for (int x = tid; x < (r1 - r0) * 64; x += kRulesThreads) {
        const int r = r0 + (x >> 6), i = x & 63;
        const unsigned long long path = s_path[r];
        if (!(path >> i & 1)) continue;
        const int v = s_token[i], at = v - v0;
        if (counts[at] || (biased && biases[at])) continue;
        uint32_t n = 0;
        bool first = true;
        for (unsigned long long p = path; p; p &= p - 1) {
            const int j = __builtin_ctzll(p);
            if (s_token[j] == v) {
                ++n;
                first = first && j >= i;
            }
        }
        const uint32_t *mask = mask_of(r);
        if (!first || (mask && !allowed(mask, v))) continue;
        out[(int64_t)r * a.out_stride_row + v] = bits_of<DTYPE>(penalty(value_of<DTYPE>(in[(int64_t)r * a.stride_row + v]), n, false));
    }
}

hipError_t launch_logits_process(RulesArgs a, int num_cus, hipStream_t stream)
{
    if (a.batch == 0) return hipSuccess;
    const int stretches = (a.vocab + kStretch - 1) / kStretch;
    a.rows_per_wg = a.rows;
    while (a.rows_per_wg > 1 && (int64_t)a.batch * stretches * ((a.rows + a.rows_per_wg - 1) / a.rows_per_wg) < 4ll * num_cus)
        a.rows_per_wg = (a.rows_per_wg + 1) / 2;
    const unsigned groups = (unsigned)((a.rows + a.rows_per_wg - 1) / a.rows_per_wg);
    const dim3 grid((unsigned)a.batch * (unsigned)stretches * groups);
    const size_t lds = kStretch * sizeof(uint32_t) * (a.bias_starts ? 2 : 1);
    auto kern = a.dtype == 0 ? logits_rules_kernel<0> : a.dtype == 1 ? logits_rules_kernel<1> : logits_rules_kernel<2>;
    hipLaunchKernelGGL(kern, grid, dim3(kRulesThreads), lds, stream, a);
    return hipGetLastError();
}

}  // namespace orthrus
