// The rules that a request's logits go through before a token is taken from them: penalties for tokens that were there already,
// biases, and the tokens that a grammar allows.  For row r of sequence b and token v, with n = how often v stands in what the
// request has written and on the row's path through its block or tree, and "seen" = n > 0 or v stands in the prompt:
//   x = seen ? (x > 0 ? x / repetition : x * repetition) : x
//   x = x - frequency * n - (n > 0 ? presence : 0) + bias;     -inf where the row's mask does not allow v
//
// A workgroup owns a stretch of the vocabulary for some rows of one sequence.  It counts the history into the stretch's counters
// in LDS once, marks the tokens that a penalty or bias touches in a bit map, and then streams the stretch of each of its rows: one
// read and one write a logit (in place: only of what changes; of what a mask takes, the write), with the few touched ones worked
// out on the way.  Every logit has one owner, nothing is counted twice, and no memory has to be cleared before the call.
#include "orthrus_attn_dev.h"

namespace orthrus {

constexpr int kStretch = 8192;      // tokens of a workgroup
constexpr int kRulesThreads = 512;
constexpr int kRulesWaves = kRulesThreads / 64;
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
// Element e of 16 bytes, and another value in its place (e differs from lane to lane).
template <int DTYPE>
__device__ __forceinline__ uint32_t element(const u32x4 &y, int e)
{
    const int d = DTYPE == 0 ? e : e >> 1;
    const uint32_t lo = d & 1 ? y[1] : y[0], hi = d & 1 ? y[3] : y[2], w = d & 2 ? hi : lo;
    return DTYPE == 0 ? w : (w >> 16 * (e & 1)) & 0xffffu;
}
template <int DTYPE>
__device__ __forceinline__ void replace(u32x4 &y, int e, uint32_t bits)
{
    const int d = DTYPE == 0 ? e : e >> 1, shift = DTYPE == 0 ? 0 : 16 * (e & 1);
    const uint32_t keep = DTYPE == 0 ? 0u : ~(0xffffu << shift), put = bits << shift;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = d == i ? (y[i] & keep) | put : y[i];
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

// TOUCH: there may be penalties or biases (else masks alone: no LDS).  IN_PLACE: out is logits.
template <int DTYPE, bool TOUCH, bool IN_PLACE>
__global__ void __launch_bounds__(kRulesThreads) logits_rules_kernel(const RulesArgs a)
{
    using T = typename Value<DTYPE>::T;
    using vec_t = typename Value<DTYPE>::Vec;
    constexpr int VEC = 16 / sizeof(T);
    constexpr int U = kStretch / (kRulesThreads * VEC);  // 16-byte pieces of a lane's share: a wave's of a stretch, once through it
    static_assert(U == 4 || U == 2, "");
    constexpr uint32_t kAll = (1u << VEC) - 1u;
    extern __shared__ uint32_t smem[];                   // TOUCH:
    uint32_t *counts = smem;                             // [kStretch] times written, kInPrompt
    uint32_t *touched = smem + kStretch;                 // [kStretch / 32] bits: a counter or a bias is set
    int *s_token = (int *)(touched + kStretch / 32);     // [kMaxNodes]
    unsigned long long *s_path = (unsigned long long *)(s_token + kMaxNodes);  // [kMaxNodes] nodes on a row's path whose token lies in the stretch
    uint32_t *biases = (uint32_t *)(s_path + kMaxNodes); // [kStretch], with biases only: 1 + the entry's place in the list

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int stretches = (a.vocab + kStretch - 1) / kStretch, groups = (a.rows + a.rows_per_wg - 1) / a.rows_per_wg;
    const int stretch = (int)(blockIdx.x % (unsigned)stretches), group = (int)(blockIdx.x / (unsigned)stretches % (unsigned)groups);
    const int b = (int)(blockIdx.x / ((unsigned)stretches * (unsigned)groups));
    const int v0 = stretch * kStretch, v1 = min(a.vocab, v0 + kStretch);
    const int r0 = group * a.rows_per_wg, r1 = min(a.rows, r0 + a.rows_per_wg);
    const T *in = (const T *)a.logits + (int64_t)b * a.rows * a.stride_row;
    T *out = (T *)a.out + (int64_t)b * a.rows * a.out_stride_row;
    // wave w streams tokens first .. first + U * 64 * VEC - 1 of every row, piece u of a lane at `at(u)`
    const int first = v0 + wave * (U * 64 * VEC);
    auto at = [&](int u) __attribute__((always_inline)) { return first + (u * 64 + lane) * VEC; };

    // What the mask of row r allows of the lane's pieces, VEC bits each.
    struct Allowed {
        uint32_t bits[U];
        bool all;  // there is no mask
    };
    auto allowed_of = [&](int r) __attribute__((always_inline)) {
        Allowed x;
        x.all = true;
#pragma unroll
        for (int u = 0; u < U; ++u) x.bits[u] = kAll;
        if (a.mask_rows) {
            const int m = __builtin_amdgcn_readfirstlane(a.mask_rows[(int64_t)b * a.rows + r]);
            if (m >= 0 && m < a.num_masks) {
                x.all = false;
                const uint32_t *mask = a.masks + (int64_t)m * a.mask_stride;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int v = at(u);
                    x.bits[u] = v < v1 ? mask[v >> 5] : 0u;
                }
#pragma unroll
                for (int u = 0; u < U; ++u) x.bits[u] = x.bits[u] >> (at(u) & 31) & kAll;
            }
        }
        return x;
    };
    struct Piece {
        u32x4 y[U];
    };
    // the pieces of row r that `need` asks for; -inf in the place of the others
    auto load = [&](int r, auto need) __attribute__((always_inline)) {
        const T *row = in + (int64_t)r * a.stride_row;
        Piece p;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int v = at(u);
            p.y[u] = u32x4{Value<DTYPE>::kLow, Value<DTYPE>::kLow, Value<DTYPE>::kLow, Value<DTYPE>::kLow};
            if (v + VEC <= v1) {
                if (need(u)) p.y[u] = *(const vec_t *)(row + v);
            } else if (v < v1) {
                for (int e = 0; v + e < v1; ++e) replace<DTYPE>(p.y[u], e, row[v + e]);
            }
        }
        return p;
    };

    // Not in place every row is read: the first one's logits are on their way while the history is counted.
    Allowed ok = allowed_of(r0);
    Piece piece;
    if constexpr (!IN_PLACE) piece = load(r0, [&](int u) { return ok.bits[u] != 0; });

    const Penalty penalty(a, b);
    const bool penalise = TOUCH && penalty.any();
    int64_t bias0 = 0, bias1 = 0;
    if (TOUCH && a.bias_starts) {
        bias0 = max((int64_t)a.bias_starts[b], (int64_t)0);
        bias1 = min((int64_t)a.bias_starts[b + 1], a.num_biases);
    }
    const bool biased = bias0 < bias1;

    if (TOUCH && (penalise || biased)) {
        for (int i = tid; i < kStretch / 4; i += kRulesThreads) {
            ((uint4 *)counts)[i] = make_uint4(0, 0, 0, 0);
            if (biased) ((uint4 *)biases)[i] = make_uint4(0, 0, 0, 0);
        }
        if (tid < kStretch / 32) touched[tid] = 0;
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
            constexpr int RUN = 8;  // loads in flight
            for (int64_t i0 = tid; i0 < n; i0 += RUN * kRulesThreads) {
                int t[RUN];
#pragma unroll
                for (int k = 0; k < RUN; ++k) t[k] = i0 + k * kRulesThreads < n ? text[i0 + k * kRulesThreads] : -1;
#pragma unroll
                for (int k = 0; k < RUN; ++k) {
                    const uint32_t x = (uint32_t)t[k] - (uint32_t)v0;
                    if (t[k] >= 0 && x < (uint32_t)(v1 - v0)) {
                        if (i0 + k * kRulesThreads < n0) atomicOr(&counts[x], kInPrompt);
                        else atomicAdd(&counts[x], 1u);
                        atomicOr(&touched[x >> 5], 1u << (x & 31));
                    }
                }
            }
        }
        if (biased) {
            for (int64_t i = bias0 + tid; i < bias1; i += kRulesThreads) {
                const uint32_t x = (uint32_t)a.bias_tokens[i] - (uint32_t)v0;
                if (x < (uint32_t)(v1 - v0)) {
                    atomicMax(&biases[x], (uint32_t)(i - bias0 + 1));  // the last entry of a token counts
                    atomicOr(&touched[x >> 5], 1u << (x & 31));
                }
            }
        }
        __syncthreads();
    }

    for (int r = r0; r < r1; ++r) {
        // ---- which of the lane's logits a penalty or a bias touches
        uint32_t hit[U];
#pragma unroll
        for (int u = 0; u < U; ++u) hit[u] = 0;
        unsigned long long path = 0;
        if (TOUCH && (penalise || biased)) {
            path = s_path[r];
            path = (unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((int)(path >> 32)) << 32 |
                   (uint32_t)__builtin_amdgcn_readfirstlane((int)path);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = at(u) - v0;
                hit[u] = touched[x >> 5] >> (x & 31) & kAll;
            }
            for (unsigned long long p = path; p; p &= p - 1) {
                const int t = s_token[__builtin_ctzll(p)];
#pragma unroll
                for (int u = 0; u < U; ++u) hit[u] |= (uint32_t)(t - at(u)) < (uint32_t)VEC ? 1u << ((t - at(u)) & 31) : 0u;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) hit[u] &= ok.bits[u];
        }
        if constexpr (IN_PLACE) {
            // what changes only: the pieces with a touched logit, and those that keep a part
            piece = load(r, [&](int u) { return hit[u] != 0 || (ok.bits[u] != 0 && ok.bits[u] != kAll); });
        }
        // the next row's are on their way while this one's are worked out
        Piece next_piece;
        Allowed next_ok;
        if (r + 1 < r1) {
            next_ok = allowed_of(r + 1);
            if constexpr (!IN_PLACE) next_piece = load(r + 1, [&](int u) { return next_ok.bits[u] != 0; });
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int v = at(u);
            u32x4 y = piece.y[u];
            if (TOUCH) {
                uint32_t left = hit[u];
                while (__any(left != 0)) {
                    if (left) {
                        const int e = __builtin_ctz(left), x = v + e - v0;
                        left &= left - 1;
                        const uint32_t word = counts[x];
                        uint32_t n = word & ~kInPrompt;
                        for (unsigned long long p = path; p; p &= p - 1) n += s_token[__builtin_ctzll(p)] == v + e ? 1u : 0u;
                        float z = value_of<DTYPE>(element<DTYPE>(y, e));
                        if (penalise) z = penalty(z, n, word >> 31);
                        if (biased && biases[x]) z += a.bias_values[bias0 + biases[x] - 1];
                        replace<DTYPE>(y, e, bits_of<DTYPE>(z));
                    }
                }
            }
            if (!ok.all) {
                const uint32_t bits = ok.bits[u];
                if (bits != kAll) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (DTYPE == 0) {
                            y[i] = bits >> i & 1u ? y[i] : Value<DTYPE>::kLow;
                        } else {
                            const uint32_t keep = (bits >> 2 * i & 1u ? 0xffffu : 0u) | (bits >> 2 * i & 2u ? 0xffff0000u : 0u);
                            y[i] = (y[i] & keep) | (Value<DTYPE>::kLow & ~keep);
                        }
                    }
                }
            }
            if (v < v1 && (!IN_PLACE || hit[u] || ok.bits[u] != kAll)) {
                T *dst = out + (int64_t)r * a.out_stride_row + v;
                if (v + VEC <= v1) *(vec_t *)dst = y;
                else
                    for (int e = 0; v + e < v1; ++e) dst[e] = (T)element<DTYPE>(y, e);
            }
        }
        if (r + 1 < r1) {
            ok = next_ok;
            if constexpr (!IN_PLACE) piece = next_piece;
        }
    }
}

template <int DTYPE>
static auto rules_kernel(bool touch, bool in_place)
{
    if (touch) return in_place ? logits_rules_kernel<DTYPE, true, true> : logits_rules_kernel<DTYPE, true, false>;
    return in_place ? logits_rules_kernel<DTYPE, false, true> : logits_rules_kernel<DTYPE, false, false>;
}

hipError_t launch_logits_process(RulesArgs a, int num_cus, hipStream_t stream)
{
    if (a.batch == 0) return hipSuccess;
    const bool touch = a.repetition || a.presence || a.frequency || a.bias_starts;
    const int stretches = (a.vocab + kStretch - 1) / kStretch;
    a.rows_per_wg = a.rows;
    while (a.rows_per_wg > 1 && (int64_t)a.batch * stretches * ((a.rows + a.rows_per_wg - 1) / a.rows_per_wg) < 4ll * num_cus)
        a.rows_per_wg = (a.rows_per_wg + 1) / 2;
    const unsigned groups = (unsigned)((a.rows + a.rows_per_wg - 1) / a.rows_per_wg);
    const dim3 grid((unsigned)a.batch * (unsigned)stretches * groups);
    size_t lds = 0;
    if (touch) lds = kStretch * 4 + kStretch / 8 + kMaxNodes * 12 + (a.bias_starts ? kStretch * 4 : 0);
    auto kern = a.dtype == 0 ? rules_kernel<0>(touch, a.in_place) : a.dtype == 1 ? rules_kernel<1>(touch, a.in_place) : rules_kernel<2>(touch, a.in_place);
    hipLaunchKernelGGL(kern, grid, dim3(kRulesThreads), lds, stream, a);
    return hipGetLastError();
}

}  // namespace orthrus
