// The rules that a request's logits go through before a token is taken from them: penalties for tokens that were there already,
// biases, and the tokens that a grammar allows.  For row r of sequence b and token v, with n = how often v stands in what the
// request has written and on the row's path through its block or tree, and "seen" = n > 0 or v stands in the prompt:
//   x = seen ? (x > 0 ? x / repetition : x * repetition) : x
//   x = x - frequency * n - (n > 0 ? presence : 0) + bias;     -inf where the row's mask does not allow v
//
// A workgroup owns a stretch of the vocabulary for some rows of one sequence.  It counts the history into the stretch's counters
// in LDS once, looks which of its tokens a penalty or bias touches, and then streams the stretch of each of its rows: one
// read and one write a logit (in place: only of what changes; of what a mask takes, the write), with the few touched ones worked
// out on the way.  Every logit has one owner, nothing is counted twice, and no memory has to be cleared before the call.
//
// What bounds it.  1024 rows of 151936 in fp32 with every rule: 222 us, where streaming them alone takes 198 (the touched ones are 11);
// 256 rows of 151669 in bf16, histories of 50..8000 (4000 on average): 46 us, of which the stream 29, filling and clearing the counters
// with their two barriers 6, the history, which each of 19 stretches reads, 2.5 per thousand tokens.  Tried: 16384 tokens a workgroup 50
// and 375 us (two workgroups to a CU), with 1024 threads 46 and 240, with half a word a token, so that there are four again, 55 (spills);
// 256 threads 49 and 283; 4096 tokens and 256 threads 48 and 270; the touched logits listed and written over the stream by gathers and
// stores of their own 58 and 334; a bit map of the touched tokens and jumps around what is of another stretch 47 and 250; whole
// sequences to an XCD, so that one L2 sees a history, 45.8 and 226 but one sequence of 64 rows 25 -> 119.
// The 256 rows with texts of one length, the same logits over and over: of 500 tokens 32 us, 4000 38, 16000 53, 30000 69.  In place, where
// what is read hangs on the counters, 40 -> 46, but the 1024 rows 221 -> 186: what no rule touches is not moved.
#include "orthrus_attn_dev.h"

namespace orthrus {

constexpr int kStretch = 8192;     // tokens of a workgroup
constexpr int kRulesThreads = 512;

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
    float rep, inv, pres, freq;
    __device__ __forceinline__ Penalty(float r, float p, float f) : rep(r), pres(p), freq(f)
    {
        if (!(rep > 0.f) || rep == INFINITY) rep = 1.f;
        inv = 1.f / rep;
        if (!(fabsf(pres) < INFINITY)) pres = 0.f;
        if (!(fabsf(freq) < INFINITY)) freq = 0.f;
    }
    __device__ __forceinline__ bool any() const { return rep != 1.f || pres != 0.f || freq != 0.f; }
    // Of a token that was seen.  32 bits throughout, each step rounded once; the count is whole up to 2^24.  The quotient from the
    // correctly rounded reciprocal: x * inv is at most a step off, what it leaves of x is exact in one multiply-add, and adding that
    // remainder's share rounds as the division does (Markstein, 1990); three instructions for ten.  Where the remainder is none
    // (infinities, NaN, a reciprocal or quotient out of range) the division itself.
    __device__ __forceinline__ float operator()(float x, uint32_t n) const
    {
        const float q = x * inv, rest = __builtin_fmaf(-q, rep, x);
        float d = __builtin_fmaf(rest, inv, q);
        const bool plain = fabsf(q) > 1e-30f && fabsf(q) < 1e30f && fabsf(x) > 1e-30f;
        if (__builtin_expect(!plain, 0)) d = x / rep;
        x = x > 0.f ? d : x * rep;
        const float y = __builtin_fmaf(-freq, (float)n, x) - pres;
        return n > 0 ? y : x;
    }
};

// The mask of a row, NULL: it has none, and what that allows of N pieces of VEC logits, VEC bits each.
template <int VEC, int N, class At>
__device__ __forceinline__ const uint32_t *allowed_of(const RulesArgs &a, int64_t row, int end, uint32_t (&bits)[N], At at)
{
    constexpr uint32_t kAll = (1u << VEC) - 1u;
#pragma unroll
    for (int u = 0; u < N; ++u) bits[u] = kAll;
    if (!a.mask_rows) return nullptr;
    const int m = ((const const_i32 *)a.mask_rows)[row];
    if (m < 0 || m >= a.num_masks) return nullptr;
    const uint32_t *mask = a.masks + (int64_t)m * a.mask_stride;
#pragma unroll
    for (int u = 0; u < N; ++u) bits[u] = at(u) < end ? mask[at(u) >> 5] : 0u;
#pragma unroll
    for (int u = 0; u < N; ++u) bits[u] = bits[u] >> (at(u) & 31) & kAll;
    return mask;
}

// -inf in the place of what is not allowed.
template <int DTYPE>
__device__ __forceinline__ void strike(u32x4 &y, uint32_t bits)
{
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

template <int DTYPE>
__device__ __forceinline__ u32x4 all_low() { return u32x4{Value<DTYPE>::kLow, Value<DTYPE>::kLow, Value<DTYPE>::kLow, Value<DTYPE>::kLow}; }

// A lane's piece of a row at v, whole or up to the row's end.  NT: logits that the last-level cache does not hold go past it.
template <int DTYPE, bool NT>
__device__ __forceinline__ u32x4 load_piece(const typename Value<DTYPE>::T *row, int v, int end)
{
    constexpr int VEC = 16 / sizeof(*row);
    u32x4 y = all_low<DTYPE>();
    const auto *whole = (const typename Value<DTYPE>::Vec *)(row + v);
    if (v + VEC <= end) y = NT ? __builtin_nontemporal_load(whole) : *whole;
    else
        for (int e = 0; v + e < end; ++e) replace<DTYPE>(y, e, row[v + e]);
    return y;
}
template <int DTYPE, bool NT>
__device__ __forceinline__ void store_piece(typename Value<DTYPE>::T *row, int v, int end, const u32x4 &y)
{
    constexpr int VEC = 16 / sizeof(*row);
    auto *whole = (typename Value<DTYPE>::Vec *)(row + v);
    if (v + VEC <= end) {
        if (NT) __builtin_nontemporal_store((typename Value<DTYPE>::Vec)y, whole);
        else *whole = y;
    } else {
        for (int e = 0; v + e < end; ++e) row[v + e] = (typename Value<DTYPE>::T)element<DTYPE>(y, e);
    }
}

// Masks alone: a workgroup to 16 KB of a row and nothing in LDS.  In place a piece that keeps something is read and written whole:
// 1024 rows of 128256 with one token in 32 allowed 172 us (writing everything without a read 95, reading everything 193; storing the
// struck out logits of such a piece one by one 224).
template <int DTYPE, bool IN_PLACE, bool NT>
__global__ void __launch_bounds__(256) logits_mask_kernel(const RulesArgs a)
{
    using T = typename Value<DTYPE>::T;
    constexpr int VEC = 16 / sizeof(T), U = 4;
    constexpr uint32_t kAll = (1u << VEC) - 1u;
    const int64_t row = (int64_t)blockIdx.z * a.rows + blockIdx.y;
    const int first = (int)blockIdx.x * (256 * VEC * U) + threadIdx.x * VEC, V = a.vocab;
    auto at = [&](int u) __attribute__((always_inline)) { return first + u * 256 * VEC; };
    uint32_t bits[U];
    if (!allowed_of<VEC>(a, row, V, bits, at) && IN_PLACE) return;
    const T *in = (const T *)a.logits + row * a.stride_row;
    T *out = (T *)a.out + row * a.out_stride_row;
    u32x4 y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        y[u] = all_low<DTYPE>();
        if (bits[u] && (!IN_PLACE || bits[u] != kAll)) y[u] = load_piece<DTYPE, NT>(in, at(u), V);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (bits[u] != kAll) strike<DTYPE>(y[u], bits[u]);
        if (at(u) < V && (!IN_PLACE || bits[u] != kAll)) store_piece<DTYPE, NT>(out, at(u), V, y[u]);
    }
}

// PACKED: a token's word holds how often it was written (15 bits), kPromptBit and 16 bits for the bias's place in the list, where the
// host knows that they fit; else two words, the first with the count in 31 bits.  IN_PLACE: out is logits.
template <int DTYPE, bool PACKED, bool IN_PLACE, bool NT>
__global__ void __launch_bounds__(kRulesThreads, 8) logits_rules_kernel(const RulesArgs a)
{
    using T = typename Value<DTYPE>::T;
    constexpr int VEC = 16 / sizeof(T);
    constexpr int U = kStretch / (kRulesThreads * VEC);  // pieces of a lane: a wave's share of a stretch
    static_assert(U * kRulesThreads * VEC == kStretch, "");
    constexpr uint32_t kAll = (1u << VEC) - 1u, kPromptBit = PACKED ? 0x8000u : 0x80000000u;
    extern __shared__ uint32_t smem[];
    uint32_t *words = smem;                              // [kStretch + 64]: behind them a word for each lane's tokens of other stretches
    int *s_token = (int *)(words + kStretch + 64);       // [kMaxNodes]
    unsigned long long *s_path = (unsigned long long *)(s_token + kMaxNodes);  // [kMaxNodes] nodes on a row's path whose token lies in the stretch
    uint32_t *biases = (uint32_t *)(s_path + kMaxNodes); // [kStretch], not PACKED and with biases: 1 + the entry's place in the list

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // The launch has an axis for each of these: divisions by their sizes are a tenth of a small workgroup's instructions (256 rows in bf16
    // 48.0 -> 46.3 us).  In fp32 one axis: with three the compiler spills eight registers (1024 rows 222 -> 236 us).
    int stretch = (int)blockIdx.x, group = (int)blockIdx.y, b = (int)blockIdx.z;
    if constexpr (DTYPE == 0) {
        const unsigned stretches = (unsigned)(a.vocab + kStretch - 1) / kStretch, groups = (unsigned)(a.rows + a.rows_per_wg - 1) / (unsigned)a.rows_per_wg;
        stretch = (int)(blockIdx.x % stretches);
        group = (int)(blockIdx.x / stretches % groups);
        b = (int)(blockIdx.x / (stretches * groups));
    }
    const int v0 = stretch * kStretch, v1 = min(a.vocab, v0 + kStretch);
    const int r0 = group * a.rows_per_wg, r1 = min(a.rows, r0 + a.rows_per_wg);
    const int64_t row0 = (int64_t)b * a.rows;
    // wave w streams tokens first .. first + U * 64 * VEC - 1 of every row, piece u of a lane at `at(u)`
    const int first = v0 + wave * (U * 64 * VEC);
    auto at = [&](int u) __attribute__((always_inline)) { return first + (u * 64 + lane) * VEC; };

    // Everything that hangs on nothing but the sequence goes out first and at once (what is not there is read from the context's
    // word, without a jump), then the first of the history and the first row's logits, so that the counting, which they wait out,
    // is behind three round trips to memory and not ten.
    auto of = [&](const void *p, int at) __attribute__((always_inline)) {
        return ((const const_i32 *)(p ? p : (const void *)a.err_word))[p ? at : 0];
    };
    const int rep = of(a.repetition, b), pres = of(a.presence, b), freq = of(a.frequency, b);
    const int start = of(a.bias_starts, b), stop = of(a.bias_starts, b + 1), len = of(a.history_lens, b), prompt_len = of(a.prompt_lens, b);
    const Penalty penalty(a.repetition ? __int_as_float(rep) : 1.f, a.presence ? __int_as_float(pres) : 0.f, a.frequency ? __int_as_float(freq) : 0.f);
    const bool penalise = penalty.any();
    const int bias0 = max(start, 0), bias1 = a.bias_starts ? (int)min((int64_t)stop, a.num_biases) : 0;
    const int n = penalise && a.history ? (int)min((int64_t)max(len, 0), a.history_stride) : 0;
    const int n0 = a.prompt_lens ? min(max(prompt_len, 0), n) : 0;
    const bool biased = bias0 < bias1;

    // A wave takes every eighth run of 256 tokens of the history, a lane four in a row.
    constexpr int RUN = 256, STEP = RUN * (kRulesThreads / 64);
    const int32_t *text = a.history + (int64_t)b * a.history_stride;
    auto load_text = [&](int i) __attribute__((always_inline)) {
        u32x4 t = {~0u, ~0u, ~0u, ~0u};
        if (i + RUN <= n) {
            t = *(const vec_of_4 *)(text + i + lane * 4);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + lane * 4 + k < n) t[k] = (uint32_t)text[i + lane * 4 + k];
        }
        return t;
    };
    u32x4 t = load_text(wave * RUN);

    // Row r: its mask, what that allows of the lane's pieces, and its logits; in place those that change only.
    const uint32_t *mask;
    uint32_t bits[U], hit[U];  // `hit`: by `touched` and the row's path
    u32x4 y[U];
    auto load_row = [&](int r, auto wanted) __attribute__((always_inline)) {
        const T *in = (const T *)a.logits + (row0 + r) * a.stride_row;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            y[u] = all_low<DTYPE>();
            if (wanted(u)) y[u] = load_piece<DTYPE, NT>(in, at(u), v1);
        }
    };
    mask = allowed_of<VEC>(a, row0 + r0, v1, bits, at);
    if constexpr (!IN_PLACE) load_row(r0, [&](int u) { return bits[u] != 0; });

    uint32_t touched[U];  // by a penalty or a bias, of the lane's pieces
#pragma unroll
    for (int u = 0; u < U; ++u) touched[u] = 0;
    if (penalise || biased) {
        for (int i = tid; i < kStretch / 4; i += kRulesThreads) {
            ((uint4 *)words)[i] = make_uint4(0, 0, 0, 0);
            if (!PACKED && biased) ((uint4 *)biases)[i] = make_uint4(0, 0, 0, 0);
        }
        if (wave == 0) {
            int token = -1;
            unsigned long long path = 0;
            if (penalise && a.tokens) {
                if (lane < a.rows) token = a.tokens[row0 + lane];
                if (token < v0 || token >= v1) token = -1;
                if (a.parents) {
                    const uint2 on = tree_path(a.parents + row0, a.rows);
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
        const uint32_t size = (uint32_t)(v1 - v0);
        for (int i = wave * RUN; i < n; i += STEP) {
            const u32x4 now = t;
            if (i + STEP < n) t = load_text(i + STEP);
            // every lane counts, without a jump: what is of another stretch or no token goes to the lane's own word behind them
            uint32_t *at_word[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t x = now[k] - (uint32_t)v0;
                at_word[k] = &words[x < size ? x : (uint32_t)(kStretch + lane)];
            }
            if (i >= n0) {
#pragma unroll
                for (int k = 0; k < 4; ++k) atomicAdd(at_word[k], 1u);
            } else if (i + RUN <= n0) {  // of the prompt (added twice, the bit would carry)
#pragma unroll
                for (int k = 0; k < 4; ++k) atomicOr(at_word[k], kPromptBit);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (i + lane * 4 + k < n0) atomicOr(at_word[k], kPromptBit);
                    else atomicAdd(at_word[k], 1u);
                }
            }
        }
        for (int i = bias0 + tid; i < bias1; i += kRulesThreads) {
            const uint32_t x = (uint32_t)a.bias_tokens[i] - (uint32_t)v0, place = (uint32_t)(i - bias0 + 1);
            if (x < size) {  // the last entry of a token counts
                if constexpr (PACKED) {
                    uint32_t word = words[x];
                    while (word >> 16 < place) {  // (ends: the place that stands there only grows, and counting is finite)
                        const uint32_t was = atomicCAS(&words[x], word, (word & 0xffffu) | place << 16);
                        if (was == word) break;
                        word = was;
                    }
                } else {
                    atomicMax(&biases[x], place);
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
                const u32x4 w = *(const u32x4 *)&words[at(u) - v0 + e];
                u32x4 p = {0, 0, 0, 0};
                if (!PACKED && biased) p = *(const u32x4 *)&biases[at(u) - v0 + e];
#pragma unroll
                for (int k = 0; k < 4; ++k) touched[u] |= (w[k] | p[k]) ? 1u << (e + k) : 0u;
            }
        }
    }

    for (int r = r0; r < r1; ++r) {
        if (r != r0) mask = allowed_of<VEC>(a, row0 + r, v1, bits, at);
#pragma unroll
        for (int u = 0; u < U; ++u) hit[u] = touched[u];
        unsigned long long path = 0;
        if (penalise || biased) {
            path = s_path[r];
            path = (unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((int)(path >> 32)) << 32 |
                   (uint32_t)__builtin_amdgcn_readfirstlane((int)path);
            for (unsigned long long p = path; p; p &= p - 1) {
                const int s = s_token[__builtin_ctzll(p)];
#pragma unroll
                for (int u = 0; u < U; ++u) hit[u] |= (uint32_t)(s - at(u)) < (uint32_t)VEC ? 1u << ((s - at(u)) & 31) : 0u;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) hit[u] &= bits[u];
        }
        if constexpr (IN_PLACE) load_row(r, [&](int u) { return hit[u] != 0 || (bits[u] != 0 && bits[u] != kAll); });
        else if (r != r0) load_row(r, [&](int u) { return bits[u] != 0; });
        T *out = (T *)a.out + (row0 + r) * a.out_stride_row;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t left = hit[u];
            while (__any(left != 0)) {
                if (left) {
                    const int e = __builtin_ctz(left), v = at(u) + e;
                    left &= left - 1;
                    const uint32_t word = words[v - v0];
                    uint32_t times = word & (kPromptBit - 1u);
                    for (unsigned long long p = path; p; p &= p - 1) times += s_token[__builtin_ctzll(p)] == v ? 1u : 0u;
                    float z = value_of<DTYPE>(element<DTYPE>(y[u], e));
                    if (penalise && (times > 0 || (word & kPromptBit))) z = penalty(z, times);
                    const uint32_t place = PACKED ? word >> 16 : biased ? biases[v - v0] : 0u;
                    if (place) z += a.bias_values[bias0 + place - 1];
                    replace<DTYPE>(y[u], e, bits_of<DTYPE>(z));
                }
            }
            if (mask && bits[u] != kAll) strike<DTYPE>(y[u], bits[u]);
            if (at(u) < v1 && (!IN_PLACE || hit[u] || bits[u] != kAll)) store_piece<DTYPE, NT>(out, at(u), v1, y[u]);
        }
    }
}

template <int DTYPE, bool NT>
static auto rules_kernel(bool packed, bool in_place)
{
    if (packed) return in_place ? logits_rules_kernel<DTYPE, true, true, NT> : logits_rules_kernel<DTYPE, true, false, NT>;
    return in_place ? logits_rules_kernel<DTYPE, false, true, NT> : logits_rules_kernel<DTYPE, false, false, NT>;
}
template <int DTYPE, bool NT>
static auto mask_kernel(bool in_place) { return in_place ? logits_mask_kernel<DTYPE, true, NT> : logits_mask_kernel<DTYPE, false, NT>; }

template <int DTYPE, bool NT>
static hipError_t launch_rules(RulesArgs a, int num_cus, hipStream_t stream)
{
    if (!a.repetition && !a.presence && !a.frequency && !a.bias_starts) {
        constexpr int PART = 256 * 4 * (DTYPE == 0 ? 4 : 8);
        const dim3 grid((unsigned)((a.vocab + PART - 1) / PART), (unsigned)a.rows, (unsigned)a.batch);
        hipLaunchKernelGGL((mask_kernel<DTYPE, NT>(a.in_place)), grid, dim3(256), 0, stream, a);
        return hipGetLastError();
    }
    // Rows share a workgroup's counters as long as there are eight rounds of workgroups, four of which are resident on a CU (1024 rows
    // of 151936, histories of 500..30000: four rounds 240 us, eight 222, sixteen 241).
    const int stretches = (a.vocab + kStretch - 1) / kStretch;
    a.rows_per_wg = a.rows;
    while (a.rows_per_wg > 1 && (int64_t)a.batch * stretches * ((a.rows + a.rows_per_wg - 1) / a.rows_per_wg) < 32ll * num_cus)
        a.rows_per_wg = (a.rows_per_wg + 1) / 2;
    const unsigned groups = (unsigned)((a.rows + a.rows_per_wg - 1) / a.rows_per_wg);
    const dim3 grid = DTYPE == 0 ? dim3((unsigned)stretches * groups * (unsigned)a.batch) : dim3((unsigned)stretches, groups, (unsigned)a.batch);
    // By what the buffers can hold: the host does not see the lengths.  Texts of 50..8000 in a buffer of 65536: with biases (two words, half the
    // workgroups on a CU) 40 -> 54 us, without 37.5 -> 38.7; the 1024 rows 221 -> 256.
    const bool packed = (!a.history || a.history_stride < 0x8000) && a.num_biases < 0x10000;
    const size_t lds = (kStretch + 64) * 4 + kMaxNodes * 12 + (!packed && a.bias_starts ? kStretch * 4 : 0);
    hipLaunchKernelGGL((rules_kernel<DTYPE, NT>(packed, a.in_place)), grid, dim3(kRulesThreads), lds, stream, a);
    return hipGetLastError();
}

hipError_t launch_logits_process(const RulesArgs &a, int num_cus, hipStream_t stream)
{
    if (a.batch == 0 || (a.in_place && !a.masks && !a.repetition && !a.presence && !a.frequency && !a.bias_starts)) return hipSuccess;
    // What the 256 MB last-level cache cannot keep for whoever reads it next: 1024 rows of 128256 in fp32, masks in place 174 -> 148 us, of
    // 151936 with every rule out of place 246 -> 236.  Below that ordinary accesses, though 256 rows in bf16, 155 MB, would take 2 us less.
    const double bytes = (double)a.batch * a.rows * a.vocab * (a.dtype == 0 ? 4 : 2) * (a.in_place ? 1 : 2);
    const bool nt = bytes > 1.25 * 256.0 * 1024 * 1024;
    switch (a.dtype) {
    case 0: return nt ? launch_rules<0, true>(a, num_cus, stream) : launch_rules<0, false>(a, num_cus, stream);
    case 1: return nt ? launch_rules<1, true>(a, num_cus, stream) : launch_rules<1, false>(a, num_cus, stream);
    default: return nt ? launch_rules<2, true>(a, num_cus, stream) : launch_rules<2, false>(a, num_cus, stream);
    }
}

}  // namespace orthrus
