// Sampling filters on gfx950: temperature, top-k, top-p and min-p of a logits row, the token drawn from what they keep by a
// given uniform number, and the lossless consensus of a block whose two views are both filtered.
//
// With M the row's maximum and w_v = exp((x_v - M) / T), the filters cut the tokens ordered by (logit falling, index
// rising): the first top_k; of those the shortest prefix that holds top_p of their weight; of those the ones with
// w >= min_p.  The token is the first one in index order at which the running sum of the kept weights exceeds u times
// their sum.  Every step is "find where a running sum over an order crosses a target".  The sums are whole numbers (weights
// in fixed point, scaled so that the row's sum fills 61 bits), so they do not depend on the order in which they are taken;
// the weights are taken in 64 bits, because a token next to a cut or to the uniform number is decided by the last bits
// of a sum over the vocabulary: with a sum good to 1e-7 one row in a few thousand would draw another token.
//
//   filter_row_kernel      one workgroup per row (and view).
//   filtered_draw_kernel   one workgroup per sequence: keep decisions, the replacement drawn from the first rejected row.
//   filtered_commit_kernel grid (sequence, layer): outputs and the commit, as sample_commit_kernel does it.
#include "orthrus_internal.h"

#include <cfloat>

namespace orthrus {

typedef unsigned long long u64;

constexpr int kRowThreads = 1024;
constexpr int kBins = 2048;

// ---- logits, their order and their weights

template <int DT> __device__ __forceinline__ float raw_logit(const void *row, int i)
{
    if constexpr (DT == 0) return ((const float *)row)[i];
    else if constexpr (DT == 1) return __uint_as_float((uint32_t)((const uint16_t *)row)[i] << 16);
    else return (float)((const _Float16 *)row)[i];
}

// NaN counts as -inf (never kept), +inf as the largest float, -0 as 0.
__device__ __forceinline__ float clean_logit(float x)
{
    return x > -INFINITY ? fminf(x, FLT_MAX) + 0.f : -INFINITY;
}

template <int DT> __device__ __forceinline__ float logit(const void *row, int i) { return clean_logit(raw_logit<DT>(row, i)); }

template <int DT> __device__ __forceinline__ const void *logit_row(const FilterArgs &a, int side, int row)
{
    return (const char *)a.logits[side] + (int64_t)row * a.stride_row * (DT == 0 ? 4 : 2);
}

// A whole number that orders like the logit.
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u >> 31 ? ~u : u | 0x80000000u;
}

// 2^t for t <= 0: t = n + f with n whole and |f| <= 1/2, 2^f by a polynomial in f that interpolates 2^f at the Chebyshev
// nodes of [-1/2, 1/2] (off by 4e-14 at most, exactly 1 at 0), n added to the exponent.  Below 2^-1000: 2^-1000.
__device__ __forceinline__ double exp2_neg(double t)
{
    t = fmax(t, -1000.0);
    constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52: adding it rounds to a whole number, in the low bits
    const double s = t + kRound;
    const double f = t - (s - kRound);
    double q = 0x1.b63880a30e9ffp-24;
    q = fma(q, f, 0x1.63d136366db24p-20);
    q = fma(q, f, 0x1.ffcb9515a8016p-17);
    q = fma(q, f, 0x1.4308ac85aa947p-13);
    q = fma(q, f, 0x1.5d87fe86fe88ep-10);
    q = fma(q, f, 0x1.3b2ab7181b755p-7);
    q = fma(q, f, 0x1.c6b08d7047e52p-5);
    q = fma(q, f, 0x1.ebfbdff823cedp-3);
    q = fma(q, f, 0x1.62e42fefa39efp-1);
    const double p = fma(q, f, 1.0);
    return __hiloint2double(__double2hiint(p) + (__double2loint(s) << 20), __double2loint(p));
}

// Weight of a logit relative to the row's maximum; scale = log2(e) / T.
__device__ __forceinline__ double weight(float x, float top, double scale) { return exp2_neg(((double)x - (double)top) * scale); }

struct RowFilter {
    double scale;  // log2(e) / T
    int top_k;     // 0: off
    double top_p;  // >= 1: off
    double min_p;  // 0: off
};

__device__ __forceinline__ RowFilter row_filter(const FilterArgs &a, int b)
{
    RowFilter f;
    const float t = a.temperature[b];
    const int k = a.top_k ? a.top_k[b] : 0;
    const float p = a.top_p ? a.top_p[b] : 1.f, m = a.min_p ? a.min_p[b] : 0.f;
    const bool greedy = !(t > 0.f);  // T <= 0 or NaN: the largest logit, the lowest index among equals
    f.scale = greedy ? 1.4426950408889634 : 1.4426950408889634 / (double)fminf(t, FLT_MAX);
    f.top_k = greedy ? 1 : k > 0 && k < a.vocab ? k : 0;
    f.top_p = greedy || !(p < 1.f) ? 1.0 : fmax((double)p, 0.0);
    f.min_p = greedy || !(m > 0.f) ? 0.0 : (double)fminf(m, 1.f);
    return f;
}

// What the row's cuts keep.
__device__ __forceinline__ bool kept(const RowCut &c, float x, int i)
{
    const uint32_t key = order_key(x);
    return x > -INFINITY && (key > c.key || (key == c.key && i <= c.tie));
}

// ---- running sums over bins in LDS

struct Crossing {
    int bin;      // first bin whose running sum reaches the target, -1 if none does
    u64 before;   // the running sum before it
    u64 at;       // the bin's own amount
};

struct RowShared {
    u64 bins[kBins];
    u64 wave_sum[kRowThreads / 64];
    double wave_z[kRowThreads / 64];
    float wave_max[kRowThreads / 64];
    int wave_alive[kRowThreads / 64];
    Crossing hit;
};

__device__ __forceinline__ void clear_bins(RowShared &s, int tid)
{
    __syncthreads();
    for (int i = tid; i < kBins; i += kRowThreads) s.bins[i] = 0;
    __syncthreads();
}

// Contains barriers; target >= 1.
__device__ __forceinline__ Crossing find_crossing(RowShared &s, int tid, u64 target)
{
    static_assert(kBins == 2 * kRowThreads, "two bins to a thread");
    __syncthreads();
    const u64 h0 = s.bins[2 * tid], h1 = s.bins[2 * tid + 1];
    u64 sum = h0 + h1;
    const int lane = tid & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const u64 o = __shfl_up(sum, off);
        if (lane >= off) sum += o;
    }
    if (lane == 63) s.wave_sum[tid >> 6] = sum;
    if (tid == 0) s.hit = {-1, 0, 0};
    __syncthreads();
    u64 before = sum - h0 - h1;
    for (int w = 0; w < (tid >> 6); ++w) before += s.wave_sum[w];
    if (before < target && target <= before + h0) s.hit = {2 * tid, before, h0};
    else if (before + h0 < target && target <= before + h0 + h1) s.hit = {2 * tid + 1, before + h0, h1};
    __syncthreads();
    return s.hit;
}

__device__ __forceinline__ u64 to_fixed(double w, double unit) { return (u64)(w * unit + 0.5); }

// One row in the hands of a workgroup.  Every method is called by all threads and contains barriers.
template <int DT> struct RowScan {
    RowShared &s;
    const void *row;
    int vocab, tid, idx_shift;   // idx_shift: tokens to a bin of the searches by index
    float top;
    double scale, unit;          // unit: fixed-point value of the weight 1
    RowCut cut;

    __device__ __forceinline__ float at(int i) const { return logit<DT>(row, i); }
    __device__ __forceinline__ double weight_of(float x) const { return weight(x, top, scale); }

    // Maximum, number of logits above -inf.
    __device__ __forceinline__ int find_top()
    {
        top = -INFINITY;
        int alive = 0;
        for (int i = tid; i < vocab; i += kRowThreads) {
            const float x = at(i);
            top = fmaxf(top, x);
            alive += x > -INFINITY;
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) {
            top = fmaxf(top, __shfl_xor(top, off));
            alive += __shfl_xor(alive, off);
        }
        if ((tid & 63) == 0) { s.wave_max[tid >> 6] = top; s.wave_alive[tid >> 6] = alive; }
        __syncthreads();
        alive = 0;
        for (int w = 0; w < kRowThreads / 64; ++w) { top = fmaxf(top, s.wave_max[w]); alive += s.wave_alive[w]; }
        return alive;
    }

    // The sum of all weights sets the fixed point: sums stay below 2^61.
    __device__ __forceinline__ void find_unit()
    {
        double z = 0.0;
        for (int i = tid; i < vocab; i += kRowThreads) z += weight_of(at(i));
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) z += __shfl_xor(z, off);
        if ((tid & 63) == 0) s.wave_z[tid >> 6] = z;
        __syncthreads();
        z = 0.0;
        for (int w = 0; w < kRowThreads / 64; ++w) z += s.wave_z[w];
        unit = exp2((double)min(50, 60 - ilogb(z)));
    }

    __device__ __forceinline__ u64 amount(float x, int i, double min_w) const
    {
        const double w = weight_of(x);
        return kept(cut, x, i) && w >= min_w ? to_fixed(w, unit) : 0;
    }

    // Weight of what the cut keeps.
    __device__ __forceinline__ u64 mass(double min_w)
    {
        u64 m = 0;
        for (int i = tid; i < vocab; i += kRowThreads) m += amount(at(i), i, min_w);
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) m += __shfl_xor(m, off);
        __syncthreads();
        if ((tid & 63) == 0) s.wave_sum[tid >> 6] = m;
        __syncthreads();
        m = 0;
        for (int w = 0; w < kRowThreads / 64; ++w) m += s.wave_sum[w];
        return m;
    }

    // The logit at which a sum in falling order reaches `target` (MASS: of weights, else of ones): eleven, eleven and ten
    // bits of the order at a time.  Returns its key, what lies above it and what lies at it (nothing: never reached).
    struct Selected {
        uint32_t key;
        u64 above, here;
    };
    template <bool MASS> __device__ __forceinline__ Selected select(u64 target)
    {
        Selected r = {0, 0, 0};
        uint32_t prefix = 0;
#pragma unroll 1
        for (int level = 0; level < 3; ++level) {
            const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
            clear_bins(s, tid);
            for (int i = tid; i < vocab; i += kRowThreads) {
                const float x = at(i);
                const uint32_t falling = ~order_key(x);
                if (x > -INFINITY && (level == 0 || falling >> (shift + bits) == prefix))
                    atomicAdd(&s.bins[(falling >> shift) & ((1u << bits) - 1)], MASS ? to_fixed(weight_of(x), unit) : 1ull);
            }
            const Crossing c = find_crossing(s, tid, target - r.above);
            if (c.bin < 0) return {0, 0, 0};
            r.above += c.before;
            r.here = c.at;
            prefix = prefix << bits | (uint32_t)c.bin;
        }
        r.key = ~prefix;
        return r;
    }

    // First token in index order at which the running sum of `amount_at(token)` reaches the target; -1: none.
    template <typename F> __device__ __forceinline__ int first_index(u64 target, F amount_at)
    {
        clear_bins(s, tid);
        for (int i = tid; i < vocab; i += kRowThreads) {
            const u64 n = amount_at(i);
            if (n) atomicAdd(&s.bins[i >> idx_shift], n);
        }
        const Crossing c = find_crossing(s, tid, target);
        if (c.bin < 0 || idx_shift == 0) return c.bin;
        const int base = c.bin << idx_shift, end = min(vocab, base + (1 << idx_shift));
        clear_bins(s, tid);
        for (int i = base + tid; i < end; i += kRowThreads) s.bins[i - base] = amount_at(i);
        return base + find_crossing(s, tid, target - c.before).bin;
    }

    __device__ __forceinline__ int nth_of_key(uint32_t key, u64 n)
    {
        const int i = first_index(n, [&](int j) __attribute__((always_inline)) { return (u64)(order_key(at(j)) == key); });
        return i < 0 ? 0x7fffffff : i;
    }

    __device__ __forceinline__ void cut_top_k(int k)
    {
        const Selected r = select<false>((u64)k);
        cut.key = r.key;
        if (r.above + r.here > (u64)k) cut.tie = nth_of_key(r.key, (u64)k - r.above);
    }

    // Shortest prefix of what is kept so far that holds the share p of its weight.
    __device__ __forceinline__ void cut_top_p(double p)
    {
        const u64 target = max(1ull, (u64)ceil(p * (double)mass(0.0)));
        const Selected r = select<true>(target);
        if (r.here == 0) return;
        const u64 each = to_fixed(weight_of(__uint_as_float(r.key >> 31 ? r.key & 0x7fffffffu : ~r.key)), unit);
        const u64 n = (target - r.above + each - 1) / each;   // so many of the tokens at that logit
        if (r.key > cut.key) cut.tie = 0x7fffffff;
        cut.key = r.key;
        if (n * each < r.here) cut.tie = min(cut.tie, nth_of_key(r.key, n));
    }
};

template <int DT, bool DRAW> __global__ void __launch_bounds__(kRowThreads) filter_row_kernel(const FilterArgs a)
{
    const int row = blockIdx.x, side = blockIdx.y, tid = threadIdx.x;
    __shared__ RowShared s;
    const RowFilter f = row_filter(a, row / a.block_k);
    RowScan<DT> r = {s, logit_row<DT>(a, side, row), a.vocab, tid, 0, 0.f, f.scale, 1.0, {0.0, 0.f, 0.f, 0u, 0x7fffffff}};
    while (((a.vocab - 1) >> r.idx_shift) >= kBins) ++r.idx_shift;
    const int alive = r.find_top();
    int token = -1;
    double own_weight = 0.0;
    r.cut.top = r.top;
    r.cut.min_w = (float)f.min_p;
    if (alive > 0) {
        r.find_unit();
        if (f.top_k > 0 && f.top_k < alive) r.cut_top_k(f.top_k);
        if (f.top_p < 1.0) r.cut_top_p(f.top_p);
        const u64 total = r.mass(f.min_p);
        r.cut.z = (double)total / r.unit;
        if (DRAW) {
            const float u = fminf(fmaxf(a.u[row], 0.f), 0x1.fffffep-1f);
            token = r.first_index((u64)((double)u * (double)total) + 1,
                                  [&](int i) __attribute__((always_inline)) { return r.amount(r.at(i), i, f.min_p); });
            own_weight = r.weight_of(r.at(token));
        }
    }
    if (tid == 0) {
        if (DRAW) {
            a.tokens[row] = token;
            if (a.logprobs) a.logprobs[row] = token < 0 ? -INFINITY : (float)log(own_weight / r.cut.z);
        } else {
            a.cuts[(int64_t)side * a.rows + row] = r.cut;
        }
    }
}

size_t filter_workspace_bytes(int64_t, int, int) { return 0; }

template <bool DRAW> static hipError_t launch_filter_rows(const FilterArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)a.rows, DRAW ? 1u : 2u);
    if (a.dtype == 0) hipLaunchKernelGGL((filter_row_kernel<0, DRAW>), grid, dim3(kRowThreads), 0, stream, a);
    else if (a.dtype == 1) hipLaunchKernelGGL((filter_row_kernel<1, DRAW>), grid, dim3(kRowThreads), 0, stream, a);
    else hipLaunchKernelGGL((filter_row_kernel<2, DRAW>), grid, dim3(kRowThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_sample_tokens(const FilterArgs &a, hipStream_t stream) { return launch_filter_rows<true>(a, stream); }

// ---- consensus

// Probability that a row's filters leave a token (0: cut, or an empty row).
__device__ __forceinline__ double kept_prob(const RowCut &c, double scale, float x, int i)
{
    if (!kept(c, x, i)) return 0.0;
    const double t = ((double)x - (double)c.top) * scale, w = t < -1000.0 ? 0.0 : exp2_neg(t);
    return w >= (double)c.min_w ? w / c.z : 0.0;
}

struct Candidate {
    double score;
    int index;
    __device__ __forceinline__ void take(double v, int i)
    {
        if (v > score || (v == score && i < index)) { score = v; index = i; }
    }
};

template <int DT> __global__ void __launch_bounds__(kRowThreads) filtered_draw_kernel(const FilteredArgs a)
{
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int K = a.c.block_k, V = a.c.vocab;
    const double scale = row_filter(a.f, b).scale;
    __shared__ int s_keep[32];
    __shared__ Candidate s_best[2][kRowThreads / 64];
    if (tid < K) {
        const int row = b * K + tid, x = a.c.draft_tokens[row];
        bool keep = false;
        if (x >= 0 && x < V) {
            const double p = kept_prob(a.f.cuts[row], scale, logit<DT>(logit_row<DT>(a.f, 0, row), x), x);
            const double q = kept_prob(a.f.cuts[a.f.rows + row], scale, logit<DT>(logit_row<DT>(a.f, 1, row), x), x);
            keep = (double)a.accept_u[row] * q < p;
        }
        s_keep[tid] = keep;
    }
    __syncthreads();
    const unsigned long long rej = ~__ballot(lane >= K || s_keep[lane < K ? lane : 0]);
    const int j = rej ? __ffsll((long long)rej) - 1 : K;
    if (tid == 0) {
        a.c.decided[b] = j;
        if (a.c.do_commit) commit_snapshot(a.c, b);
    }
    if (j >= K) return;
    const int row = b * K + j;
    const void *pr = logit_row<DT>(a.f, 0, row), *qr = logit_row<DT>(a.f, 1, row);
    const RowCut cp = a.f.cuts[row], cq = a.f.cuts[a.f.rows + row];
    Candidate more = {-INFINITY, 0x7fffffff}, any = {-INFINITY, 0x7fffffff};  // best among p > q, best of p
    for (int i = tid; i < V; i += kRowThreads) {
        const double p = kept_prob(cp, scale, logit<DT>(pr, i), i);
        if (p > 0.0) {
            const double q = kept_prob(cq, scale, logit<DT>(qr, i), i), g = (double)a.gumbel[(int64_t)b * V + i];
            if (p > q) more.take(log(p - q) + g, i);
            any.take(log(p) + g, i);
        }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        const double v0 = __shfl_xor(more.score, off), v1 = __shfl_xor(any.score, off);
        const int i0 = __shfl_xor(more.index, off), i1 = __shfl_xor(any.index, off);
        more.take(v0, i0);
        any.take(v1, i1);
    }
    if (lane == 0) { s_best[0][wave] = more; s_best[1][wave] = any; }
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kRowThreads / 64; ++w) {
            more.take(s_best[0][w].score, s_best[0][w].index);
            any.take(s_best[1][w].score, s_best[1][w].index);
        }
        a.replacement[b] = more.index != 0x7fffffff ? more.index : any.index != 0x7fffffff ? any.index : -1;
    }
}

// The workgroup of layer 0 writes the outputs, every layer's copies its layer's kept rows.  Only layer 0's reads the
// drafts, before it writes the tokens: out_tokens may be draft_tokens.
__global__ void __launch_bounds__(256) filtered_commit_kernel(const FilteredArgs a)
{
    const ConsensusArgs &c = a.c;
    const int b = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x;
    const bool lead = layer == 0;
    const int K = c.block_k;
    __shared__ int s_L, s_m;
    __shared__ int s_pg[32];
    if (tid < 64) {
        const int lane = tid, j = c.decided[b];
        CommitProbe probe = {0, -1};
        if (c.do_commit) probe = commit_probe(c, b, lane);
        const int m = min(j + 1, K);
        if (lead) {
            const int repl = j < K ? a.replacement[b] : -1;
            const int draft = lane < K ? c.draft_tokens[(int64_t)b * K + lane] : -1;
            if (lane < K) c.out_tokens[(int64_t)b * K + lane] = lane < j ? draft : lane == j ? repl : -1;
            const int last = __shfl(draft, K - 1);
            if (lane == 0) {
                c.accept_len[b] = j;
                c.next_anchor[b] = j < K ? repl : last;
            }
        }
        int committed = m;
        if (c.do_commit) {
            committed = commit_decide(c, b, lane, m, probe, lead);
            if (lane < K) s_pg[lane] = probe.pg;
        }
        if (lane == 0) {
            if (lead) c.num_committed[b] = committed;
            s_L = probe.L;
            s_m = c.do_commit ? committed : 0;
        }
    }
    __syncthreads();
    if (s_m > 0) append_rows(c, b, layer, s_L, s_m, tid, 256, s_pg);
}

hipError_t launch_filtered_consensus(const FilteredArgs &a, hipStream_t stream)
{
    const ConsensusArgs &c = a.c;
    hipError_t e = launch_filter_rows<false>(a.f, stream);
    if (e != hipSuccess) return e;
    if (a.f.dtype == 0) hipLaunchKernelGGL((filtered_draw_kernel<0>), dim3(c.batch), dim3(kRowThreads), 0, stream, a);
    else if (a.f.dtype == 1) hipLaunchKernelGGL((filtered_draw_kernel<1>), dim3(c.batch), dim3(kRowThreads), 0, stream, a);
    else hipLaunchKernelGGL((filtered_draw_kernel<2>), dim3(c.batch), dim3(kRowThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(filtered_commit_kernel, dim3(c.batch, c.do_commit ? c.num_layers : 1), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace orthrus
