// Sampling filters on gfx950: temperature, top-k, top-p and min-p of a logits row, the token drawn from what they keep by a
// given uniform number, and the lossless consensus of a block whose two views are both filtered.
//
// With M the row's maximum and w_v = exp((x_v - M) / T), the filters cut the tokens ordered by (logit falling, index
// rising): the first top_k; of those the shortest prefix that holds top_p of their weight; of those the ones with
// w >= min_p.  The token is the first one in index order at which the running sum of the kept weights exceeds u times
// their sum.  Every step is "find where a running sum over an order crosses a target".  Running sums are of whole numbers (weights
// in fixed point, scaled so that the row's sum fills 61 bits), so they do not depend on the order in which they are taken;
// the weights are taken in 64 bits, because a token next to a cut or to the uniform number is decided by the last bits
// of a sum over the vocabulary: with a sum good to 1e-7 one row in a few thousand would draw another token.  The sum of a whole row
// that the scan leaves (top-p's target, an unfiltered row's chunks) is one of 64-bit floats over chunks that begin at 16-byte
// boundaries: always the same for a row, but a copy of it at another alignment may differ in the last bits.
//
//   filter_scan_kernel     a wave to a chunk of 2048 logits, the one pass over them: the chunk's maximum, the sum of its weights
//                          and a list of its largest logits, some thirty.  Bound by the vector unit where weights are summed
//                          (18 instructions each, 64 bits at full rate), else near the stream: 1024 rows of 151936, 622 MB,
//                          104 us without the weights of any row, 156 with those of all, 94 for the plain argmax scan.
//   filter_pick_kernel     a workgroup to a row: cuts and token from the lists of its chunks, which together hold every logit down to
//                          the highest of their thresholds (some thousand); what the first cut leaves is ranked in the lanes of a
//                          wave.  A row without filters: from the chunks' sums, and one chunk read again.  A row whose cut lies
//                          below the lists goes to the next kernel.  Rows of at most 1792 logits come here at once.  Bound by
//                          its chain of memory and LDS round trips, 7 to 19 us; 1024 rows 35 us.
//   filter_wide_kernel     a workgroup to such a row: a histogram pass and a pass that gathers the step of the cut; bound by the
//                          weights of both passes (256 rows of 151936, nuclei of tens of thousands: 124 us).
//   filtered_stage_kernel  keep decisions between the consensus's two stages.
//   filtered_draw_kernel   grid (piece, sequence): keep decisions, the replacement drawn from the first rejected row.
//   filtered_commit_kernel grid (sequence, layer): outputs and the commit, as sample_commit_kernel does it.
#include "orthrus_internal.h"
#include "orthrus_lanes.h"

#include <cfloat>

namespace orthrus {

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

// The i-th of the rows that a launch is about: block rows first_k .. first_k + stage_k - 1 of every sequence and view.  -1: the
// sequence has lost a draft already, its later rows are not asked for.
__device__ __forceinline__ int stage_row(const FilterArgs &a, int i)
{
    const int side = i >= a.stage_rows, r = i - side * a.stage_rows, b = r / a.stage_k;
    if (a.decided && a.decided[b] < a.first_k) return -1;
    return side * a.rows + b * a.block_k + a.first_k + (r - b * a.stage_k);
}

// A whole number that orders like the logit.
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u >> 31 ? ~u : u | 0x80000000u;
}

// Weight of a logit d <= 0 away from the row's maximum: 2^(d * scale) with scale = log2(e) / T.  d * scale = n + f with n whole and
// |f| <= 1/2; 2^f by a polynomial that interpolates it at the Chebyshev nodes of [-1/2, 1/2] (off by 4e-14 at most, exactly 1
// at 0), n added to the exponent.  d is exact and the product rounded once at f, so equal logits weigh exactly 1 at any
// temperature.  Weights end at 2^-1000 (d = floor).
struct Scale {
    double scale, floor;
};
__device__ __forceinline__ double weight(double d, const Scale &t)
{
    d = fmax(d, t.floor);
    constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52: adding it rounds to a whole number, in the low bits
    const double s = fma(d, t.scale, kRound);
    const double f = fma(d, t.scale, -(s - kRound));
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
__device__ __forceinline__ double weight(float x, float top, const Scale &t) { return weight((double)x - (double)top, t); }

struct RowFilter {
    Scale t;
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
    f.t.scale = greedy ? 1.4426950408889634 : 1.4426950408889634 / (double)fminf(t, FLT_MAX);
    f.t.floor = (greedy ? 1.0 : (double)fminf(t, FLT_MAX)) * -693.14718055994531;
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

// Bins of a workgroup of THREADS, PER of them to a thread.  They are zero except between the first amount that is added and
// the search, which leaves zeros behind.  Every function contains barriers, the last of them behind its last access.
template <int THREADS, int PER> struct Bins {
    static constexpr int kCount = THREADS * PER, kWaves = THREADS / 64;
    u64 amount[kCount];
    u64 wave_total[kWaves];
    Crossing hit;

    __device__ __forceinline__ void clear(int tid)   // once, before the first use
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) amount[i * THREADS + tid] = 0;
        __syncthreads();
    }

    // target >= 1
    __device__ __forceinline__ Crossing crossing(int tid, u64 target)
    {
        __syncthreads();
        u64 h[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) { h[i] = amount[tid * PER + i]; sum += h[i]; }
#pragma unroll
        for (int i = 0; i < PER; ++i) amount[tid * PER + i] = 0;
        const u64 run = wave_scan(sum);
        if ((tid & 63) == 63) wave_total[tid >> 6] = run;
        if (tid == 0) hit = {-1, 0, 0};
        __syncthreads();
        u64 before = run - sum;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) before += w < (tid >> 6) ? wave_total[w] : 0;
        if (before < target && target <= before + sum) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (before < target && target <= before + h[i]) hit = {tid * PER + i, before, h[i]};
                before += h[i];
            }
        }
        __syncthreads();
        const Crossing c = hit;
        __syncthreads();
        return c;
    }

    __device__ __forceinline__ u64 sum_of(int tid, u64 v)
    {
        v = wave_sum(v);
        if ((tid & 63) == 0) wave_total[tid >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += wave_total[w];
        __syncthreads();
        return v;
    }
};

__device__ __forceinline__ u64 to_fixed(double w, double unit) { return (u64)(w * unit + 0.5); }

// ---- the pass over the logits

constexpr int kScanThreads = 256;  // four waves

template <int DT> struct Vector {
    static constexpr int kCount = DT == 0 ? 4 : 8;  // logits to 16 bytes
};

// The logits of 16 bytes as they are.
template <int DT> __device__ __forceinline__ void unpack(uint4 q, float *x)
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == 0) {
            x[i] = __uint_as_float(w[i]);
        } else if constexpr (DT == 1) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            const uint16_t lo = (uint16_t)w[i], hi = (uint16_t)(w[i] >> 16);
            x[2 * i] = (float)__builtin_bit_cast(_Float16, lo);
            x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, hi);
        }
    }
}

// A chunk of a row, one wave's: kChunk logits from a 16-byte boundary on, so that all but a row's first and last vector are
// loaded whole.  `first` is the row index of its first logit (negative in a row that starts inside a vector).
constexpr int kEach = 32, kChunk = 64 * kEach, kListCap = 128;

template <int DT> __device__ __forceinline__ int row_skew(const void *row)   // logits between the boundary and the row's start
{
    constexpr int kVec = Vector<DT>::kCount;
    return (int)((uintptr_t)row / (16 / kVec)) & (kVec - 1);
}

template <int DT> struct Chunk {
    static constexpr int kVec = Vector<DT>::kCount, kLoads = kEach / kVec;
    const void *row;
    int first, vocab;

    __device__ __forceinline__ int index(int load, int lane) const { return first + (load * 64 + lane) * kVec; }
    // (raw: not cleaned)
    template <bool NT> __device__ __forceinline__ void load(int lane, float (&x)[kEach]) const
    {
        typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
        const u32x4 *at = (const u32x4 *)((const char *)row + (int64_t)first * (16 / kVec)) + lane;
        auto one = [&](int u) __attribute__((always_inline)) {
            u32x4 q;
            if constexpr (NT) q = __builtin_nontemporal_load(at + u * 64);
            else q = at[u * 64];
            return make_uint4(q[0], q[1], q[2], q[3]);
        };
        if (first >= 0 && first + kChunk <= vocab) {
            uint4 q[kLoads];
#pragma unroll
            for (int u = 0; u < kLoads; ++u) q[u] = one(u);
#pragma unroll
            for (int u = 0; u < kLoads; ++u) unpack<DT>(q[u], &x[u * kVec]);
        } else {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const int i = index(u, lane);
                if (i >= 0 && i + kVec <= vocab) {
                    unpack<DT>(one(u), &x[u * kVec]);
                } else {
#pragma unroll
                    for (int r = 0; r < kVec; ++r)
                        x[u * kVec + r] = i + r >= 0 && i + r < vocab ? raw_logit<DT>(row, i + r) : -INFINITY;
                }
            }
        }
    }
};

// Which rows need the sum of all their weights: those that a share of it cuts, and those that nothing cuts.
__device__ __forceinline__ bool wants_sum(const RowFilter &f) { return f.top_k == 0 && (f.top_p < 1.0 || f.min_p == 0.0); }

// The three least of two sorted triples.
struct Least {
    float a, b, c;
    __device__ __forceinline__ void merge(float a2, float b2, float c2)
    {
        const float c3 = fminf(fminf(c, c2), fminf(fmaxf(b, a2), fmaxf(a, b2)));
        b = fminf(fminf(b, b2), fmaxf(a, a2));
        a = fminf(a, a2);
        c = c3;
    }
};

// A wave to a chunk, without a word to the others: waves that wait for their loads then run beside waves that compute.
// The list's threshold is the third least of the maxima of sixteen groups of four lanes (of those that hold anything): 30
// logits +- 10 reach it in a row without order.  (The least one of all leaves 54, with a tail that overruns a list of 128
// in one chunk of 200.)  NT: the logits are more than the last-level cache holds.
template <int DT, bool NT> __global__ void __launch_bounds__(kScanThreads) filter_scan_kernel(const FilterArgs a)
{
    const int lane = threadIdx.x & 63;
    const uint32_t item = blockIdx.x * (kScanThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item == 0 && lane == 0) a.unresolved[0] = 0;
    const int nth = (int)(item / (uint32_t)a.chunks), chunk = (int)(item - (uint32_t)nth * a.chunks);
    if (nth >= a.all_rows) return;
    const int rr = stage_row(a, nth);
    if (rr < 0) return;
    const int side = rr >= a.rows, row = rr - side * a.rows;
    const int64_t place = (int64_t)rr * a.chunks + chunk;
    const void *logits = logit_row<DT>(a, side, row);
    const Chunk<DT> c = {logits, chunk * kChunk - row_skew<DT>(logits), a.vocab};
    float x[kEach];
    c.template load<NT>(lane, x);
    float top = x[0];
#pragma unroll
    for (int i = 1; i < kEach; ++i) top = fmaxf(top, x[i]);
    top = fmaxf(top, swap_f32<kSwap1>(top));
    top = fmaxf(top, swap_f32<kSwap2>(top));
    const bool hollow = !(top > -INFINITY);   // (also where all are NaN)
    Least low = {hollow ? INFINITY : top, INFINITY, INFINITY};
    if (hollow) top = -INFINITY;
    low.merge(swap_f32<kMirror8>(low.a), swap_f32<kMirror8>(low.b), swap_f32<kMirror8>(low.c));
    low.merge(swap_f32<kMirror16>(low.a), swap_f32<kMirror16>(low.b), swap_f32<kMirror16>(low.c));
    low.merge(__shfl_xor(low.a, 16), __shfl_xor(low.b, 16), __shfl_xor(low.c, 16));
    low.merge(__shfl_xor(low.a, 32), __shfl_xor(low.b, 32), __shfl_xor(low.c, 32));
    top = wave_max(top);
    float tau = low.c < INFINITY ? low.c : low.b < INFINITY ? low.b : low.a < INFINITY ? low.a : -INFINITY;
    if (top == INFINITY) {   // +inf counts as the largest float.  (A NaN drops out of all that follows by itself.)
        top = FLT_MAX;
#pragma unroll
        for (int i = 0; i < kEach; ++i) x[i] = clean_logit(x[i]);
        tau = low.a < INFINITY ? fminf(tau, FLT_MAX) : FLT_MAX;
    }
    if (__ballot(hollow) != 0) {   // few logits, the others masked: list them all if there is room
        int alive = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) alive += __popcll(__ballot(x[i] > -INFINITY));
        if (alive <= kListCap) tau = -INFINITY;
    }
    // ---- the list, in the order of loads and lanes; through LDS, so that it leaves with one store (stores of one or two
    // lanes each took 24 us of 113)
    __shared__ uint2 s_list[kScanThreads / 64][kListCap];
    uint2 *mine = s_list[threadIdx.x >> 6];
    const float line = fmaxf(tau, -FLT_MAX);   // (-inf is never listed)
    int n = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const bool hit = x[i] >= line;
        const u64 hits = __ballot(hit);
        if (hits) {
            const int more = n + __popcll(hits);
            if (more <= kListCap && hit)
                mine[n + __builtin_amdgcn_mbcnt_hi((uint32_t)(hits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hits, 0))] =
                    make_uint2(__float_as_uint(x[i]), c.index(i / c.kVec, lane) + i % c.kVec);
            n = more;
        }
    }
    if (n <= kListCap)
        for (int i = lane; i < n; i += 64) a.lists[place * kListCap + i] = mine[i];
    // ---- the weights, relative to the chunk's maximum
    double sum = 0.0;
    if (top > -INFINITY) {
        const RowFilter f = row_filter(a, row / a.block_k);
        if (wants_sum(f)) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) sum += weight(x[i], top, f.t);
            sum = wave_sum(sum);
        }
    }
    if (lane == 0) {
        ChunkStat r;
        r.sum = sum;
        r.top = top;
        r.tau = n <= kListCap ? tau : INFINITY;   // more equal ones than the list holds: nothing is listed
        r.count = n <= kListCap ? n : 0;
        a.stats[place] = r;
    }
}

// ---- cuts and token from the lists

constexpr int kPickThreads = 512, kPickWaves = kPickThreads / 64;
// Logits of a row's lists that are looked at, and of a row that has no scan: as many as leave room for four workgroups (all the waves
// a CU holds) in its LDS.  A row of 1792: 7.3 us in this one launch, 14.7 with a scan; 1024 such rows 23.6 and 50.8.  With room for
// 3584 (two workgroups) 1024 rows of 1792 take 28.1, 256 rows of 151936 113.2 instead of 112.6; with room for 1024 those take 119.
constexpr int kPickEntries = 1792;
constexpr int kMaxChunks = 1024, kChunksEach = kMaxChunks / kPickThreads;

__device__ __forceinline__ float key_logit(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }
__device__ __forceinline__ int bits_of(uint32_t v) { return v ? 32 - __clz(v) : 1; }

// The crossing of a running sum of amounts over n entries ordered by a number of `bits` bits, ten bits at a time.
struct Found {
    uint32_t number;
    u64 before, here;   // amounts of smaller numbers, of this one (0: never reached)
};
template <typename B, typename N, typename A>
__device__ __forceinline__ Found search_entries(B &bins, int tid, int threads, int n, int bits, u64 target, N number_of, A amount_of)
{
    static_assert(B::kCount >= 1024, "ten bits");
    Found r = {0, 0, 0};
#pragma unroll 1
    for (int shift = bits; shift > 0;) {
        const int next = max(0, shift - 10);
        for (int i = tid; i < n; i += threads) {
            const uint32_t d = number_of(i);
            if (shift >= 32 || d >> shift == r.number) {
                const u64 m = amount_of(i);
                if (m) atomicAdd(&bins.amount[(d >> next) & ((1u << (shift - next)) - 1)], m);
            }
        }
        const Crossing c = bins.crossing(tid, target - r.before);
        if (c.bin < 0) return {0, 0, 0};
        r.before += c.before;
        r.here = c.at;
        r.number = r.number << (shift - next) | (uint32_t)c.bin;
        shift = next;
    }
    return r;
}

constexpr int kFew = 64;   // so many logits are ranked one against the other, in the lanes of a wave

struct PickShared {
    Bins<kPickThreads, 2> bins;
    u64 mass[kPickEntries];
    uint32_t key[kPickEntries];
    int index[kPickEntries];
    ulonglong2 few[kFew];           // (order, weight)
    uint8_t listed[kMaxChunks];
    float top[kPickWaves], tau[kPickWaves];
    double z[kPickWaves];
    u64 before[kFew], run[kFew];   // of the few: weight of those in front by order, by index
    int rank[kFew];
    int count, few_count;
};

static_assert(sizeof(PickShared) <= 160 * 1024 / 4, "four workgroups to a CU");

// SCANNED: the row's chunks have been listed; else it has at most kPickEntries logits and is read here.
template <int DT, bool SCANNED, bool DRAW> __global__ void __launch_bounds__(kPickThreads, 4) filter_pick_kernel(const FilterArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int rr = stage_row(a, blockIdx.x), side = rr >= a.rows, row = rr - side * a.rows;
    if (rr < 0) return;
    __shared__ PickShared s;
    const RowFilter f = row_filter(a, row / a.block_k);
    const void *logits = logit_row<DT>(a, side, row);
    // ---- the row's maximum, down to where its lists hold everything
    float top = -INFINITY, tau = -INFINITY;
    ChunkStat st[kChunksEach];
    // A list to a wave; the loads of the first ones go out with those of the counts, which say later how much of them is one.
    constexpr int kAhead = 10;
    const uint2 *lists = a.lists + (int64_t)rr * a.chunks * kListCap;
    uint2 ahead[SCANNED ? kAhead : 1];
    if constexpr (SCANNED) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (wave + k * kPickWaves < a.chunks) ahead[k] = lists[(int64_t)(wave + k * kPickWaves) * kListCap + lane];
        const ChunkStat *stats = a.stats + (int64_t)rr * a.chunks;
#pragma unroll
        for (int i = 0; i < kChunksEach; ++i) {
            const int c = i * kPickThreads + tid;
            st[i] = {0.0, -INFINITY, -INFINITY, 0};
            if (c < a.chunks) st[i] = stats[c];
            s.listed[c] = (uint8_t)st[i].count;
            top = fmaxf(top, st[i].top);
            tau = fmaxf(tau, st[i].tau);
        }
    } else {
        for (int i = tid; i < a.vocab; i += kPickThreads) top = fmaxf(top, logit<DT>(logits, i));
    }
    top = wave_max(top);
    tau = wave_max(tau);
    if (lane == 0) { s.top[wave] = top; s.tau[wave] = tau; }
    if (tid == 0) s.count = s.few_count = 0;
    if (tid < kFew) { s.before[tid] = s.run[tid] = 0; s.rank[tid] = 0; }
    s.bins.clear(tid);
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) { top = fmaxf(top, s.top[w]); tau = fmaxf(tau, s.tau[w]); }
    RowCut cut = {0.0, top, (float)f.min_p, 0u, 0x7fffffff, 0};
    int token = -1;
    double own = 1.0;
    bool resolved = true;
    if (top > -INFINITY) {
        const bool plain = f.top_k == 0 && f.top_p >= 1.0 && f.min_p == 0.0;
        const float u = DRAW ? fminf(fmaxf(a.u[row], 0.f), 0x1.fffffep-1f) : 0.f;
        double part[kChunksEach], z = 0.0;   // the chunks' sums, relative to the row's maximum
        if constexpr (SCANNED) {
#pragma unroll
            for (int i = 0; i < kChunksEach; ++i) {
                part[i] = st[i].sum * weight(st[i].top, top, f.t);
                z += part[i];
            }
            z = wave_sum(z);
            if (lane == 0) s.z[wave] = z;
            __syncthreads();
            z = 0.0;
#pragma unroll
            for (int w = 0; w < kPickWaves; ++w) z += s.z[w];
        }
        if (SCANNED && plain) {
            // ---- no filter: the chunk at which the running sum crosses, and its logits once more
            cut.z = z;
            if constexpr (DRAW && SCANNED) {
                const double unit = exp2((double)min(50, 60 - ilogb(z)));
                u64 sum = 0;
#pragma unroll
                for (int i = 0; i < kChunksEach; ++i) {
                    // (A chunk none of whose logits has an amount of its own has none, whatever the sum of its weights:
                    // the chunk that the target falls into always holds a token to draw.)
                    const u64 m = to_fixed(weight(st[i].top, top, f.t), unit) ? to_fixed(part[i], unit) : 0;
                    s.bins.amount[i * kPickThreads + tid] = m;
                    sum += m;
                }
                const u64 total = s.bins.sum_of(tid, sum);
                const u64 target = (u64)((double)u * (double)total) + 1;
                const Crossing at = s.bins.crossing(tid, target);
                // 1024 bins, a few neighbours to each; a thread looks at logits 256 apart
                constexpr int kPerBin = kChunk / 1024, kPlaces = kChunk / kPickThreads;
                const int first = at.bin * kChunk - row_skew<DT>(logits);
                u64 m[kPlaces];
                int last = -1;
#pragma unroll
                for (int e = 0; e < kPlaces; ++e) {
                    const int i = first + e * kPickThreads + tid;
                    const float x = i >= 0 && i < a.vocab ? logit<DT>(logits, i) : -INFINITY;
                    m[e] = x > -INFINITY ? to_fixed(weight(x, top, f.t), unit) : 0;
                }
#pragma unroll
                for (int e = 0; e < kPlaces; ++e)
                    if (m[e]) {
                        last = e * kPickThreads + tid;
                        atomicAdd(&s.bins.amount[last / kPerBin], m[e]);
                    }
                const Crossing in = s.bins.crossing(tid, target - at.before);
                if (tid == 0) s.count = -1;
                __syncthreads();
                atomicMax(&s.count, last);
                __syncthreads();
                if (in.bin < 0) {   // the chunk's sum, rounded once, is more than that of its parts: its last token with an amount
                    token = s.count;
                } else {
#pragma unroll
                    for (int e = 0; e < kPlaces; ++e) {
                        const int place = e * kPickThreads + tid;
                        if (place / kPerBin == in.bin) s.bins.amount[place % kPerBin] = m[e];
                    }
                    token = in.bin * kPerBin + s.bins.crossing(tid, target - at.before - in.before).bin;
                }
                token += first;
                own = weight(logit<DT>(logits, token), top, f.t);
            }
        } else if (tau == INFINITY) {
            resolved = false;
        } else {
            // ---- every logit down to tau
            const bool whole = tau == -INFINITY;   // that is all there are
            const uint32_t top_key = order_key(top + 0.f);
            auto put = [&](int at, uint32_t x, int i) __attribute__((always_inline)) {   // (the logit's bits; its order later)
                s.key[at] = x;
                s.index[at] = i;
            };
            if constexpr (SCANNED) {
                for (int c0 = wave; c0 < a.chunks; c0 += kAhead * kPickWaves) {
                    if (c0 >= kAhead * kPickWaves) {
#pragma unroll
                        for (int k = 0; k < kAhead; ++k)
                            if (c0 + k * kPickWaves < a.chunks) ahead[k] = lists[(int64_t)(c0 + k * kPickWaves) * kListCap + lane];
                    }
                    bool hit[kAhead];
                    int count = 0, most = 0;
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) {
                        const int c = c0 + k * kPickWaves, have = c < a.chunks ? s.listed[c] : 0;
                        hit[k] = lane < have && __uint_as_float(ahead[k].x) >= tau;
                        count += __popcll(__ballot(hit[k]));
                        most = max(most, have);
                    }
                    int at = 0;
                    if (lane == 0) at = atomicAdd(&s.count, count);
                    at = __builtin_amdgcn_readfirstlane(at);
                    if (at + count <= kPickEntries) {
#pragma unroll
                        for (int k = 0; k < kAhead; ++k) {
                            const u64 hits = __ballot(hit[k]);
                            if (hit[k])
                                put(at + __builtin_amdgcn_mbcnt_hi((uint32_t)(hits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hits, 0)),
                                    ahead[k].x, (int)ahead[k].y);
                            at += __popcll(hits);
                        }
                    }
                    if (most > 64)
                        for (int k = 0; k < kAhead; ++k) {
                            const int c = c0 + k * kPickWaves, have = c < a.chunks ? s.listed[c] : 0;
                            for (int i = 64 + lane; i < have; i += 64) {
                                const uint2 w = lists[(int64_t)c * kListCap + i];
                                if (__uint_as_float(w.x) >= tau) {
                                    const int more = atomicAdd(&s.count, 1);
                                    if (more < kPickEntries) put(more, w.x, (int)w.y);
                                }
                            }
                        }
                }
            } else {
                for (int i = tid; i < a.vocab; i += kPickThreads) {
                    const float x = logit<DT>(logits, i);
                    if (x > -INFINITY) put(atomicAdd(&s.count, 1), __float_as_uint(x), i);
                }
            }
            __syncthreads();
            const int n = s.count;
            resolved = n <= kPickEntries;
            if (resolved) {
                constexpr double kUnit = 0x1p50;
                const int key_bits = bits_of(top_key - (whole ? order_key(-FLT_MAX) : order_key(tau + 0.f)));
                const int index_bits = bits_of((uint32_t)(a.vocab - 1)), coarse = max(0, key_bits - 10);
                auto fall_of = [&](int i) __attribute__((always_inline)) { return top_key - s.key[i]; };
                auto weight_of = [&](int i) __attribute__((always_inline)) { return weight(key_logit(s.key[i]), top, f.t); };
                u64 known = 0;
                for (int i = tid; i < n; i += kPickThreads) {
                    const float x = __uint_as_float(s.key[i]);
                    const u64 m = to_fixed(weight(x, top, f.t), kUnit);
                    s.key[i] = order_key(x + 0.f);
                    s.mass[i] = m;
                    known += m;
                }
                known = s.bins.sum_of(tid, known);
                // what min-p keeps is known if what is not listed is below its line; the other cuts are then only asked
                // whether they cut higher
                const bool min_p_known = whole || (f.min_p > 0.0 && weight(tau, top, f.t) < f.min_p);
                const bool by_k = f.top_k > 0 && f.top_k < n, top_k_known = f.top_k <= n || whole;
                const double all = f.top_k > 0 || whole ? (double)known : z * kUnit;   // (where top-k cuts nothing more)
                const double share = f.top_p < 1.0 && !by_k ? fmax(1.0, ceil(f.top_p * all)) : 0.0;
                const bool by_p = f.top_p < 1.0 && !by_k && share <= (double)known;
                if (f.top_p < 1.0) resolved = top_k_known && (by_k || by_p || min_p_known);
                else resolved = (f.top_k > 0 && top_k_known) || min_p_known;
                if (resolved) {
                    // ---- the few that can be kept: everything down to the step in which the first cut falls
                    int step = 1024;
                    if (by_k || by_p) {
                        for (int i = tid; i < n; i += kPickThreads) atomicAdd(&s.bins.amount[fall_of(i) >> coarse], by_k ? 1ull : s.mass[i]);
                        step = s.bins.crossing(tid, by_k ? (u64)f.top_k : min(known, (u64)share)).bin;
                    }
                    const bool by_m = !by_k && !by_p && f.min_p > 0.0;
                    for (int i = tid; i < n; i += kPickThreads)
                        if ((int)(fall_of(i) >> coarse) <= step && !(by_m && !(weight_of(i) >= f.min_p))) {
                            const int at = atomicAdd(&s.few_count, 1);
                            if (at < kFew) s.few[at] = make_ulonglong2((u64)s.key[i] << 32 | (uint32_t)~s.index[i], s.mass[i]);
                        }
                    __syncthreads();
                    const int m = s.few_count;
                    u64 total;
                    if (m <= kFew) {
                        // every wave has them all in its lanes and compares them with an eighth of them
                        const ulonglong2 e = lane < m ? s.few[lane] : make_ulonglong2(0, 0);
                        const uint32_t key = (uint32_t)(e.x >> 32);
                        const int index = (int)~(uint32_t)e.x;
                        u64 before = 0;
                        int rank = 0;
                        for (int i = wave; i < m; i += kPickWaves) {
                            const u64 w = lane_value(e.y, i);
                            if (lane_value(e.x, i) > e.x) { before += w; ++rank; }
                        }
                        if (lane < m) { atomicAdd(&s.before[lane], before); atomicAdd(&s.rank[lane], rank); }
                        __syncthreads();
                        before = s.before[lane];
                        rank = s.rank[lane];
                        bool in = lane < m && (!by_k || rank < f.top_k);
                        if (f.top_p < 1.0) {
                            const double z1 = by_k ? (double)wave_sum(in ? e.y : (u64)0) : all;
                            in = in && (double)before < fmax(1.0, ceil(f.top_p * z1));
                        }
                        const u64 mine = in && (f.min_p == 0.0 || weight(key_logit(key), top, f.t) >= f.min_p) ? e.y : 0;
                        total = wave_sum(mine);
                        if constexpr (DRAW) {
                            const u64 target = (u64)((double)u * (double)total) + 1;
                            u64 run = 0;
                            for (int i = wave; i < m; i += kPickWaves) {
                                const u64 w = lane_value(mine, i);
                                if (__builtin_amdgcn_readlane(index, i) < index) run += w;
                            }
                            if (lane < m) atomicAdd(&s.run[lane], run);
                            __syncthreads();
                            run = s.run[lane];
                            const int from = __ffsll((long long)__ballot(run < target && target <= run + mine)) - 1;
                            token = __builtin_amdgcn_readlane(index, from);
                            own = weight(key_logit((uint32_t)__builtin_amdgcn_readlane((int)key, from)), top, f.t);
                        } else {
                            // those in front, up to the last that both cuts leave: the first so many of the order
                            const int last = __popcll(__ballot(in)) - 1;
                            const int from = __ffsll((long long)__ballot(in && rank == last)) - 1;
                            cut.key = (uint32_t)__builtin_amdgcn_readlane((int)key, from);
                            cut.tie = __builtin_amdgcn_readlane(index, from);
                            if constexpr (SCANNED) {
                                const u64 keeps = __ballot(mine != 0);
                                cut.listed = __popcll(keeps);
                                if (wave == 0 && mine)
                                    a.lists[(int64_t)rr * a.chunks * kListCap +
                                            __builtin_amdgcn_mbcnt_hi((uint32_t)(keeps >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)keeps, 0))] =
                                        make_uint2(__float_as_uint(key_logit(key)), index);
                            }
                        }
                        cut.z = (double)total / kUnit;
                    } else {
                        // ---- many: the same cuts digit by digit
                        auto index_of = [&](int i) __attribute__((always_inline)) { return (uint32_t)s.index[i]; };
                        auto mass_of = [&](int i) __attribute__((always_inline)) { return s.mass[i]; };
                        uint32_t cut_fall = 0xffffffffu;
                        int cut_tie = 0x7fffffff;
                        auto cut_at = [&](const Found &c, u64 nth, u64 here) __attribute__((always_inline)) {
                            if (c.number < cut_fall) cut_tie = 0x7fffffff;
                            cut_fall = c.number;
                            if (nth < here)   // not all of those at the cut's logit: the n-th of them by index
                                cut_tie = min(cut_tie, (int)search_entries(s.bins, tid, kPickThreads, n, index_bits, nth, index_of,
                                                                           [&](int i) __attribute__((always_inline)) { return (u64)(fall_of(i) == cut_fall); }).number);
                            u64 sum = 0;
                            for (int i = tid; i < n; i += kPickThreads) {
                                const uint32_t d = fall_of(i);
                                if (d > cut_fall || (d == cut_fall && s.index[i] > cut_tie)) s.mass[i] = 0;
                                sum += s.mass[i];
                            }
                            return s.bins.sum_of(tid, sum);
                        };
                        double z1 = all;
                        if (by_k) {
                            const Found k = search_entries(s.bins, tid, kPickThreads, n, key_bits, (u64)f.top_k, fall_of,
                                                           [&](int) __attribute__((always_inline)) { return (u64)1; });
                            known = cut_at(k, (u64)f.top_k - k.before, k.here);
                            z1 = (double)known;
                        }
                        if (by_p || (by_k && f.top_p < 1.0)) {
                            const u64 goal = min(known, (u64)fmax(1.0, ceil(f.top_p * z1)));
                            const Found p = search_entries(s.bins, tid, kPickThreads, n, key_bits, goal, fall_of, mass_of);
                            const u64 each = to_fixed(weight(key_logit(top_key - p.number), top, f.t), kUnit);
                            cut_at(p, (goal - p.before + each - 1) / each, p.here / each);
                        }
                        u64 sum = 0;
                        for (int i = tid; i < n; i += kPickThreads) {
                            if (f.min_p > 0.0 && !(weight_of(i) >= f.min_p)) s.mass[i] = 0;
                            sum += s.mass[i];
                        }
                        total = s.bins.sum_of(tid, sum);
                        cut.z = (double)total / kUnit;
                        // (no cut among the listed ones, of which top-k may keep all: nothing below them is kept)
                        cut.key = cut_fall != 0xffffffffu ? top_key - cut_fall : whole ? 0u : order_key(tau + 0.f);
                        cut.tie = cut_tie;
                        if constexpr (DRAW) {
                            token = (int)search_entries(s.bins, tid, kPickThreads, n, index_bits, (u64)((double)u * (double)total) + 1,
                                                        index_of, mass_of).number;
                            own = weight(logit<DT>(logits, token), top, f.t);
                        } else if constexpr (SCANNED) {
                            if (tid == 0) s.count = 0;
                            __syncthreads();
                            for (int i = tid; i < n; i += kPickThreads)
                                if (s.mass[i])
                                    a.lists[(int64_t)rr * a.chunks * kListCap + atomicAdd(&s.count, 1)] =
                                        make_uint2(__float_as_uint(key_logit(s.key[i])), s.index[i]);
                            __syncthreads();
                            cut.listed = s.count;
                        }
                    }
                }
            }
        }
    }
    if (tid == 0) {
        if (!resolved) {
            a.unresolved[1 + atomicAdd(a.unresolved, 1)] = rr;
        } else if (DRAW) {
            a.tokens[row] = token;
            if (a.logprobs) a.logprobs[row] = token < 0 ? -INFINITY : (float)log(own / cut.z);
        } else {
            a.cuts[rr] = cut;
        }
    }
}

// ---- rows whose cut lies below the lists

// (A workgroup to each such row, the others leave at once: with a loop over the rows the compiler kept 80 registers more alive,
// for half the waves.)

// A whole row in the hands of a workgroup, read in blocks: a wave takes a block of 512 vectors, eight loads at a time, so
// that a block's sum is one reduction.  Cuts are found by a histogram over 4096 steps of the logit (a hundredth of a
// binade of the weight each) and then among the logits of one step, gathered in the second pass, which also sums what lies
// above them; steps that hold more logits than the gather has room for (rows of equal logits) go digit by digit.
constexpr int kWideThreads = 1024, kWideWaves = kWideThreads / 64;
constexpr int kWideEntries = 4096;
constexpr int kSteps = 4096, kMaxBlocks = 520;   // of 2048 logits (or 4096): 2^20 and what a row's start takes

struct WideShared {
    Bins<kWideThreads, 2> bins;
    Bins<kWideThreads, (kSteps + kWideThreads - 1) / kWideThreads> steps;
    u64 block[kMaxBlocks];
    u64 mass[kWideEntries];
    uint32_t key[kWideEntries];
    int index[kWideEntries];
    float top[kWideWaves], tau[kWideWaves];
    double z[kWideWaves];
    int count;
};

template <int DT> struct WideRow {
    static constexpr int kVec = Vector<DT>::kCount, kBlock = 512 * kVec;
    WideShared &s;
    const void *row;
    int vocab, skew, blocks, tid;
    float top, step_scale;       // step of a logit: (top - x) * step_scale
    Scale t;
    double unit;                 // fixed-point value of the weight 1
    RowCut cut;

    __device__ __forceinline__ double weight_of(float x) const { return weight(x, top, t); }
    __device__ __forceinline__ u64 mass_of(float x) const { return to_fixed(weight_of(x), unit); }
    __device__ __forceinline__ int step_of(float x) const { return (int)fminf((top - x) * step_scale, (float)(kSteps - 1)); }
    // weight of what the cut and min-p keep
    __device__ __forceinline__ u64 kept_mass(float x, int i) const
    {
        const double w = weight_of(x);
        return kept(cut, x, i) && w >= (double)cut.min_w ? to_fixed(w, unit) : 0;
    }

    // visit(x, index) for every logit of the wave's block, two vectors ahead of it.
    template <typename F> __device__ __forceinline__ void block_logits(int blk, F visit)
    {
        const int lane = tid & 63, first = (blk * 512 + lane) * kVec - skew;
        auto load = [&](int u) __attribute__((always_inline)) {
            const int i = first + u * 64 * kVec;
            uint4 q = make_uint4(0, 0, 0, 0);
            if (u < 8 && i >= 0 && i + kVec <= vocab) q = *(const uint4 *)((const char *)row + (int64_t)i * (16 / kVec));
            return q;
        };
        uint4 q0 = load(0), q1 = load(1);
#pragma unroll 1
        for (int u = 0; u < 8; ++u) {
            const uint4 q = q0;
            q0 = q1;
            q1 = load(u + 2);
            const int i = first + u * 64 * kVec;
            if (i >= 0 && i + kVec <= vocab) {
                float x[kVec];
                unpack<DT>(q, x);
#pragma unroll
                for (int r = 0; r < kVec; ++r) visit(clean_logit(x[r]), i + r);
            } else {
#pragma unroll 1
                for (int r = 0; r < kVec; ++r)
                    if (i + r >= 0 && i + r < vocab) visit(logit<DT>(row, i + r), i + r);
            }
        }
    }
    template <typename F> __device__ __forceinline__ void each_logit(F visit)
    {
        for (int blk = tid >> 6; blk < blocks; blk += kWideWaves) block_logits(blk, visit);
    }

    // s.block[]: the sums of amount_at(x, index) over the blocks; returns their sum.
    template <typename F> __device__ __forceinline__ u64 sum_blocks(F amount_at)
    {
        __syncthreads();
        u64 all = 0;
        for (int blk = tid >> 6; blk < blocks; blk += kWideWaves) {
            u64 sum = 0;
            block_logits(blk, [&](float x, int i) __attribute__((always_inline)) { sum += amount_at(x, i); });
            all += sum;
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
            if ((tid & 63) == 0) s.block[blk] = sum;
        }
        return s.bins.sum_of(tid, all);
    }

    // With s.block[] made of amount_at: the first index at which the running sum reaches the target (-1: none).
    template <typename F> __device__ __forceinline__ int find_in_blocks(u64 target, F amount_at)
    {
        static_assert(kMaxBlocks <= 2 * kWideThreads, "two blocks to a thread at most");
        __syncthreads();
        const u64 b0 = 2 * tid < blocks ? s.block[2 * tid] : 0, b1 = 2 * tid + 1 < blocks ? s.block[2 * tid + 1] : 0;
        s.bins.amount[2 * tid] = b0;
        s.bins.amount[2 * tid + 1] = b1;
        const Crossing at = s.bins.crossing(tid, target);
        if (at.bin < 0) return -1;
        // the block's 512 vectors, one to a thread
        const int first = tid < 512 ? (at.bin * 512 + tid) * kVec - skew : vocab;
        u64 part[kVec], sum = 0;
#pragma unroll
        for (int r = 0; r < kVec; ++r) {
            const int i = first + r;
            part[r] = i >= 0 && i < vocab ? amount_at(logit<DT>(row, i), i) : 0;
            sum += part[r];
        }
        s.bins.amount[tid] = sum;
        const Crossing in = s.bins.crossing(tid, target - at.before);
        if (tid == in.bin) {
            u64 run = at.before + in.before;
            int found = -1;
#pragma unroll
            for (int r = 0; r < kVec; ++r) {
                run += part[r];
                if (found < 0 && run >= target) found = first + r;
            }
            s.count = found;
        }
        __syncthreads();
        const int found = in.bin < 0 ? -1 : s.count;
        __syncthreads();
        return found;
    }

    __device__ __forceinline__ int nth_of_key(uint32_t key, u64 n)
    {
        auto there = [&](float x, int) __attribute__((always_inline)) { return (u64)(order_key(x) == key); };
        sum_blocks(there);
        const int i = find_in_blocks(n, there);
        return i < 0 ? 0x7fffffff : i;
    }

    struct Selected {
        uint32_t key;
        u64 above, here;  // amounts above the logit, at it (0: never reached)
    };

    // The logit at which a sum in falling order reaches the target, digit by digit.
    template <bool MASS> __device__ __forceinline__ Selected select_digits(u64 target)
    {
        Selected r = {0, 0, 0};
        uint32_t prefix = 0;
#pragma unroll 1
        for (int shift = 32; shift > 0;) {
            const int next = max(0, shift - 12);
            each_logit([&](float x, int) __attribute__((always_inline)) {
                const uint32_t fall = ~order_key(x);
                if (x > -INFINITY && (shift == 32 || fall >> shift == prefix))
                    atomicAdd(&s.steps.amount[(fall >> next) & ((1u << (shift - next)) - 1)], MASS ? mass_of(x) : 1ull);
            });
            const Crossing c = s.steps.crossing(tid, target - r.above);
            if (c.bin < 0) return {0, 0, 0};
            r.above += c.before;
            r.here = c.at;
            prefix = prefix << (shift - next) | (uint32_t)c.bin;
            shift = next;
        }
        r.key = ~prefix;
        return r;
    }

    // Cuts where the sum in falling order (MASS: of weights, else of ones) reaches the target.  `summed`: s.block[] then holds
    // the kept weights, else it does not.  Returns the weight of what is kept without regard to min-p (0: not known).
    // The first pass's weights are single precision (they only say which step to gather); the second's sums say whether it was
    // the right one.
    template <bool MASS> __device__ __forceinline__ u64 cut_at(u64 target, bool &summed)
    {
        summed = false;
        const float rate = (float)t.scale;
        each_logit([&](float x, int) __attribute__((always_inline)) {
            if (x > -INFINITY)
                atomicAdd(&s.steps.amount[step_of(x)],
                          MASS ? (u64)(uint32_t)(__builtin_amdgcn_exp2f((x - top) * rate) * 0x1p31f) : 1ull);
        });
        const double goal1 = MASS ? (double)target * (0x1p31 / unit) : (double)target;
        const Crossing c = s.steps.crossing(tid, max((u64)1, (u64)goal1));
        if (!MASS && c.bin < 0) return 0;   // everything together does not reach it: no cut
        int step = c.bin < 0 ? kSteps - 1 : c.bin;
        const double min_w = (double)cut.min_w;
        u64 over, at_step = 0;   // weight of the steps above, of this one
        int n;
#pragma unroll 1
        for (int round = 0;; ++round) {
            if (tid == 0) s.count = 0;
            __syncthreads();
            over = 0;
            u64 here = 0;
            sum_blocks([&](float x, int i) __attribute__((always_inline)) {
                const int st = x > -INFINITY ? step_of(x) : kSteps;
                u64 m = 0;
                if (st <= step) {
                    const double w = weight_of(x);
                    m = to_fixed(w, unit);
                    if (st == step) {
                        here += m;
                        m = 0;
                        const int at = atomicAdd(&s.count, 1);
                        if (at < kWideEntries) { s.key[at] = order_key(x); s.index[at] = i; }
                    } else {
                        over += m;
                        if (!(w >= min_w)) m = 0;
                    }
                }
                return m;
            });
            over = s.bins.sum_of(tid, over);
            n = s.count;
            if (!MASS) break;
            at_step = s.bins.sum_of(tid, here);
            // (the rounding of single precision can miss by a step or two)
            const int other = target <= over ? step - 1 : target > over + at_step ? step + 1 : step;
            if (other == step || other < 0 || other >= kSteps || round == 8) break;
            step = other;
        }
        __syncthreads();
        if (MASS && target > over + at_step && step == kSteps - 1) return 0;   // all of it does not reach the target: no cut
        if (n > kWideEntries || (MASS && (target <= over || target > over + at_step))) {
            const Selected r = select_digits<MASS>(target);
            if (r.here == 0) return 0;
            const u64 each = MASS ? mass_of(key_logit(r.key)) : 1;
            const u64 nth = (target - r.above + each - 1) / each;
            if (r.key > cut.key) cut.tie = 0x7fffffff;
            cut.key = r.key;
            if (nth * each < r.here) cut.tie = min(cut.tie, nth_of_key(r.key, nth));
            return 0;
        }
        // ---- among the gathered logits
        for (int i = tid; i < n; i += kWideThreads) s.mass[i] = mass_of(key_logit(s.key[i]));
        const u64 goal = target - (MASS ? over : c.before);
        const Found r = search_entries(s.bins, tid, kWideThreads, n, 32, goal, [&](int i) __attribute__((always_inline)) { return ~s.key[i]; },
                                       [&](int i) __attribute__((always_inline)) { return MASS ? s.mass[i] : 1ull; });
        if (r.here == 0) return 0;
        const uint32_t key = ~r.number;
        const u64 each = MASS ? mass_of(key_logit(key)) : 1;
        const u64 nth = (goal - r.before + each - 1) / each;
        if (key > cut.key) cut.tie = 0x7fffffff;
        cut.key = key;
        if (nth * each < r.here)
            cut.tie = min(cut.tie, (int)search_entries(s.bins, tid, kWideThreads, n, bits_of((uint32_t)(vocab - 1)), nth,
                                                       [&](int i) __attribute__((always_inline)) { return (uint32_t)s.index[i]; },
                                                       [&](int i) __attribute__((always_inline)) { return (u64)(s.key[i] == key); }).number);
        u64 more = 0;
        for (int i = tid; i < n; i += kWideThreads) {
            const float x = key_logit(s.key[i]);
            const int index = s.index[i];
            if (kept(cut, x, index)) {
                more += s.mass[i];
                if (weight_of(x) >= min_w) atomicAdd(&s.block[(index + skew) / kBlock], s.mass[i]);
            }
        }
        summed = true;
        return over + s.bins.sum_of(tid, more);
    }

};

template <int DT, bool DRAW> __global__ void __launch_bounds__(kWideThreads, 4) filter_wide_kernel(const FilterArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, count = a.unresolved[0];
    if ((int)blockIdx.x >= count) return;
    __shared__ WideShared s;
    s.bins.clear(tid);
    s.steps.clear(tid);
    const int rr = a.unresolved[1 + blockIdx.x], side = rr >= a.rows, row = rr - side * a.rows;
    const RowFilter f = row_filter(a, row / a.block_k);
    const ChunkStat *stats = a.stats + (int64_t)rr * a.chunks;
    float top = -INFINITY, tau = INFINITY;
    for (int c = tid; c < a.chunks; c += kWideThreads) { top = fmaxf(top, stats[c].top); tau = fminf(tau, stats[c].tau); }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) { top = fmaxf(top, __shfl_xor(top, off)); tau = fminf(tau, __shfl_xor(tau, off)); }
    if (lane == 0) { s.top[wave] = top; s.tau[wave] = tau; }
    __syncthreads();
    for (int w = 0; w < kWideWaves; ++w) { top = fmaxf(top, s.top[w]); tau = fminf(tau, s.tau[w]); }
    double z = 0.0;
    for (int c = tid; c < a.chunks; c += kWideThreads) z += stats[c].sum * weight(stats[c].top, top, f.t);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) z += __shfl_xor(z, off);
    if (lane == 0) s.z[wave] = z;
    __syncthreads();
    z = 0.0;
    for (int w = 0; w < kWideWaves; ++w) z += s.z[w];
    const void *logits = logit_row<DT>(a, side, row);
    const int skew = row_skew<DT>(logits);
    // fixed point: the sum of all weights (at most one each) stays below 2^61
    const double unit = uniform(exp2((double)min(50, z >= 1.0 ? 60 - ilogb(z) : 60 - bits_of((uint32_t)a.vocab))));
    top = uniform(top);
    WideRow<DT> r = {s, logits, a.vocab, skew, (a.vocab + skew + WideRow<DT>::kBlock - 1) / WideRow<DT>::kBlock, tid, top,
                     uniform((float)(f.t.scale * (kSteps / 40.0))), {uniform(f.t.scale), uniform(f.t.floor)}, unit, {0.0, top, (float)f.min_p, 0u, 0x7fffffff, 0}};
    bool summed = false;
    u64 z1 = 0;
    if (f.top_k > 0) {
        // steps that reach well below the lists' logits, whatever the temperature
        const float by_weight = r.step_scale;
        if (top - tau > 0.f && top - tau < INFINITY) r.step_scale = kSteps / (8.f * (top - tau));
        z1 = r.template cut_at<false>((u64)f.top_k, summed);
        r.step_scale = by_weight;
    } else if (f.top_p < 1.0) {
        z1 = (u64)(z * unit);
    }
    if (f.top_p < 1.0) {
        const float min_w = r.cut.min_w;
        if (z1 == 0) {
            r.cut.min_w = 0.f;
            z1 = r.sum_blocks([&](float x, int i) __attribute__((always_inline)) { return r.kept_mass(x, i); });
            r.cut.min_w = min_w;
        }
        r.template cut_at<true>(max((u64)1, (u64)ceil(f.top_p * (double)z1)), summed);
    }
    auto amount = [&](float x, int i) __attribute__((always_inline)) { return r.kept_mass(x, i); };
    u64 total;
    if (summed) {
        __syncthreads();
        u64 part = 0;
        for (int blk = tid; blk < r.blocks; blk += kWideThreads) part += s.block[blk];
        total = s.bins.sum_of(tid, part);
    } else {
        total = r.sum_blocks(amount);
    }
    r.cut.z = (double)total / unit;
    int token = -1;
    if (DRAW) {
        const float u = fminf(fmaxf(a.u[row], 0.f), 0x1.fffffep-1f);
        token = r.find_in_blocks((u64)((double)u * (double)total) + 1, amount);
    }
    if (tid == 0) {
        if (DRAW) {
            a.tokens[row] = token;
            if (a.logprobs) a.logprobs[row] = token < 0 ? -INFINITY : (float)log(r.weight_of(logit<DT>(logits, token)) / r.cut.z);
        } else {
            a.cuts[rr] = r.cut;
        }
    }
}

// ---- launch plan: chunk size, workspace

struct FilterPlan {
    int chunks;   // 0: no scan
    size_t stats, lists, unresolved, total;   // byte offsets
};

static FilterPlan filter_plan(int64_t rows, int vocab)   // rows of all views
{
    FilterPlan p = {};
    if (vocab <= kPickEntries) return p;
    p.chunks = (vocab + 7 + kChunk - 1) / kChunk;   // (a row may start seven logits behind a boundary)
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    p.lists = up((size_t)rows * p.chunks * sizeof(ChunkStat));
    p.unresolved = p.lists + up((size_t)rows * p.chunks * kListCap * sizeof(uint2));
    p.total = p.unresolved + up((size_t)(rows + 1) * sizeof(int32_t));
    return p;
}

// A launch counts its threads in 32 bits.
bool filter_fits(int64_t rows, int vocab, int views)
{
    const int64_t all = rows * views;
    return all * kWideThreads < 0xffffffffll && (all * filter_plan(1, vocab).chunks + 4) * 64 < 0xffffffffll;
}
size_t filter_workspace_bytes(int64_t rows, int vocab, int views) { return filter_plan(rows * views, vocab).total; }

// Logits of more than this leave nothing behind in the last-level cache that a later kernel of the call would find.
constexpr int64_t kKeepBytes = (int64_t)192 << 20;

template <int DT, bool DRAW> static hipError_t launch_filters_of(const FilterArgs &a, hipStream_t stream)
{
    if (a.chunks == 0) {
        hipLaunchKernelGGL((filter_pick_kernel<DT, false, DRAW>), dim3(a.all_rows), dim3(kPickThreads), 0, stream, a);
        return hipGetLastError();
    }
    const dim3 scan((unsigned)(((int64_t)a.all_rows * a.chunks + 3) / 4));
    if ((int64_t)a.all_rows * a.vocab * (DT == 0 ? 4 : 2) > kKeepBytes)
        hipLaunchKernelGGL((filter_scan_kernel<DT, true>), scan, dim3(kScanThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((filter_scan_kernel<DT, false>), scan, dim3(kScanThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((filter_pick_kernel<DT, true, DRAW>), dim3(a.all_rows), dim3(kPickThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((filter_wide_kernel<DT, DRAW>), dim3(a.all_rows), dim3(kWideThreads), 0, stream, a);
    return hipGetLastError();
}

template <bool DRAW> static hipError_t launch_filters(const FilterArgs &a, hipStream_t stream)
{
    if (a.dtype == 0) return launch_filters_of<0, DRAW>(a, stream);
    if (a.dtype == 1) return launch_filters_of<1, DRAW>(a, stream);
    return launch_filters_of<2, DRAW>(a, stream);
}

// Lays out the workspace for all rows of `views` views.
static void place_workspace(FilterArgs &a, int views)
{
    const FilterPlan p = filter_plan((int64_t)a.rows * views, a.vocab);
    char *ws = (char *)a.workspace;
    a.stats = (ChunkStat *)(ws + p.stats);
    a.lists = (uint2 *)(ws + p.lists);
    a.unresolved = (int32_t *)(ws + p.unresolved);
    a.chunks = p.chunks;
}

// Block rows k0 .. k1-1 of every sequence and view.
static void set_stage(FilterArgs &a, int views, int k0, int k1)
{
    a.first_k = k0;
    a.stage_k = k1 - k0;
    a.stage_rows = a.rows / a.block_k * a.stage_k;
    a.all_rows = a.stage_rows * views;
}

hipError_t launch_sample_tokens(FilterArgs a, hipStream_t stream)
{
    place_workspace(a, 1);
    set_stage(a, 1, 0, a.block_k);
    a.decided = nullptr;
    return launch_filters<true>(a, stream);
}

// ---- consensus

constexpr int kDrawThreads = 512, kDrawPiece = 8192;

// Probability that a row's filters leave a token (0: cut, or an empty row).
__device__ __forceinline__ double kept_prob(const RowCut &c, double inv_z, const Scale &t, float x, int i)
{
    if (!kept(c, x, i)) return 0.0;
    const double d = (double)x - (double)c.top, w = d <= t.floor ? 0.0 : weight(d, t);
    return w >= (double)c.min_w ? w * inv_z : 0.0;
}

struct Candidate {
    double score;
    int index;
    __device__ __forceinline__ void take(double v, int i)
    {
        if (v > score || (v == score && i < index)) { score = v; index = i; }
    }
};

template <int DT> __device__ __forceinline__ bool keeps_draft(const FilteredArgs &a, const Scale &t, int row)
{
    const int x = a.c.draft_tokens[row];
    const RowCut cp = a.f.cuts[row], cq = a.f.cuts[a.f.rows + row];
    const float u = a.accept_u[row];
    if (x < 0 || x >= a.c.vocab) return false;
    const float xp = logit<DT>(logit_row<DT>(a.f, 0, row), x), xq = logit<DT>(logit_row<DT>(a.f, 1, row), x);
    return (double)u * kept_prob(cq, 1.0 / cq.z, t, xq, x) < kept_prob(cp, 1.0 / cp.z, t, xp, x);
}

// Between two stages: a wave per sequence, the leading drafts of the first `rows` that are kept.
template <int DT> __global__ void __launch_bounds__(64) filtered_stage_kernel(const FilteredArgs a, int rows)
{
    const int b = blockIdx.x, k = threadIdx.x;
    const Scale t = row_filter(a.f, b).t;
    const bool keep = k >= rows || keeps_draft<DT>(a, t, b * a.c.block_k + k);
    const u64 lost = ~__ballot(keep);
    if (k == 0) a.c.decided[b] = lost ? __ffsll((long long)lost) - 1 : rows;
}

// Grid (piece, sequence).  Every workgroup repeats the keep decisions of its sequence (three dependent round trips), the first
// records them.  The first rejected row's kept tokens are in the row's lists, which the first workgroup goes through, or
// anywhere (no filter, a wide cut): then each goes through its piece of the row.
template <int DT> __global__ void __launch_bounds__(kDrawThreads) filtered_draw_kernel(const FilteredArgs a)
{
    const int b = blockIdx.y, piece = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int K = a.c.block_k, V = a.c.vocab;
    const Scale t = row_filter(a.f, b).t;
    __shared__ int s_keep[32];
    __shared__ Candidate s_best[2][kDrawThreads / 64];
    // (rows behind a lost one may not have been looked at: what is found for them does not matter)
    if (tid < K) s_keep[tid] = keeps_draft<DT>(a, t, b * K + tid);
    __syncthreads();
    const unsigned long long rej = ~__ballot(lane >= K || s_keep[lane < K ? lane : 0]);
    const int j = rej ? __ffsll((long long)rej) - 1 : K;
    if (piece == 0 && tid == 0) {
        a.c.decided[b] = j;
        if (a.c.do_commit) commit_snapshot(a.c, b);
    }
    if (j >= K) return;
    const int row = b * K + j;
    const void *pr = logit_row<DT>(a.f, 0, row), *qr = logit_row<DT>(a.f, 1, row);
    const RowCut cp = a.f.cuts[row], cq = a.f.cuts[a.f.rows + row];
    const float *gr = a.gumbel + (int64_t)b * V;
    const double inv_p = 1.0 / cp.z, inv_q = 1.0 / cq.z;
    Candidate more = {-INFINITY, 0x7fffffff}, any = {-INFINITY, 0x7fffffff};  // best among p > q, best of p
    float more_near = -INFINITY, any_near = -INFINITY;   // single precision: the full logarithm only for what comes near the best
    auto visit = [&](float xp, float xq, float g, int i) __attribute__((always_inline)) {
        const double p = kept_prob(cp, inv_p, t, xp, i);
        if (p > 0.0) {
            const double q = kept_prob(cq, inv_q, t, xq, i), r = p - q;
            auto consider = [&](double v, float &near, Candidate &best) __attribute__((always_inline)) {
                const float f = (float)v, score = __logf(f) + g;
                if (!(score < near - 0.01f) || f < 1e-30f) {
                    best.take(log(v) + (double)g, i);
                    near = fmaxf(near, score);
                }
            };
            if (r > 0.0) consider(r, more_near, more);
            else if (more_near == -INFINITY) consider(p, any_near, any);   // (asked for only where nothing is positive)
        }
    };
    if (!cp.listed) {
        const int end = min(V, (piece + 1) * kDrawPiece);
        constexpr int kAtOnce = 8;
        for (int i0 = piece * kDrawPiece; i0 < end; i0 += kAtOnce * kDrawThreads) {   // (the same rounds for all lanes)
            float x[kAtOnce], y[kAtOnce], g[kAtOnce];
#pragma unroll
            for (int e = 0; e < kAtOnce; ++e) {
                const int i = i0 + e * kDrawThreads + tid;
                x[e] = i < end ? logit<DT>(pr, i) : -INFINITY;
                y[e] = i < end ? logit<DT>(qr, i) : -INFINITY;
                g[e] = i < end ? gr[i] : 0.f;
            }
#pragma unroll 1
            for (int e = 0; e < kAtOnce; ++e) {   // (one copy of the visit; what it needs moves down by one)
                visit(x[0], y[0], g[0], i0 + e * kDrawThreads + tid);
#pragma unroll
                for (int r = 0; r + 1 < kAtOnce; ++r) { x[r] = x[r + 1]; y[r] = y[r + 1]; g[r] = g[r + 1]; }
                more_near = wave_max(more_near);
            }
            any_near = wave_max(any_near);
        }
    } else if (piece == 0) {
        const uint2 *list = a.f.lists + (int64_t)row * a.f.chunks * kListCap;
        for (int at = tid; at < cp.listed; at += kDrawThreads) {
            const uint2 v = list[at];
            visit(__uint_as_float(v.x), logit<DT>(qr, (int)v.y), gr[v.y], (int)v.y);
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
        for (int w = 1; w < kDrawThreads / 64; ++w) {
            more.take(s_best[0][w].score, s_best[0][w].index);
            any.take(s_best[1][w].score, s_best[1][w].index);
        }
        a.best[(int64_t)b * gridDim.x + piece] = {more.score, any.score, more.index, any.index};
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
            Candidate more = {-INFINITY, 0x7fffffff}, any = {-INFINITY, 0x7fffffff};
            if (j < K) {
                for (int i = lane; i < a.pieces; i += 64) {
                    const DrawBest d = a.best[(int64_t)b * a.pieces + i];
                    more.take(d.more, d.more_index);
                    any.take(d.any, d.any_index);
                }
#pragma unroll
                for (int off = 32; off >= 1; off >>= 1) {
                    const double v0 = __shfl_xor(more.score, off), v1 = __shfl_xor(any.score, off);
                    const int i0 = __shfl_xor(more.index, off), i1 = __shfl_xor(any.index, off);
                    more.take(v0, i0);
                    any.take(v1, i1);
                }
            }
            const int repl = more.index != 0x7fffffff ? more.index : any.index != 0x7fffffff ? any.index : -1;
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

int draw_pieces(int vocab) { return (vocab + kDrawPiece - 1) / kDrawPiece; }

// Logits that take long to go through are gone through in two stages, the second for the sequences that kept every draft of the
// first.  With a share r of drafts kept and 16 rows, 6 + 10 r^6 of them are read: 7 at r = 0.7, 10 at 0.85, 13 at 0.95; the second
// stage's four launches take 12 us, what a third of kKeepBytes takes to read.  (64 x 16 rows of 151936, r about 0.9: 336 us in one
// stage.)
static int first_stage(const FilterArgs &a)
{
    const int64_t bytes = (int64_t)a.rows * 2 * a.vocab * (a.dtype == 0 ? 4 : 2);
    return a.chunks > 0 && a.block_k >= 4 && bytes > kKeepBytes ? (3 * a.block_k + 7) / 8 : a.block_k;
}

template <int DT> static hipError_t launch_filtered_of(FilteredArgs &a, hipStream_t stream)
{
    const ConsensusArgs &c = a.c;
    const int k1 = first_stage(a.f);
    set_stage(a.f, 2, 0, k1);
    hipError_t e = launch_filters_of<DT, false>(a.f, stream);
    if (e != hipSuccess) return e;
    if (k1 < c.block_k) {
        hipLaunchKernelGGL((filtered_stage_kernel<DT>), dim3(c.batch), dim3(64), 0, stream, a, k1);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        set_stage(a.f, 2, k1, c.block_k);
        a.f.decided = c.decided;
        e = launch_filters_of<DT, false>(a.f, stream);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((filtered_draw_kernel<DT>), dim3((unsigned)a.pieces, (unsigned)c.batch), dim3(kDrawThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(filtered_commit_kernel, dim3(c.batch, c.do_commit ? c.num_layers : 1), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_filtered_consensus(FilteredArgs a, hipStream_t stream)
{
    place_workspace(a.f, 2);
    a.f.decided = nullptr;
    if (a.f.dtype == 0) return launch_filtered_of<0>(a, stream);
    if (a.f.dtype == 1) return launch_filtered_of<1>(a, stream);
    return launch_filtered_of<2>(a, stream);
}

}  // namespace orthrus
