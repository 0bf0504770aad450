// Page tables, slot maps and the store of packed K/V rows on gfx950: what a serving loop does between requests and the
// attention, on the device, so that consecutive steps queue without a round trip to the host.
//
//   tables_count_kernel  one workgroup per sequence: how many pages it lacks (or returns), and where the first lies.
//   tables_scan_kernel   one workgroup: running sums over the sequences of pages and tokens, who is granted what, the ring's
//                        new state.  The ring's old state is kept for the next kernel.
//   tables_apply_kernel  grid (sequence, strip): page-table entries, the ring's new tail, the slots of the new tokens.  An
//                        entry's page follows from its place alone (entries that lack a page are almost always the last
//                        ones of the range), so strips need nothing from each other; a range with holes goes to one
//                        workgroup.  Pages come from the head of the ring and go back to its tail: nothing that this
//                        kernel reads there is written by it.
//   tables_small_kernel  the three of them in one workgroup, for small batches.
//   kv_store_kernel      grid (rows, layer): 16-byte chunks, four of K and of V in flight per thread.
#include "orthrus_internal.h"
#include "orthrus_lanes.h"

namespace orthrus {

constexpr int kBadSequence = INT32_MIN;

__device__ __forceinline__ bool is_mapped(const TablesArgs &a, int page) { return page >= 0 && page < a.num_pages; }

// The entries a sequence's call is about: [first, last].
struct EntryRange {
    int first, last;
};
__device__ __forceinline__ EntryRange entry_range(const TablesArgs &a, int L, int n)
{
    if (n < 0) return {0, a.max_pages_per_seq - 1};
    return {L >> a.page_shift, n > 0 ? (L + n - 1) >> a.page_shift : (L >> a.page_shift) - 1};
}

// By `threads` threads of which this is the tid-th (a wave or a workgroup); `sum_up` makes what they found one.
template <typename F> __device__ __forceinline__ void count_sequence(const TablesArgs &a, int b, int tid, int threads, F sum_up)
{
    const int L = a.seq_lens[b], n = a.new_lens[b];
    bool bad = n >= 0 && (L < 0 || (int64_t)L + n > a.max_seq_len);
    int count = 0, first = INT32_MAX, last = -1;
    EntryRange r = {0, -1};
    if (!bad) {
        const int32_t *row = a.page_table + (int64_t)b * a.max_pages_per_seq;
        r = entry_range(a, L, n);
        // ended: mapped entries, else unmapped ones; four loads in flight
        for (int e0 = r.first + tid; e0 <= r.last; e0 += 4 * threads) {
            int page[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) page[u] = row[min(e0 + u * threads, r.last)];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int e = e0 + u * threads;
                if (e <= r.last && is_mapped(a, page[u]) == (n < 0)) { ++count; first = min(first, e); last = e; }
            }
        }
    }
    sum_up(count, first, last);
    // the page of tokens that are cached already must be there
    if (n > 0 && (L & ((1 << a.page_shift) - 1)) && first == r.first) bad = true;
    if (tid == 0) {
        a.need[b] = bad ? kBadSequence : n < 0 ? -1 - count : count;
        // entry of the first; -1 - entry: those behind it are not all alike (up to the last new token's entry, where it grows)
        const bool whole = last - first + 1 == count && (n < 0 || last == r.last);
        a.first[b] = count == 0 ? INT32_MAX : whole ? first : -1 - first;
    }
}

__device__ __forceinline__ void wave_sum_up(int &count, int &first, int &last)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        count += __shfl_xor(count, off);
        first = min(first, __shfl_xor(first, off));
        last = max(last, __shfl_xor(last, off));
    }
}

__global__ void __launch_bounds__(256) tables_count_kernel(const TablesArgs a)
{
    const int tid = threadIdx.x;
    __shared__ int s_count, s_first, s_last;
    if (tid == 0) { s_count = 0; s_first = INT32_MAX; s_last = -1; }
    __syncthreads();
    count_sequence(a, blockIdx.x, tid, blockDim.x, [&](int &count, int &first, int &last) __attribute__((always_inline)) {
        wave_sum_up(count, first, last);
        if ((tid & 63) == 0 && count) { atomicAdd(&s_count, count); atomicMin(&s_first, first); atomicMax(&s_last, last); }
        __syncthreads();
        count = s_count; first = s_first; last = s_last;
    });
}

constexpr int kScanThreads = 1024;

struct Pair {
    int64_t a, b;
};
__device__ __forceinline__ int64_t last_lane(int64_t v)
{
    return (int64_t)lane_value((u64)v, 63);
}
// Running sums of two numbers over the threads, in their order: `up to` a thread and `all` of them.
struct WaveSums {   // 64 threads
    __device__ __forceinline__ void operator()(Pair v, Pair &upto, Pair &all)
    {
        upto = {(int64_t)wave_scan((u64)v.a), (int64_t)wave_scan((u64)v.b)};
        all = {last_lane(upto.a), last_lane(upto.b)};
    }
    __device__ __forceinline__ int64_t most(int64_t v)
    {
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) v = max(v, (int64_t)__shfl_xor((long long)v, off));
        return v;
    }
};
struct BlockSums {   // kScanThreads of them; contains barriers
    Pair *sums;
    int64_t *top;
    __device__ __forceinline__ void operator()(Pair v, Pair &upto, Pair &all)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        upto = {(int64_t)wave_scan((u64)v.a), (int64_t)wave_scan((u64)v.b)};
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        const Pair w = lane < kScanThreads / 64 ? sums[lane] : Pair{0, 0};
        upto.a += (int64_t)wave_sum(lane < wave ? (u64)w.a : (u64)0);
        upto.b += (int64_t)wave_sum(lane < wave ? (u64)w.b : (u64)0);
        all = {(int64_t)wave_sum((u64)w.a), (int64_t)wave_sum((u64)w.b)};
        __syncthreads();
    }
    __device__ __forceinline__ int64_t most(int64_t v)
    {
        if (threadIdx.x == 0) *top = 0;
        __syncthreads();
        if (v > 0) atomicMax((long long *)top, (long long)v);
        __syncthreads();
        return *top;
    }
};

// Who is granted what: a thread to a run of neighbouring sequences.  The pages that granted sequences take are those that
// they and all before them want (a sequence that wants any is granted only if all of those are there).
template <typename S> __device__ __forceinline__ void scan_sequences(const TablesArgs &a, int tid, int threads, S sums)
{
    const int N = (int)a.num_pages;
    int head = a.free_state[0];
    if (head < 0 || head >= N) head = head % N + (head % N < 0 ? N : 0);
    const int free = min(max(a.free_state[1], 0), N);
    const int each = (a.batch + threads - 1) / threads;
    const int b0 = min(tid * each, a.batch), b1 = min(b0 + each, a.batch);
    Pair sum = {0, 0}, run, all;   // pages wanted, returned
    for (int b = b0; b < b1; ++b) {
        const int need = a.need[b];
        if (need >= 0) sum.a += need;
        else if (need != kBadSequence) sum.b += -1 - (int64_t)need;
    }
    sums(sum, run, all);
    const int64_t all_returned = all.b;
    int64_t wanted = run.a - sum.a, returned = run.b - sum.b, tokens = 0, taken = 0;
    bool error = false;
    for (int b = b0; b < b1; ++b) {
        const int need = a.need[b], n = a.new_lens[b];
        if (need >= 0) wanted += need;
        const bool granted = n >= 0 && need >= 0 && (need == 0 || wanted <= free);
        if (granted && need > 0) taken = wanted;
        error |= n >= 0 && !granted;
        a.granted[b] = granted ? n : 0;
        a.pages_before[b] = (int32_t)(need >= 0 ? min(wanted - need, (int64_t)INT32_MAX) : min(returned, (int64_t)INT32_MAX));
        if (need < 0 && need != kBadSequence) returned += -1 - (int64_t)need;
        tokens += granted ? n : 0;
    }
    sums({tokens, 0}, run, all);
    int64_t start = run.a - tokens;
    for (int b = b0; b < b1; ++b) {
        a.token_starts[b] = (int32_t)min(start, (int64_t)INT32_MAX);
        start += a.granted[b];
    }
    taken = sums.most(taken);
    error |= all_returned > N - free || all.a > a.max_tokens;
    if (error) atomicExch(a.err_word, -4);
    if (tid == 0) {
        const int64_t next = head + taken;   // (at most `free` pages are taken)
        a.token_starts[a.batch] = (int32_t)min(all.a, (int64_t)INT32_MAX);
        a.ring_before[0] = head;
        a.ring_before[1] = free;
        a.free_state[0] = (int32_t)(next < N ? next : next - N);
        a.free_state[1] = (int32_t)(free - taken + min(all_returned, (int64_t)(N - free)));
    }
}

// (WAVE: for a few hundred sequences one wave, which waits for nobody, is the faster.)
template <bool WAVE> __global__ void __launch_bounds__(kScanThreads) tables_scan_kernel(const TablesArgs a)
{
    if constexpr (WAVE) {
        scan_sequences(a, threadIdx.x, 64, WaveSums());
    } else {
        __shared__ Pair s_sums[kScanThreads / 64];
        __shared__ int64_t s_top;
        scan_sequences(a, threadIdx.x, kScanThreads, BlockSums{s_sums, &s_top});
    }
}

// What a sequence's entries and slots are made from.
struct Sequence {
    int32_t *row;
    int L, n, need, first;
    int64_t before;          // pages taken (returned) by the sequences before it
    int head, free, pages;   // the ring before the call

    __device__ __forceinline__ Sequence(const TablesArgs &a, int b)
        : row(a.page_table + (int64_t)b * a.max_pages_per_seq), L(a.seq_lens[b]), n(a.new_lens[b]), need(a.need[b]), first(a.first[b]),
          before(a.pages_before[b]), head(a.ring_before[0]), free(a.ring_before[1]), pages((int)a.num_pages)
    {
        if (need == kBadSequence) n = 0;
        else if (n > 0) n = a.granted[b];
    }
    __device__ __forceinline__ bool holes() const { return first < 0; }
    __device__ __forceinline__ int place(int64_t at) const   // at < 2 * pages - head
    {
        const int64_t p = head + at;
        return (int)(p < pages ? p : p - pages);
    }
    __device__ __forceinline__ void give_back(const TablesArgs &a, int64_t at, int page) const
    {
        if (at < pages - free) a.free_pages[place(free + at)] = page;
    }
};

// A range with holes, by one wave: entries in order, 64 at a time.
__device__ __forceinline__ void apply_ordered(const TablesArgs &a, const Sequence &s, int lane)
{
    const EntryRange r = entry_range(a, s.L, s.n);
    int64_t before = s.before;
    for (int e0 = r.first; e0 <= r.last; e0 += 64) {
        const int e = e0 + lane, page = e <= r.last ? s.row[e] : 0;
        const bool hit = e <= r.last && is_mapped(a, page) == (s.n < 0);
        const u64 hits = __ballot(hit);
        if (hit) {
            const int64_t at = before + __popcll(hits & ((1ull << lane) - 1));
            if (s.n >= 0) s.row[e] = a.free_pages[s.place(at)];
            else { s.give_back(a, at, page); s.row[e] = -1; }
        }
        before += __popcll(hits);
    }
}

// Slot of token i of a granted sequence, and its entry where the token is the entry's first.  (Ranges with holes: the entries
// are there.)
__device__ __forceinline__ bool apply_token(const TablesArgs &a, const Sequence &s, int i, int64_t slot_at)
{
    const int pos = s.L + i, e = pos >> a.page_shift, off = pos & ((1 << a.page_shift) - 1);
    int page;
    if (!s.holes() && e >= s.first) {
        page = a.free_pages[s.place(s.before + (e - s.first))];
        if (off == 0) s.row[e] = page;
    } else {
        page = s.row[e];
    }
    const bool ok = is_mapped(a, page);   // (the ring may hold anything)
    a.slot_map[slot_at] = ok ? (page << a.page_shift) + off : -1;
    return ok;
}

// The entries that a granted sequence without holes lacked: for calls whose tokens do not all have a slot.
__device__ __forceinline__ void apply_entries(const TablesArgs &a, const Sequence &s, int from, int step)
{
    const int last = (s.L + s.n - 1) >> a.page_shift;
    if (s.need > 0 && !s.holes())
        for (int e = s.first + from; e <= last; e += step) s.row[e] = a.free_pages[s.place(s.before + (e - s.first))];
}

__device__ __forceinline__ void return_pages(const TablesArgs &a, const Sequence &s, int from, int step)
{
    const int count = -1 - s.need;
    for (int i = from; i < count; i += step) {
        s.give_back(a, s.before + i, s.row[s.first + i]);
        s.row[s.first + i] = -1;
    }
}

__global__ void __launch_bounds__(256) tables_apply_kernel(const TablesArgs a)
{
    const int b = blockIdx.x, strip = blockIdx.y, strips = gridDim.y, tid = threadIdx.x;
    const Sequence s(a, b);
    if (s.n == 0 || (s.holes() && strip > 0)) return;
    if (s.holes()) {
        if (tid < 64) apply_ordered(a, s, tid);
        __syncthreads();  // (the entries are read below by other threads of this workgroup)
    }
    if (s.n < 0) {
        if (!s.holes()) return_pages(a, s, strip * 256 + tid, strips * 256);
        return;
    }
    bool error = false;
    const int step = s.holes() ? 256 : strips * 256;
    // Tokens behind the last slot are not gone through (there may be 2^31 of them): their entries are, and the scan has
    // reported them.
    const int64_t start = a.token_starts[b], slots = min((int64_t)s.n, a.max_tokens - start);
    if (slots < s.n) apply_entries(a, s, strip * 256 + tid, strips * 256);
    for (int64_t i = strip * 256 + tid; i < slots; i += step) error |= !apply_token(a, s, (int)i, start + i);
    if (error) atomicExch(a.err_word, -4);
}

// All three in one workgroup, for few sequences with few new tokens.  What the steps hand to each other stays in LDS; the
// sequences are counted side by side, 1024 / batch threads to each.  In microseconds, against the three launches, each with 7 of
// a copy that puts the tables back: 256 sequences of 16 tokens 13 and 18, of 32 17 and 18, of 64 23 and 18; one of 4096 tokens 12 and
// 18, of 16384 19 and 18.  Rows of ended requests are walked over whole: 256 rows of 256 entries take 13 where none is full, but 33
// where every fifth is and its request over (18): they end once in hundreds of steps.
constexpr int kSmallBatch = 256, kSmallTokens = 4096, kSmallEntries = 65536;

__global__ void __launch_bounds__(kScanThreads) tables_small_kernel(const TablesArgs g)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    __shared__ int s_len[kSmallBatch], s_new[kSmallBatch], s_need[kSmallBatch], s_first[kSmallBatch], s_before[kSmallBatch],
        s_granted[kSmallBatch], s_start[kSmallBatch + 1], s_ring[2];
    TablesArgs a = g;
    a.seq_lens = s_len; a.new_lens = s_new;
    a.need = s_need; a.first = s_first; a.pages_before = s_before; a.granted = s_granted; a.token_starts = s_start; a.ring_before = s_ring;
    for (int b = tid; b < a.batch; b += kScanThreads) { s_len[b] = g.seq_lens[b]; s_new[b] = g.new_lens[b]; }
    __syncthreads();
    int threads = 64;
    while (threads * a.batch > kScanThreads) threads >>= 1;
    const int own = tid / threads, sub = tid & (threads - 1);
    if (own < a.batch)
        count_sequence(a, own, sub, threads, [&](int &count, int &first, int &last) __attribute__((always_inline)) {
            for (int off = threads / 2; off >= 1; off >>= 1) {
                count += __shfl_xor(count, off);
                first = min(first, __shfl_xor(first, off));
                last = max(last, __shfl_xor(last, off));
            }
        });
    __syncthreads();
    if (wave == 0) scan_sequences(a, lane, 64, WaveSums());
    __syncthreads();
    if (own < a.batch && s_first[own] >= 0 && s_new[own] < 0) return_pages(a, Sequence(a, own), sub, threads);
    for (int b = wave; b < a.batch; b += kScanThreads / 64)
        if (s_first[b] < 0) {
            const Sequence s(a, b);
            if (s.n != 0) apply_ordered(a, s, lane);
        }
    for (int b = tid; b <= a.batch; b += kScanThreads) {
        g.token_starts[b] = s_start[b];
        if (b < a.batch) g.granted[b] = s_granted[b];
    }
    __syncthreads();
    bool error = false;
    const int tokens = (int)min((int64_t)s_start[a.batch], a.max_tokens);   // (as in tables_apply_kernel)
    if (tokens < s_start[a.batch])
        for (int b = wave; b < a.batch; b += kScanThreads / 64) {
            const Sequence s(a, b);
            if (s.n > 0) apply_entries(a, s, lane, 64);
        }
    for (int t = tid; t < tokens; t += kScanThreads) {
        int b = 0;   // the last sequence that starts at t or before, which is the one that holds it
#pragma unroll
        for (int half = kSmallBatch / 2; half >= 1; half >>= 1)
            if (b + half < a.batch && s_start[b + half] <= t) b += half;
        const Sequence s(a, b);
        error |= !apply_token(a, s, t - s_start[b], t);
    }
    if (error) atomicExch(a.err_word, -4);
}

hipError_t launch_page_tables(const TablesArgs &a, hipStream_t stream)
{
    hipError_t e = hipSuccess;
    if (a.batch > 0 && a.batch <= kSmallBatch && a.max_tokens <= kSmallTokens &&
        (int64_t)a.batch * a.max_pages_per_seq <= kSmallEntries) {
        hipLaunchKernelGGL(tables_small_kernel, dim3(1), dim3(kScanThreads), 0, stream, a);
        return hipGetLastError();
    }
    if (a.batch > 0) {
        hipLaunchKernelGGL(tables_count_kernel, dim3(a.batch), dim3(a.batch > 1024 ? 64 : 256), 0, stream, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.batch <= kSmallBatch) hipLaunchKernelGGL((tables_scan_kernel<true>), dim3(1), dim3(64), 0, stream, a);
    else hipLaunchKernelGGL((tables_scan_kernel<false>), dim3(1), dim3(kScanThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess || a.batch == 0) return e;
    const int64_t most = a.max_tokens > a.max_pages_per_seq ? a.max_tokens : a.max_pages_per_seq;
    // A strip to 256 tokens, up to 2048 workgroups, as many as the chip holds at once: 48 sequences of 30000 tokens and 4 of 300000
    // take the same within a microsecond with 1024 and 4096.
    int64_t strips = (most + 255) / 256;
    if (strips > 2048 / a.batch) strips = 2048 / a.batch;
    hipLaunchKernelGGL(tables_apply_kernel, dim3(a.batch, strips > 1 ? (unsigned)strips : 1u), dim3(256), 0, stream, a);
    return hipGetLastError();
}

// ---- the store

constexpr int kStoreChunks = 1024;  // 16-byte chunks of K (and as many of V) per workgroup, where rows are that short

__global__ void __launch_bounds__(256) kv_store_kernel(const StoreArgs a, int rows_per_wg)
{
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    const int tid = threadIdx.x, layer = blockIdx.y;
    const int64_t row0 = (int64_t)blockIdx.x * rows_per_wg;
    int valid = a.rows;
    if (a.num_valid) valid = min(max(*a.num_valid, 0), a.rows);
    if (row0 >= valid) return;
    const int rows = (int)min((int64_t)rows_per_wg, valid - row0);
    const int cpr = a.head_dim / 8, per_tok = a.num_kv_heads * cpr, total = rows * per_tok;
    const int64_t slots = a.num_pages << a.page_shift;
    const uint16_t *ks = a.k_new + layer * a.blk_stride_layer + row0 * a.blk_stride_row;
    const uint16_t *vs = a.v_new + layer * a.blk_stride_layer + row0 * a.blk_stride_row;
    bool error = false;
    for (int e0 = tid; e0 < total; e0 += 4 * 256) {
        u32x4 k[4], v[4];
        int64_t dst[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int e = min(e0 + u * 256, total - 1);  // (past the end: the last chunk again, not stored)
            const int t = e / per_tok, rem = e - t * per_tok, g = rem / cpr, ch = rem - g * cpr;
            const int slot = a.slot_map[row0 + t];
            const int64_t src = t * a.blk_stride_row + g * a.blk_stride_head + ch * 8;
            const bool ok = slot >= 0 && slot < slots;
            error |= slot >= 0 && !ok;
            dst[u] = !ok ? -1 : layer * a.stride_layer + (int64_t)(slot >> a.page_shift) * a.stride_page + g * a.stride_head +
                                (int64_t)(slot & ((1 << a.page_shift) - 1)) * a.stride_tok + ch * 8;
            k[u] = *(const u32x4 *)(ks + src);
            v[u] = *(const u32x4 *)(vs + src);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (e0 + u * 256 < total && dst[u] >= 0) {
                *(u32x4 *)(a.k_pool + dst[u]) = k[u];
                *(u32x4 *)(a.v_pool + dst[u]) = v[u];
            }
    }
    if (error) atomicExch(a.err_word, -4);
}

static int store_rows_per_wg(int num_kv_heads, int head_dim)
{
    const int per_tok = num_kv_heads * (head_dim / 8);
    return per_tok >= kStoreChunks ? 1 : kStoreChunks / per_tok;
}

// A launch counts its threads in 32 bits.
bool kv_store_fits(int rows, int num_kv_heads, int head_dim)
{
    const int rows_per_wg = store_rows_per_wg(num_kv_heads, head_dim);
    return ((int64_t)rows + rows_per_wg - 1) / rows_per_wg * 256 < 0xffffffffll;
}

hipError_t launch_kv_store(const StoreArgs &a, hipStream_t stream)
{
    const int rows_per_wg = store_rows_per_wg(a.num_kv_heads, a.head_dim);
    const dim3 grid((unsigned)(((int64_t)a.rows + rows_per_wg - 1) / rows_per_wg), (unsigned)a.num_layers);
    hipLaunchKernelGGL(kv_store_kernel, grid, dim3(256), 0, stream, a, rows_per_wg);
    return hipGetLastError();
}

}  // namespace orthrus
