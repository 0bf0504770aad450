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
//   kv_store_kernel      grid (rows, layer): 16-byte chunks, four of K and of V in flight per thread.
#include "orthrus_internal.h"

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

__global__ void __launch_bounds__(256) tables_count_kernel(const TablesArgs a)
{
    const int b = blockIdx.x, tid = threadIdx.x;
    const int L = a.seq_lens[b], n = a.new_lens[b];
    __shared__ int s_count, s_first, s_last;
    if (tid == 0) { s_count = 0; s_first = INT32_MAX; s_last = -1; }
    __syncthreads();
    bool bad = n >= 0 && (L < 0 || (int64_t)L + n > a.max_seq_len);
    if (!bad) {
        const int32_t *row = a.page_table + (int64_t)b * a.max_pages_per_seq;
        const EntryRange r = entry_range(a, L, n);
        // ended: mapped entries, else unmapped ones
        int count = 0, first = INT32_MAX, last = -1;
        for (int e = r.first + tid; e <= r.last; e += blockDim.x)
            if (is_mapped(a, row[e]) == (n < 0)) { ++count; first = min(first, e); last = e; }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) {
            count += __shfl_xor(count, off);
            first = min(first, __shfl_xor(first, off));
            last = max(last, __shfl_xor(last, off));
        }
        if ((tid & 63) == 0 && count) { atomicAdd(&s_count, count); atomicMin(&s_first, first); atomicMax(&s_last, last); }
        __syncthreads();
        // the page of tokens that are cached already must be there
        if (n > 0 && (L & ((1 << a.page_shift) - 1)) && s_first == r.first) bad = true;
    }
    if (tid == 0) {
        a.need[b] = bad ? kBadSequence : n < 0 ? -1 - s_count : s_count;
        // entry of the first; -1 - entry: those behind it are not all alike (up to the last new token's entry, where it grows)
        const bool whole = s_last - s_first + 1 == s_count && (n < 0 || s_last == entry_range(a, L, n).last);
        a.first[b] = s_count == 0 ? INT32_MAX : whole ? s_first : -1 - s_first;
    }
}

constexpr int kScanThreads = 1024;

// Inclusive sum over a workgroup, in thread order.  Contains barriers.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t *sums, int tid)
{
    const int lane = tid & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t o = __shfl_up((long long)v, off);
        if (lane >= off) v += o;
    }
    __syncthreads();
    if (lane == 63) sums[tid >> 6] = v;
    __syncthreads();
    for (int w = 0; w < (tid >> 6); ++w) v += sums[w];
    return v;
}

__global__ void __launch_bounds__(kScanThreads) tables_scan_kernel(const TablesArgs a)
{
    const int tid = threadIdx.x;
    __shared__ int64_t sums[kScanThreads / 64];
    __shared__ int64_t s_carry[4];  // pages wanted, taken, returned; tokens
    const int64_t N = a.num_pages;
    const int64_t head = ((int64_t)a.free_state[0] % N + N) % N;
    const int64_t free = min(max((int64_t)a.free_state[1], (int64_t)0), N);
    if (tid < 4) s_carry[tid] = 0;
    bool error = false;
    for (int b0 = 0; b0 < a.batch; b0 += kScanThreads) {
        const int b = b0 + tid;
        const int need = b < a.batch ? a.need[b] : 0, n = b < a.batch ? a.new_lens[b] : 0;
        const bool bad = need == kBadSequence;
        const int64_t lacks = bad || need < 0 ? 0 : need, back = bad || need >= 0 ? 0 : -1 - (int64_t)need;
        __syncthreads();
        const int64_t wanted0 = s_carry[0], taken0 = s_carry[1], back0 = s_carry[2], tokens0 = s_carry[3];
        const int64_t wanted = wanted0 + block_scan(lacks, sums, tid);
        const bool granted = n >= 0 && !bad && (lacks == 0 || wanted <= free);
        const int64_t taken = taken0 + block_scan(granted ? lacks : 0, sums, tid);
        const int64_t returned = back0 + block_scan(back, sums, tid);
        const int64_t tokens = tokens0 + block_scan(granted ? n : 0, sums, tid);
        error |= (n >= 0 && !granted && b < a.batch) || returned > N - free || tokens > a.max_tokens;
        if (b < a.batch) {
            a.granted[b] = granted ? n : 0;
            a.token_starts[b] = (int32_t)min(tokens - (granted ? n : 0), (int64_t)INT32_MAX);
            a.pages_before[b] = (int32_t)(need < 0 ? min(returned - back, (int64_t)INT32_MAX) : taken - (granted ? lacks : 0));
        }
        __syncthreads();
        if (tid == kScanThreads - 1) { s_carry[0] = wanted; s_carry[1] = taken; s_carry[2] = returned; s_carry[3] = tokens; }
    }
    __syncthreads();
    if (__syncthreads_or(error) && tid == 0) atomicExch(a.err_word, -4);
    if (tid == 0) {
        a.token_starts[a.batch] = (int32_t)min(s_carry[3], (int64_t)INT32_MAX);
        a.ring_before[0] = (int32_t)head;
        a.ring_before[1] = (int32_t)free;
        a.free_state[0] = (int32_t)((head + s_carry[1]) % N);
        a.free_state[1] = (int32_t)(free - s_carry[1] + min(s_carry[2], N - free));
    }
}

// A range with holes, by one workgroup: entries in order, 256 at a time.
__device__ __forceinline__ void apply_ordered(const TablesArgs &a, int b, int tid, int L, int n, int64_t head, int64_t free)
{
    __shared__ int s_wave[4];
    int32_t *row = a.page_table + (int64_t)b * a.max_pages_per_seq;
    const EntryRange r = entry_range(a, L, n);
    int64_t before = a.pages_before[b];
    for (int e0 = r.first; e0 <= r.last; e0 += 256) {
        const int e = e0 + tid, page = e <= r.last ? row[e] : 0;
        const bool hit = e <= r.last && is_mapped(a, page) == (n < 0);
        const unsigned long long mask = __ballot(hit);
        __syncthreads();
        if ((tid & 63) == 0) s_wave[tid >> 6] = __popcll(mask);
        __syncthreads();
        int rank = __popcll(mask & ((1ull << (tid & 63)) - 1)), total = 0;
        for (int w = 0; w < 4; ++w) { rank += w < (tid >> 6) ? s_wave[w] : 0; total += s_wave[w]; }
        if (hit) {
            const int64_t at = before + rank;
            if (n >= 0) row[e] = a.free_pages[(head + at) % a.num_pages];
            else {
                if (at < a.num_pages - free) a.free_pages[(head + free + at) % a.num_pages] = page;
                row[e] = -1;
            }
        }
        before += total;
    }
    __syncthreads();  // (the entries are read below by other threads of this workgroup)
}

__global__ void __launch_bounds__(256) tables_apply_kernel(const TablesArgs a)
{
    const int b = blockIdx.x, strip = blockIdx.y, strips = gridDim.y, tid = threadIdx.x;
    const int need = a.need[b], L = a.seq_lens[b], first = a.first[b];
    int n = a.new_lens[b];
    if (need == kBadSequence) return;
    const int64_t head = a.ring_before[0], free = a.ring_before[1], N = a.num_pages;
    int32_t *row = a.page_table + (int64_t)b * a.max_pages_per_seq;
    const bool holes = first < 0;
    if (holes && strip > 0) return;
    const int64_t before = a.pages_before[b];
    if (n < 0) {
        if (holes) { apply_ordered(a, b, tid, L, n, head, free); return; }
        const int count = -1 - need;
        for (int i = strip * 256 + tid; i < count; i += strips * 256) {
            const int page = row[first + i];
            if (before + i < N - free) a.free_pages[(head + free + before + i) % N] = page;
            row[first + i] = -1;
        }
        return;
    }
    n = a.granted[b];
    if (n == 0) return;
    if (holes) apply_ordered(a, b, tid, L, n, head, free);
    const int step = holes ? 256 : strips * 256, start = a.token_starts[b];
    bool error = false;
    for (int i = (holes ? 0 : strip * 256) + tid; i < n; i += step) {
        const int pos = L + i, e = pos >> a.page_shift, off = pos & ((1 << a.page_shift) - 1);
        int page;
        if (!holes && e >= first) {
            page = a.free_pages[(head + before + (e - first)) % N];
            if (off == 0 || i == 0) row[e] = page;
        } else {
            page = row[e];
        }
        const bool ok = is_mapped(a, page);   // (the ring may hold anything)
        error |= !ok;
        if ((int64_t)start + i < a.max_tokens) a.slot_map[start + i] = ok ? (page << a.page_shift) + off : -1;
    }
    if (error) atomicExch(a.err_word, -4);
}

hipError_t launch_page_tables(const TablesArgs &a, hipStream_t stream)
{
    hipError_t e = hipSuccess;
    if (a.batch > 0) {
        hipLaunchKernelGGL(tables_count_kernel, dim3(a.batch), dim3(a.batch > 1024 ? 64 : 256), 0, stream, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(tables_scan_kernel, dim3(1), dim3(kScanThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess || a.batch == 0) return e;
    const int64_t most = a.max_tokens > a.max_pages_per_seq ? a.max_tokens : a.max_pages_per_seq;
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

hipError_t launch_kv_store(const StoreArgs &a, hipStream_t stream)
{
    const int per_tok = a.num_kv_heads * (a.head_dim / 8);
    const int rows_per_wg = per_tok >= kStoreChunks ? 1 : kStoreChunks / per_tok;
    const dim3 grid((unsigned)(((int64_t)a.rows + rows_per_wg - 1) / rows_per_wg), (unsigned)a.num_layers);
    hipLaunchKernelGGL(kv_store_kernel, grid, dim3(256), 0, stream, a, rows_per_wg);
    return hipGetLastError();
}

}  // namespace orthrus
