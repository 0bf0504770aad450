// Greedy consensus of a tree of drafts and the commit of its path (the consensus rule of Section 3.3, Eq. 8, with several drafts
// for a position): from the root down, node after node, to the child whose token is the node's largest logit.
//
// Only the logits rows on the path decide anything, and which those are is known one at a time.
//   walk   a launch per level: every workgroup of a sequence finds the level's node for itself, from the chunk maxima of the
//          level before, the children and their tokens, and takes the maximum of its own chunk of that node's row.
//   all    one launch over every node's row, where that is less than a launch per level.
//   commit grid (sequence, layer): finishes the path, writes tokens and lengths (layer 0) and copies its rows' K/V.
// What bounds it: 64 sequences the logits of their paths (177 MB, 25 us at the memory's rate; 51 with eight levels, 7 to 9 us where
// rows are read and 3 where every path is over), fewer of them the chain of launches (batch 1: scan 4, commit 6).
#include "orthrus_internal.h"
#include "orthrus_lanes.h"

#include <type_traits>

namespace orthrus {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

// A logit and its place as one number whose order is that of the candidates: NaN above everything, then by value (both zeros
// alike), among equals the lower index.  0 stands for no candidate.
__device__ __forceinline__ u64 argmax_key(float v, int index)
{
    uint32_t u = __float_as_uint(v);
    u = u == 0x80000000u ? 0u : u;
    u = v != v ? 0xffffffffu : (u >> 31) ? ~u : u | 0x80000000u;
    return (u64)u << 32 | (uint32_t)~index;
}
// The token of a row's largest key: its index, or kNothing where the row holds nothing but -inf, as a mask that allows no token leaves
// it.  No child has that token, so the path ends there.
constexpr int kNothing = -1;
__device__ __forceinline__ int key_token(u64 key) { return (uint32_t)(key >> 32) == ~0xff800000u ? kNothing : (int)~(uint32_t)key; }

__device__ __forceinline__ u64 larger(u64 x, u64 y) { return x > y ? x : y; }
__device__ __forceinline__ u64 wave_largest(u64 x)
{
    x = larger(x, swap_u64<kSwap1>(x));
    x = larger(x, swap_u64<kSwap2>(x));
    x = larger(x, swap_u64<kMirror8>(x));
    x = larger(x, swap_u64<kMirror16>(x));
    x = larger(x, __shfl_xor(x, 16));
    return larger(x, __shfl_xor(x, 32));
}

template <int DTYPE>
__device__ __forceinline__ float logit_of(uint32_t bits)
{
    if constexpr (DTYPE == 0) return __uint_as_float(bits);
    else if constexpr (DTYPE == 1) return __uint_as_float(bits << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

// The largest logit of elements [begin, begin + CE) of a row of V, as every thread of the workgroup's first wave has it.
template <int DTYPE, int CE>
__device__ __forceinline__ u64 chunk_max(const void *row, int begin, int V)
{
    using T = std::conditional_t<DTYPE == 0, uint32_t, uint16_t>;
    constexpr int VEC = 16 / sizeof(T), NL = CE / (256 * VEC);
    static_assert(NL * 256 * VEC == CE, "");
    const int tid = threadIdx.x, end = min(V, begin + CE);
    const T *base = (const T *)row;
    // the 16-byte aligned middle, every load before the first comparison, and what is left on either side, an element to a thread
    const int head = min((int)((0 - ((uintptr_t)(base + begin) / sizeof(T))) & (VEC - 1)), end - begin);
    const int mid = begin + head, nvec = (end - mid) / VEC, tail = mid + nvec * VEC;
    u32x4_t x[NL];
    constexpr uint32_t kLow = DTYPE == 0 ? 0xff800000u : DTYPE == 1 ? 0xff80ff80u : 0xfc00fc00u;  // -inf
#pragma unroll
    for (int u = 0; u < NL; ++u) {
        x[u] = u32x4_t{kLow, kLow, kLow, kLow};
        if (u * 256 + tid < nvec)  // read once, never again: do not let the row displace anything in the caches
            x[u] = __builtin_nontemporal_load((const u32x4_t *)(base + mid) + u * 256 + tid);
    }
    const int edge = tid < VEC ? (tid < head ? begin + tid : end) : tid < 2 * VEC ? tail + tid - VEC : end;
    u64 best = edge < end ? argmax_key(logit_of<DTYPE>(base[edge]), edge) : 0ull;
    // a thread's own candidates come in the order of their index: a later one only wins by more, and nothing wins over a NaN
    // (nor does the -inf behind the end win over the first)
    float bv = 0.f;
    int bi = -1;
#pragma unroll
    for (int u = 0; u < NL; ++u) {
        const int i = mid + (u * 256 + tid) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float v = logit_of<DTYPE>(sizeof(T) == 4 ? x[u][e & 3] : (x[u][e / 2 & 3] >> 16 * (e & 1)) & 0xffffu);
            if (u == 0 && e == 0) {
                bv = v;
                bi = tid < nvec ? i : -1;
            } else if (bv == bv && !(v <= bv)) {
                bv = v;
                bi = i + e;
            }
        }
    }
    if (bi >= 0) {
        const u64 key = argmax_key(bv, bi);
        best = larger(best, key);
    }
    best = wave_largest(best);
    __shared__ u64 part[4];
    if ((tid & 63) == 0) part[tid >> 6] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) best = larger(best, part[w]);
    return best;
}

// The maximum over a row's chunks, in every lane.
__device__ __forceinline__ u64 row_max(const u64 *best, int chunks)
{
    u64 key = 0;
    for (int c = threadIdx.x & 63; c < chunks; c += 64) key = larger(key, best[c]);
    return wave_largest(key);
}

// What lane i knows of node i: the node that it follows (-1: none) and its token.
struct Node {
    int up, token;
    __device__ __forceinline__ Node(const TreeArgs &a, int b)
    {
        const int i = threadIdx.x & 63;
        up = token = -1;
        if (i < a.nodes) {
            up = a.parents[(int64_t)b * a.nodes + i];
            token = a.tokens[(int64_t)b * a.nodes + i];
        }
        if (up >= i) up = -1;
    }
    // the first child of `node` with that token, -1: none
    __device__ __forceinline__ int child(int node, int t) const
    {
        const u64 hit = __ballot(up == node && token == t && t != kNothing);
        return hit ? __builtin_ctzll(hit) : -1;
    }
};

// One level of the walk.
template <int DTYPE, int CE>
__global__ void __launch_bounds__(256) tree_level_kernel(const TreeArgs a, int level)
{
    const int chunk = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int64_t half = (int64_t)a.batch * a.chunks;
    int node = 0;
    if (level > 0) {  // every wave finds it for itself
        // (the maxima are read whether or not the path came to this level, so that all loads go out together)
        const Node mine(a, b);
        const int t = key_token(row_max(a.best + ((level - 1) & 1) * half + (int64_t)b * a.chunks, a.chunks));
        const int before = __builtin_amdgcn_readfirstlane(a.level_node[(int64_t)b * kMaxNodes + level - 1]);
        node = -1;
        if (before >= 0) {
            node = mine.child(before, t);
            if (chunk == 0 && tid == 0) a.level_token[(int64_t)b * kMaxNodes + level - 1] = t;
        }
    } else if (a.do_commit && chunk == 0 && tid == 0) {
        a.old_lens[b] = a.seq_lens[b];
    }
    if (chunk == 0 && tid == 0) a.level_node[(int64_t)b * kMaxNodes + level] = node;
    if (node < 0) return;
    const char *row = (const char *)a.logits + ((int64_t)b * a.nodes + node) * a.stride_row * (DTYPE == 0 ? 4 : 2);
    const u64 best = chunk_max<DTYPE, CE>(row, chunk * CE, a.vocab);
    if (tid == 0) a.best[(level & 1) * half + (int64_t)b * a.chunks + chunk] = best;
}

// Every row.
template <int DTYPE, int CE>
__global__ void __launch_bounds__(256) tree_scan_kernel(const TreeArgs a)
{
    const int chunk = blockIdx.x, b = blockIdx.z;
    const int64_t row = (int64_t)b * a.nodes + blockIdx.y;
    if (a.do_commit && threadIdx.x == 0 && chunk == 0 && blockIdx.y == 0) a.old_lens[b] = a.seq_lens[b];
    const u64 best = chunk_max<DTYPE, CE>((const char *)a.logits + row * a.stride_row * (DTYPE == 0 ? 4 : 2), chunk * CE, a.vocab);
    if (threadIdx.x == 0) a.best[row * a.chunks + chunk] = best;
}

__global__ void __launch_bounds__(256) tree_commit_kernel(const TreeArgs a)
{
    const int b = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    __shared__ int s_am[kMaxNodes], s_src[kMaxNodes], s_pg[kMaxNodes];
    __shared__ int s_m;
    // loads that do not depend on the path go out first: the tree, the length, then the page ids of the positions that may be appended
    const Node mine(a, b);
    int L = 0, pg = -1;
    if (a.do_commit) {
        L = a.old_lens[b];
        const uint32_t slot = ((uint32_t)L + lane) >> a.page_shift;
        if (wave == 0 && lane < a.max_path && L >= 0 && slot < (uint32_t)a.max_pages_per_seq) pg = a.page_table[(int64_t)b * a.max_pages_per_seq + slot];
    }
    if (!a.walk) {
        // wave w finishes rows w, w + 4, ..; every row's chunks are on their way before the first is looked at
        constexpr int ROWS = kMaxNodes / 4;
        u64 key[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int i = wave + 4 * u;
            key[u] = i < a.nodes && lane < a.chunks ? a.best[((int64_t)b * a.nodes + i) * a.chunks + lane] : 0ull;
        }
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int i = wave + 4 * u;
            if (i < a.nodes) {
                const u64 *row = a.best + ((int64_t)b * a.nodes + i) * a.chunks;
                for (int c = lane + 64; c < a.chunks; c += 64) key[u] = larger(key[u], row[c]);
                const int t = key_token(wave_largest(key[u]));
                if (lane == 0) s_am[i] = t;
            }
        }
    }
    __syncthreads();
    if (wave == 0) {
        int path = -1, token = -1, m = 0;  // lane k: the path's k-th node and the token that it emits
        if (a.walk) {
            if (lane < a.max_path) {
                path = a.level_node[(int64_t)b * kMaxNodes + lane];
                if (lane < a.max_path - 1) token = a.level_token[(int64_t)b * kMaxNodes + lane];
            }
            m = __popcll(__ballot(path >= 0));
            if (m == a.max_path) {  // nobody has looked at the last level's maxima yet
                const int t = key_token(row_max(a.best + ((m - 1) & 1) * (int64_t)a.batch * a.chunks + (int64_t)b * a.chunks, a.chunks));
                if (lane == m - 1) token = t;
            }
        } else {
            int node = 0;
            while (node >= 0 && m < a.max_path) {
                const int t = s_am[node];
                if (lane == m) {
                    path = node;
                    token = t;
                }
                node = mine.child(node, t);
                ++m;
            }
        }
        int committed = m;
        if (a.do_commit) {
            const bool bad = __any(lane < m && (pg < 0 || pg >= a.num_pages));
            if (layer == 0 && lane == 0) {
                if (bad) atomicExch(a.err_word, -4);
                else a.seq_lens[b] = L + m;
            }
            if (bad) committed = 0;
            s_src[lane] = path;
            s_pg[lane] = pg;
        }
        if (layer == 0) {
            if (lane < a.nodes) {
                a.path_nodes[(int64_t)b * a.nodes + lane] = path;
                a.out_tokens[(int64_t)b * a.nodes + lane] = lane >= m ? -1 : token == kNothing ? 0 : token;
            }
            const int anchor = __shfl(token, m - 1);  // kNothing: there is none
            if (lane == 0) {
                a.accept_len[b] = m - 1;
                a.num_committed[b] = committed;
                a.next_anchor[b] = anchor;
            }
        }
        if (lane == 0) s_m = a.do_commit ? committed : 0;
    }
    __syncthreads();
    // this layer's rows: 16-byte chunks, four of each pool in flight before the first store
    const int cpr = a.head_dim / 8, per_tok = a.num_kv_heads * cpr, total = s_m * per_tok;
    auto src_of = [&](int e) __attribute__((always_inline)) {
        const int k = e / per_tok, rem = e - k * per_tok, g = rem / cpr, ch = rem - g * cpr;
        return (int64_t)layer * a.blk_stride_layer + ((int64_t)b * a.nodes + s_src[k]) * a.blk_stride_row + (int64_t)g * a.blk_stride_head + ch * 8;
    };
    auto dst_of = [&](int e) __attribute__((always_inline)) {
        const int k = e / per_tok, rem = e - k * per_tok, g = rem / cpr, ch = rem - g * cpr;
        return (int64_t)layer * a.stride_layer + (int64_t)s_pg[k] * a.stride_page + (int64_t)g * a.stride_head +
               (int64_t)((L + k) & ((1 << a.page_shift) - 1)) * a.stride_tok + ch * 8;
    };
    for (int e0 = tid; e0 < total; e0 += 4 * 256) {
        uint4 k[4], v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            k[u] = v[u] = make_uint4(0, 0, 0, 0);
            if (e0 + u * 256 < total) {
                const int64_t src = src_of(e0 + u * 256);
                k[u] = *(const uint4 *)(a.k_blk_ar + src);
                v[u] = *(const uint4 *)(a.v_blk_ar + src);
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (e0 + u * 256 < total) {
                const int64_t dst = dst_of(e0 + u * 256);
                *(uint4 *)(a.k_pool + dst) = k[u];
                *(uint4 *)(a.v_pool + dst) = v[u];
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// host side

// Logits of a workgroup: the fewer where that brings more of them to the memory at once than it costs launches of workgroups (8192 ->
// 2048 a workgroup, fp32, vocabulary 151936; walked, 8 levels: 8 sequences 37.0 -> 33.1 us, 16 39.1 -> 36.7, 64 50.9 -> 64.2; every row
// scanned: 1 x 32 rows 15.0 -> 13.7, 4 x 16 15.2 -> 14.0, 16 x 16 31.4 -> 30.7, 4 x 64 33.4 -> 34.1, 8 x 48 in bf16 27.9 -> 34.1).  Many
// rows of 16 bits, every row scanned, lie between: a thread has twice the comparisons behind its loads (8192 -> 4096: 8 x 48 28.1 -> 27.0,
// 24 x 64 82.7 -> 77.9, 64 x 64 214 -> 206; fp32 8 x 48 31.6 both, 64 x 64 391 -> 399).
constexpr int kTreeChunk = 8192, kTreeChunkFew = 2048, kTreeChunk16 = 4096;

size_t tree_best_bytes(int batch, int nodes, int vocab)
{
    const size_t rows = (size_t)batch * (nodes < 2 ? 2 : nodes);  // the walk has two levels
    return rows * (((size_t)vocab + kTreeChunkFew - 1) / kTreeChunkFew) * sizeof(u64);
}

template <int DTYPE, int CE, bool WALK>
static hipError_t launch_tree(TreeArgs a, hipStream_t stream)
{
    a.chunks = (a.vocab + CE - 1) / CE;
    if constexpr (WALK) {
        for (int level = 0; level < a.max_path; ++level) {
            hipLaunchKernelGGL((tree_level_kernel<DTYPE, CE>), dim3((unsigned)a.chunks, (unsigned)a.batch), dim3(256), 0, stream, a, level);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    } else {
        hipLaunchKernelGGL((tree_scan_kernel<DTYPE, CE>), dim3((unsigned)a.chunks, (unsigned)a.nodes, (unsigned)a.batch), dim3(256), 0, stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(tree_commit_kernel, dim3(a.batch, a.do_commit ? a.num_layers : 1), dim3(256), 0, stream, a);
    return hipGetLastError();
}

int tree_chunk(int walk, int batch, int nodes, int vocab, int dtype)
{
    const int64_t logits = (walk ? batch : (int64_t)batch * nodes) * vocab;
    if (logits < (int64_t)(walk ? 512 : 4096) * kTreeChunk) return kTreeChunkFew;
    return walk || dtype == 0 ? kTreeChunk : kTreeChunk16;
}

template <int DTYPE>
static hipError_t launch_tree_sized(const TreeArgs &a, hipStream_t stream)
{
    const bool few = tree_chunk(a.walk, a.batch, a.nodes, a.vocab, DTYPE) == kTreeChunkFew;
    if (a.walk) return few ? launch_tree<DTYPE, kTreeChunkFew, true>(a, stream) : launch_tree<DTYPE, kTreeChunk, true>(a, stream);
    return few ? launch_tree<DTYPE, kTreeChunkFew, false>(a, stream) : launch_tree<DTYPE, DTYPE == 0 ? kTreeChunk : kTreeChunk16, false>(a, stream);
}

// Every row at once runs at 6.2 to 6.6 TB/s, a level costs some 4 us and its rows' share of that (fp32, vocabulary 151936, walked ->
// every row: 64 sequences of 64 nodes, 8 levels 51 -> 375 us, 16 39 -> 101, 8 37 -> 56, 4 37.9 -> 33.4, 4 of 16 37.5 -> 15, 16 of 16
// 39 -> 31, 16 of 32 with 5 levels 30 -> 54).
int tree_walks(int batch, int nodes, int max_path, int vocab, int dtype)
{
    const double bytes = (double)vocab * (dtype == 0 ? 4 : 2) * batch;
    const double all = nodes * bytes / 6.5e6, level = bytes / 6.5e6;  // us
    return all > (max_path < nodes ? max_path : nodes) * (level + 4.5);
}

hipError_t launch_tree_consensus(TreeArgs a, hipStream_t stream)
{
    if (a.batch == 0) return hipSuccess;
    if (a.max_path > a.nodes) a.max_path = a.nodes;
    a.walk = tree_walks(a.batch, a.nodes, a.max_path, a.vocab, a.dtype);
    return a.dtype == 0 ? launch_tree_sized<0>(a, stream) : a.dtype == 1 ? launch_tree_sized<1>(a, stream) : launch_tree_sized<2>(a, stream);
}

}  // namespace orthrus
