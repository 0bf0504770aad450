// Attention of a tree of drafted tokens over the paged cache (verification pass of Section 3.3 with drafts that branch):
//   O_i = Softmax(q_i [K_cache || K_A(i)]^T * scale) [V_cache || V_A(i)],   A(i) = the nodes from the root down to node i.
//
// A chain of drafts is the tree in which every node follows the one before it, and the mask is then the causal one.  Cache,
// queries, tiles, matrix products and softmax are those of attn_split_kernel, whose body this kernel is; its own are
//   - the mask of the block: a lane owns one query row, and the row's path is 64 bits that it finds from the parents with six
//     steps of lane exchanges (tree_path), next to the first tiles' way through memory.  A tile of the block costs a shift and
//     16 bit tests; the cache's tiles cost nothing more than a chain's;
//   - up to 64 nodes, in one or two tiles behind the cache's;
//   - more query rows (group x nodes) than eight waves hold, 256, in two workgroups that each stream the cache; in the balanced form, of
//     at most seven waves, more than 224 in two and more than 448 in three (plan_tree_attn).  64/8 heads, 4 x 32768 tokens: 32 nodes
//     (256 rows) 158 us a call, 64 nodes (512) 278; one of 4096 22 and 26.
// Launches with rows and units enough to be bound by the products run the 64-row kernel (orthrus_attn_tree_wide.hip), by the rule
// of the chains (attn_wide_pays).
// What bounds it, as it does the chains: 4 x 32768 tokens, 16 nodes (32/8 heads, 64 rows) 86.6 us a call, 6.2 TB/s of the cache; one
// sequence of 4096, 32 nodes 15.9 us, the chain of tiles, partials and merge; 16 of 512..8192 tokens, 32 nodes at 28/4 heads, shared out
// evenly, 56 to 60 us.  Short calls of one block of rows 8 us, 5 of them the kernel.
// (The rest that rounding the weights to bf16 leaves, as a second value product, takes the error from 0.0024 to the output's own 0.0017
// of its size and costs 4 x 32768 tokens, 8 nodes 85.7 -> 96.3 us, one of 4096 13.3 -> 15.1: not in the library.)
#include "orthrus_attn_dev.h"

namespace orthrus {

// Waves per SIMD that the registers must allow.  The balanced form keeps more across its segments than a third of the registers
// holds next to the tiles (eleven were spilled), so it has half of them, and at most seven row blocks to a workgroup.  With six and seven
// that costs no residency; with one to five a CU holds fewer workgroups than of the chains' form (three waves a SIMD), against
// which it was not timed.  16 trees over 512..8192 tokens at 32/8 heads, balanced / fixed splits: 8 nodes 57 / 71 us, 16 59 / 79,
// 24 71 / 80, 32 72 / 90, 48 92 / 115, 64 (two workgroups a head) 119 / 133; 64/8 heads, 32 nodes 117 / 133, 64 (three) 230 / 216.
constexpr int tree_waves(int mode) { return mode == kItemsBalanced ? 2 : 3; }
constexpr int tree_blocks(bool balanced) { return balanced ? 7 : 8; }

template <int D, int W, int NS, int MODE, int NT>
__global__ void __launch_bounds__(64 * (W + 1), tree_waves(MODE)) attn_tree_kernel(ATTN_FIRST_PARAMS, const AttnArgs rest)
{
    constexpr int PROBE = 0, ROWS = 32;
    constexpr bool TREE = true;
#include "orthrus_attn_split.inc"
}

// x / y rounded down, 0 <= x, y < 2^53: one division in 64-bit floating point and a step of correction, where one of integers is
// some 150 instructions.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y)
{
    const int64_t q = (int64_t)((double)x / (double)y), rest = x - q * y;
    return rest < 0 ? q - 1 : rest >= y ? q + 1 : q;
}

// The pieces of a row group's units merged in their order, as attn_combine_kernel does: one workgroup per (unit, 32-row block,
// 32-wide d block), a wave to four d values, a lane reads the float4 that it would hold in the accumulator.
template <int D, int BALANCED>
__global__ void __launch_bounds__(256) attn_tree_merge_kernel(ATTN_FIRST_PARAMS, const AttnArgs rest, int W)
{
    const AttnArgs a = with_first(rest, first_lens, first_batch);
    constexpr int DBLK = D / 32, CHUNK = BALANCED ? 8 : 16;
    const int lane = threadIdx.x & 63, r4 = threadIdx.x >> 6, col = lane & 31, h = lane >> 5;
    const int db = (int)(blockIdx.x % DBLK);
    const int wave = (int)(blockIdx.x / DBLK % (unsigned)W);
    const int unit = (int)(blockIdx.x / (DBLK * (unsigned)W));
    const int b = unit / a.num_kv_heads, g = unit % a.num_kv_heads;
    const int kv = g / a.row_groups, blk_tiles = (a.block_k + 31) >> 5;
    const int ridx = (g % a.row_groups * W + wave) * 32 + col;
    int live;
    size_t first_slot, rest_slot, slot_step;
    if constexpr (BALANCED) {
        int before = 0, per_head = 0, mine = 0;  // tiles of the sequences before b, of all, of b
        for (int x0 = 0; x0 < a.batch; x0 += 64) {
            const int x = x0 + lane;
            int n = 0;
            if (x < a.batch) {
                int L = a.seq_lens[x];
                L = L < 0 ? 0 : (L > a.max_seq_len ? a.max_seq_len : L);
                n = ((L + 31) >> 5) + blk_tiles;
            }
            int nb = x < b ? n : 0, nm = x == b ? n : 0;
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) {
                n += __shfl_xor(n, off);
                nb += __shfl_xor(nb, off);
                nm += __shfl_xor(nm, off);
            }
            per_head += n;
            before += nb;
            mine += nm;
        }
        const int64_t total = (int64_t)per_head * a.num_kv_heads;
        const int64_t nwg = total < (int64_t)a.bal_wgs ? total : (int64_t)a.bal_wgs;
        const int64_t U0 = (int64_t)g * per_head + before, U1 = U0 + mine;
        // workgroup w starts at tile floor(w * total / nwg): the last one that starts at or before U0, and before U1
        const int64_t w_lo = quotient((U0 + 1) * nwg + total - 1, total) - 1;
        const int64_t w_hi = quotient(U1 * nwg + total - 1, total) - 1;
        if (w_lo == w_hi) return;  // one workgroup held the whole unit and wrote its rows
        live = (int)(w_hi - w_lo + 1);
        first_slot = (size_t)w_lo * 2 + 1;
        rest_slot = (size_t)w_lo * 2;
        slot_step = 2;
    } else {
        int L = a.seq_lens[b];
        L = L < 0 ? 0 : (L > a.max_seq_len ? a.max_seq_len : L);
        live = split_cut(L, a.num_splits, 0, blk_tiles).live;
        first_slot = rest_slot = (size_t)unit * a.num_splits;
        slot_step = 1;
    }
    // Every piece's rows and their (m, l) are on their way before the first is looked at, of a fixed count before the length is known:
    // what a shorter sequence's last slots hold is dropped (one of 4096 tokens, 13 pieces 16.5 -> 16.0 us a call).
    const int slots = BALANCED ? live : a.num_splits;
    auto slot_of = [&](int s) __attribute__((always_inline)) {
        return (s == 0 ? first_slot : rest_slot + (size_t)s * slot_step) * W + wave;
    };
    float M = kNegBig;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float lsum = 0.f;
    for (int s0 = 0; s0 < slots; s0 += CHUNK) {
        float4 v[CHUNK];
        float2 e[CHUNK];
#pragma unroll
        for (int u = 0; u < CHUNK; ++u) {
            v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            e[u] = make_float2(kNegBig, 0.f);
            if (s0 + u < slots) {
                const size_t slot = slot_of(s0 + u);
                v[u] = ((const float4 *)a.part_o)[slot * (DBLK * 4 * 64) + (size_t)(db * 4 + r4) * 64 + lane];
                e[u] = ((const float2 *)a.part_ml)[slot * 32 + col];
            }
        }
        float top = M;
#pragma unroll
        for (int u = 0; u < CHUNK; ++u) top = s0 + u < live ? fmaxf(top, e[u].x) : top;
        const float before = __builtin_amdgcn_exp2f(M - top);
        M = top;
        lsum *= before;
        acc.x *= before; acc.y *= before; acc.z *= before; acc.w *= before;
#pragma unroll
        for (int u = 0; u < CHUNK; ++u) {  // fixed order: the result does not depend on timing
            if (s0 + u < live) {
                const float sc = __builtin_amdgcn_exp2f(e[u].x - M);
                lsum += sc * e[u].y;
                acc.x += sc * v[u].x; acc.y += sc * v[u].y; acc.z += sc * v[u].z; acc.w += sc * v[u].w;
            }
        }
    }
    if (ridx >= a.rows) return;
    const int G = a.group, K = a.block_k;
    const int i = ridx / G, hl = ridx - i * G;
    const float inv = lsum > 0.f ? 1.f / lsum : 0.f;
    uint16_t *op = a.out + (((int64_t)b * K + i) * a.num_q_heads + (int64_t)kv * G + hl) * D;
    uint2 pk;
    pk.x = pack_bf16(acc.x * inv, acc.y * inv);
    pk.y = pack_bf16(acc.z * inv, acc.w * inv);
    *(uint2 *)(op + 32 * db + 8 * r4 + 4 * h) = pk;
    if (a.lse && db == 0 && r4 == 0 && h == 0)
        a.lse[((int64_t)b * a.num_q_heads + (int64_t)kv * G + hl) * K + i] =
            (M + __builtin_amdgcn_logf(lsum)) * 0.6931471805599453f;
}

// ---------------------------------------------------------------------------------------------
// host side

hipError_t plan_tree_attn(int head_dim, int group, int nodes, int batch, int num_kv_heads, int max_seq_len, int requested_splits,
                          int num_cus, int num_layers, double pool_tokens, AttnPlan *plan, int *row_groups)
{
    const int blocks = (group * nodes + 31) / 32;
    const int most = tree_blocks(requested_splits < 0);
    const int groups = (blocks + most - 1) / most;
    const int rows = groups == 1 ? group * nodes : 32 * ((blocks + groups - 1) / groups);  // of one of them
    *row_groups = groups;
    const hipError_t e = plan_attn(head_dim, 1, rows, batch, num_kv_heads * groups, max_seq_len, requested_splits, num_cus,
                                   num_layers, pool_tokens, plan);
    if (!plan->wide) plan->lds_bytes += kTreePathBytes;
    if (plan->bal_wgs > 0) {  // resident at once, two partial slots each
        const int by_waves = 4 * tree_waves(kItemsBalanced) / (plan->waves + 1), by_lds = (int)(160 * 1024 / plan->lds_bytes);
        plan->bal_wgs = num_cus * (by_waves < by_lds ? by_waves : by_lds);
        plan->part_o_bytes = (size_t)plan->bal_wgs * 2 * plan->rows_padded * head_dim * sizeof(float);
        plan->part_ml_bytes = (size_t)plan->bal_wgs * 2 * plan->rows_padded * 2 * sizeof(float);
    }
    if (groups > 1) plan->kv_nt = 0;  // the cache's rows are read again by the next group of a head
    return e;
}

template <int D, int W>
static hipError_t launch_tree_w(const AttnArgs &a, const AttnPlan &plan, dim3 grid, hipStream_t stream)
{
    if (plan.bal_wgs > 0) {
        if constexpr (W <= tree_blocks(true))
            return launch_timed(attn_tree_kernel<D, W, kStages, kItemsBalanced, kNtAsked>, grid, dim3(64 * (W + 1)), plan.lds_bytes, a, stream, nullptr, 0);
        return hipErrorInvalidValue;
    }
    auto kern = plan.by_size     ? (plan.kv_nt ? attn_tree_kernel<D, W, kStages, kItemsBySize, 1> : attn_tree_kernel<D, W, kStages, kItemsBySize, 0>)
                                 : (plan.kv_nt ? attn_tree_kernel<D, W, kStages, kItemsSplit, 1> : attn_tree_kernel<D, W, kStages, kItemsSplit, 0>);
    return launch_timed(kern, grid, dim3(64 * (W + 1)), plan.lds_bytes, a, stream, nullptr, 0);
}

template <int D>
static hipError_t launch_tree_d(const AttnArgs &a, const AttnPlan &plan, hipStream_t stream)
{
    const bool bal = plan.bal_wgs > 0;
    const unsigned units = (unsigned)a.batch * (unsigned)a.num_kv_heads;
    const dim3 grid(bal ? (unsigned)plan.bal_wgs : units * (unsigned)plan.num_splits);
    if (plan.wide) return launch_tree_wide(a, plan, D, grid, stream);  // (never split)
    hipError_t e = hipErrorInvalidValue;
    switch (plan.waves) {
    case 1: e = launch_tree_w<D, 1>(a, plan, grid, stream); break;
    case 2: e = launch_tree_w<D, 2>(a, plan, grid, stream); break;
    case 3: e = launch_tree_w<D, 3>(a, plan, grid, stream); break;
    case 4: e = launch_tree_w<D, 4>(a, plan, grid, stream); break;
    case 5: e = launch_tree_w<D, 5>(a, plan, grid, stream); break;
    case 6: e = launch_tree_w<D, 6>(a, plan, grid, stream); break;
    case 7: e = launch_tree_w<D, 7>(a, plan, grid, stream); break;
    case 8: e = launch_tree_w<D, 8>(a, plan, grid, stream); break;
    }
    if (e != hipSuccess || (!bal && plan.num_splits == 1)) return e;
    auto merge = bal ? attn_tree_merge_kernel<D, 1> : attn_tree_merge_kernel<D, 0>;
    hipLaunchKernelGGL(merge, dim3(units * (unsigned)plan.waves * (D / 32)), dim3(256), 0, stream, ATTN_FIRST_VALUES(a), a, plan.waves);
    return hipGetLastError();
}

hipError_t launch_tree_attn(const AttnArgs &a, const AttnPlan &plan, int head_dim, hipStream_t stream)
{
    if (a.batch == 0) return hipSuccess;
    return head_dim == 128 ? launch_tree_d<128>(a, plan, stream) : launch_tree_d<64>(a, plan, stream);
}

}  // namespace orthrus
