// The attention kernel for launches that are bound by arithmetic: prefill, and decode-mode batches with enough query
// rows and units to fill the chip (the training block mask above all).  Same problem, MFMA forms, LDS tile layout
// and masks as attn_split_kernel, never split along the keys (orthrus_attn.hip); what differs is how a CU is filled.
//
// Why: with 32 query rows per wave every 32-token tile costs a wave 16 KB of LDS reads for 512 cycles of matrix
// instructions, and a wave's own chain (operand reads, scores, softmax, values) leaves the matrix cores idle for most
// of it: 37 % busy in an 8192-token prefill with two such waves on each SIMD.  Here a wave owns 64 rows as two blocks
// (one wave per SIMD, up to 512 registers), so an operand read serves two products, and the two blocks are half a tile
// apart: while block 0's scores of tile i and values of tile i-1 go through the matrix cores, the vector unit takes
// block 1's softmax of tile i-1, and the other way round in the second half ("slots").  Inside a slot every matrix
// instruction is followed by its share of the softmax and of the LDS reads and loads, in written order
// (sched_barrier): the compiler's own order keeps them apart.
// Every wave issues its own share of the tile loads (a loader wave would halve the registers), NS-1 tiles ahead.
//
// What bounds it: issue, and at full load the power that the products draw.  One wave issues a vector instruction every
// 6 to 8 cycles, other ones every 4, so whatever is not a product or softmax costs time: a product with its share of the
// softmax (multiply-add, exponential, sum, half a conversion) takes 35 cycles against the product's own 32, and the rest
// of a tile's instructions come on top.  The main loop therefore takes a turn of the ring at a time, so that LDS
// addresses are instruction offsets, waits for LDS twice a tile, and keeps the memory addresses of 64 tiles in vector
// registers: 190 instructions a 64x32 tile (counters: 157 vector ones with the products, 24 LDS, 5 scalar, 4 loads) where an
// address calculation and a wait at each use made it 225.  Measured before and after: one item to a CU (100 new tokens
// behind 16000, 7 heads a KV head) 351 -> 291 us a call; 16384 new tokens (32/8 heads) 1763 -> 1670, where the kernel's cycles
// fall by 13 %, the products' share of them rises from 0.61 to 0.70 and the clock falls from 1.97 to 1.81 GHz; 8192 new tokens
// 478 -> 456; ragged prefill at 28/4 heads 325 -> 300; training mask 623 -> 598.  (attn_split_kernel's form: 675, 400 and 864
// for the last three.  With the chunks ranked over all sequences the ragged prefill takes 250 to 280 by the order of the
// lengths, with 16-byte stores the mask 570 to 602 from one card to another.)
#include "orthrus_attn_wide_dev.h"

namespace orthrus {

// D head_dim, W waves of 64 query rows, NS LDS stages, MODE the work items (not kItemsBalanced), NT the
// non-temporal form of the tile loads.
template <int D, int W, int NS, int MODE, int NT = 0>
__global__ void __launch_bounds__(64 * W, 1) attn_wide_kernel(ATTN_FIRST_PARAMS, const AttnArgs rest)
{
    constexpr bool TREE = false;
#include "orthrus_attn_wide.inc"
}

// ---------------------------------------------------------------------------------------------
// host side

int attn_wide_per_cu(int waves) { return 4 / waves; }  // one wave per SIMD

size_t attn_wide_lds(int waves, int head_dim)
{
    return (size_t)wide_stages(waves) * (head_dim == 128 ? AttnGeom<128>::STAGE_B : AttnGeom<64>::STAGE_B);
}

// Decode mode: whether this kernel beats attn_split_kernel when neither cuts a unit.  It needs waves that are nearly all
// rows (7/8; of 96 rows the training mask takes 626 -> 640 us), units enough for a wave on every SIMD, and lengths over
// which its shorter tile makes up for the longer start and end.  The lines were drawn with the former main loop; both sides
// with today's (attn_split_kernel -> this kernel, us per call, lengths equal to the bound; 256 CUs):
//   d = 128, up to 128 rows: 512 units of 64 / 300 / 1000 tokens at 112 rows 13.6 -> 14.9 / 27.6 -> 27.3 / 64.4 -> 60.8, of
//     180 at 128 rows 21.1 -> 20.6, 896 of 180 40.5 -> 40.9; 256 units of 1000 32.9 -> 36.7; a second round for a few units
//     pays only when it is long or the lengths are mixed, which a long bound suggests (640 units of 400 tokens 45.0 -> 49.8,
//     544 of 1000 79.8 -> 81.5, 640 of 2000 and of 200..1800 1.01 and 1.02 times as fast, the mask's 544 over 1024 / 2048
//     tokens 1.11 and 1.25; 768 units of 400 52.2 -> 54.4)
//   d = 128, more rows: two such waves' work is what four 32-row waves with a loader do as well; 224 rows lose everywhere
//     (1024 units of 1000 tokens 160 -> 164), 256 rows gain from about 2000 tokens on (384 units of 1000 / 2500 tokens
//     76.0 -> 72.2 / 176 -> 144, 256 units of 3000 110 -> 102; masks of 384 over 1024 and of 512 over 2048 tokens 52.4 -> 52.1
//     and 105 -> 97)
//   d = 64, up to 128 rows: 512 units lose at any length (3000 tokens: 83.5 -> 90.1), 640 of 400 / 1000 tokens 22.5 ->
//     22.4 / 48.2 -> 44.6 but the mask's 640 and 704 over 2048 tokens 47.7 -> 52.6 and 52.2 -> 54.7; 768 of 180 / 256 tokens
//     16.1 -> 17.5 / 17.5 -> 18.2, 1024 of 400 38.8 -> 34.3
//   d = 64, more rows: 320 units of 300 / 512 / 1000 tokens at 256 rows 22.1 -> 20.7 / 28.7 -> 25.1 / 48.2 -> 39.0, 256 of
//     700 / 1000 19.9 -> 20.8 / 26.6 -> 25.2; at 224 rows 384 units of 700 / 2000 tokens 29.2 -> 30.5 / 81.6 -> 71.3, the
//     mask's 352 over 4096 tokens 0.96 times as fast, its 384 1.12
// So a few calls now lie on the wrong side: the 32-row kernel keeps 256 rows of d = 128 at 256 units of 3000 (7 %) and 384 of
// 1000 (5 %), and of d = 64 640 units of 1000 at 128 rows (8 %) and 320 of 300 at 256 (6 %); this kernel takes 768 units of
// 400 (4 %), and of d = 64 704 of the mask's (5 %) and 768 of 256 tokens (4 %).
bool attn_wide_pays(int head_dim, int rows, int max_seq_len, int64_t units, int num_cus)
{
    const int waves = rows > 128 ? 4 : 2;
    const int64_t cus = num_cus;
    const bool full = rows >= 60 * waves;
    if (rows < 56 * waves) return false;
    if (waves == 2) {
        if (head_dim == 64) return max_seq_len >= 256 && 4 * units >= 11 * cus;
        if (full && max_seq_len >= 128 && (units == 2 * cus || 2 * units >= 7 * cus)) return true;
        return max_seq_len >= 384 && (units == 2 * cus || units >= 3 * cus || (units > 2 * cus && max_seq_len >= 1024));
    }
    if (head_dim == 128) return full && max_seq_len >= 1920 && units > cus;
    if (!full) return max_seq_len >= 1024 && 2 * units >= 3 * cus;
    return max_seq_len >= 896 ? units >= cus : max_seq_len >= 512 && 4 * units >= 5 * cus;
}

template <int D, int W>
static auto wide_decode_kernel(const AttnPlan &plan)
{
    if (plan.by_size) return plan.kv_nt ? attn_wide_kernel<D, W, wide_stages(W), kItemsBySize, 1> : attn_wide_kernel<D, W, wide_stages(W), kItemsBySize, 0>;
    return plan.kv_nt ? attn_wide_kernel<D, W, wide_stages(W), kItemsSplit, 1> : attn_wide_kernel<D, W, wide_stages(W), kItemsSplit, 0>;
}

hipError_t launch_attn_wide(const AttnArgs &a, const AttnPlan &plan, int head_dim, dim3 grid, hipStream_t stream, AttnLaunchEvents *ev)
{
    auto kern = head_dim == 128 ? (plan.waves == 4 ? wide_decode_kernel<128, 4>(plan) : wide_decode_kernel<128, 2>(plan))
                                : (plan.waves == 4 ? wide_decode_kernel<64, 4>(plan) : wide_decode_kernel<64, 2>(plan));
    return launch_timed(kern, grid, dim3(64 * plan.waves), plan.lds_bytes, a, stream, ev, 0);
}

// Ranked order: a few sequences, and more items than are resident at once.  Items that all start together need no order, and
// finding a rank costs each of them two round trips and the search (plain -> ranked: 16 sequences of 0..2000 cached and up to
// 33 new tokens, 32/8 heads, 44.7 -> 48.8 us with the former search; 8 of 0..3000 and 100..300, 4/2 heads of 64, 48.2 -> 50.0).
bool prefill_ranked(int batch, int64_t items, int per_cu, int num_cus)
{
    return batch > 1 && batch <= kRankedBatch && items > (int64_t)per_cu * num_cus;
}

namespace {
// 64 lanes as arrays: the search above, compiled for the host
struct HostLanes {
    struct Int {
        int v[64];
        Int(int x = 0) { for (int &y : v) y = x; }
        template <class F>
        static Int each(const Int &a, const Int &b, F f) { Int r; for (int i = 0; i < 64; ++i) r.v[i] = f(a.v[i], b.v[i]); return r; }
        friend Int operator+(const Int &a, const Int &b) { return each(a, b, [](int x, int y) { return x + y; }); }
        friend Int operator-(const Int &a, const Int &b) { return each(a, b, [](int x, int y) { return x - y; }); }
        friend Int operator*(const Int &a, const Int &b) { return each(a, b, [](int x, int y) { return x * y; }); }
        friend Int operator>>(const Int &a, int n) { return each(a, n, [](int x, int y) { return x >> y; }); }
    };
    static Int lane() { Int r; for (int i = 0; i < 64; ++i) r.v[i] = i; return r; }
    static Int lesser(const Int &a, const Int &b) { return Int::each(a, b, [](int x, int y) { return x < y ? x : y; }); }
    static Int larger(const Int &a, const Int &b) { return Int::each(a, b, [](int x, int y) { return x > y ? x : y; }); }
    template <class F>
    static Int over_row(const Int &a, F f)
    {
        Int r;
        for (int i = 0; i < 64; ++i) {
            int x = a.v[i & 48];
            for (int j = 1; j < 16; ++j) x = f(x, a.v[(i & 48) + j]);
            r.v[i] = x;
        }
        return r;
    }
    static Int row_sum(const Int &a) { return over_row(a, [](int x, int y) { return x + y; }); }
    static Int row_max(const Int &a) { return over_row(a, [](int x, int y) { return x > y ? x : y; }); }
    static uint64_t less(const Int &a, const Int &b)
    {
        uint64_t m = 0;
        for (int i = 0; i < 64; ++i) m |= (uint64_t)(a.v[i] < b.v[i]) << i;
        return m;
    }
    static int read(const Int &a, int lane) { return a.v[lane]; }
};
}  // namespace

bool ranked_chunk_on_host(int rank, int batch, const int *end_levels, const int *chunks, int *seq, int *chunk)
{
    HostLanes::Int e, n;
    for (int i = 0; i < 64; ++i) {
        const int x = i & 15;
        e.v[i] = x < batch ? end_levels[x] : 0;
        n.v[i] = x < batch ? chunks[x] : 0;
    }
    return ranked_chunk<HostLanes>(rank, e, n, seq, chunk);
}

template <int D, int W>
static hipError_t launch_prefill_wide(AttnArgs a, int num_cus, hipStream_t stream)
{
    a.chunk_tokens = 64 * W / a.group;
    a.rows = 64 * W;
    a.num_splits = (a.max_new + a.chunk_tokens - 1) / a.chunk_tokens;
    dim3 grid((unsigned)a.num_splits * (unsigned)a.num_kv_heads * (unsigned)a.batch);
    a.ranked = prefill_ranked(a.batch, grid.x, attn_wide_per_cu(W), num_cus);
    hipLaunchKernelGGL((attn_wide_kernel<D, W, wide_stages(W), kItemsPrefill>), grid, dim3(64 * W), attn_wide_lds(W, D), stream, ATTN_FIRST_VALUES(a), a);
    return hipGetLastError();
}

// Prefill forms.  A 32-row wave with its own loader is the shorter chain, so for up to four waves a workgroup
// attn_split_kernel's prefill form stays while SIMDs would be idle otherwise.  How long that is depends on how the items'
// lengths are spread (32-row form -> this kernel, us per call):
//   - From 0 up, the new tokens being most of what is cached (by the bound: max_seq_len < 2 * max_new): the longest items
//     start first and short ones fill in behind them.  One sequence of n tokens:
//     d = 128: group 4, 2 heads, n = 7000 (1.7 waves per SIMD) 131 -> 141, 8 heads, n = 4000 (3.9) 164 -> 127; group 3, 2
//     heads, n = 7000 (1.3) 128 -> 135; group 2, 8 heads, n = 2000 / 4000 (1.0 / 2.0) 45 -> 50 / 105 -> 92; group 1, 8
//     heads, n = 4000 / 7000 (1.0 / 1.7) 75 -> 85 / 170 -> 150.  d = 64: group 1, 8 heads, n = 4000 / 9000 (1.0 / 2.2)
//     57 -> 67 / 151 -> 144; group 4, 8 heads, n = 2000 / 4000 (2.0 / 3.9) 36 -> 41 / 96 -> 89.
//   - Of about equal length (behind a longer cache): what does not fit at once comes as a whole round more.  One 32-row
//     wave per SIMD, all workgroups resident (LDS ring: three per CU, of four waves two; d = 64 and one wave: six):
//     3000 cached tokens, d = 128: group 1, 32 heads, n = 700 (2.75 workgroups per CU) 77 -> 89, n = 1021 (4) 132 -> 100;
//     group 2, 8 heads, n = 2000 (1.0 waves per SIMD) 118 -> 102; group 4, 8 heads, n = 700 / 2000 (0.7 / 2.0) 74 -> 79 /
//     155 -> 130.  Or where this kernel would need a second round and the 32-row form would not: group 3, 32 heads,
//     n = 700 152 -> 166.
// The lines were drawn with the former main loop (which took 57, 159, 122 and 94 us where 50, 135, 102 and 79 stand now), so
// the 32-row form keeps a little too much: group 2, 8 heads, n = 2000 behind 3000 (15 %) and d = 64, group 1, n = 9000 (5 %).
// More than four query heads per KV head: this kernel at any size.  Its former main loop against the 32-row form with five to
// eight waves that it took the place of, 4000 cached tokens, n = 32: group 5 / 6 / 7 / 8 108 -> 97 / 107 -> 97 / 111 -> 97 /
// 113 -> 97; empty cache, n = 700: 36 -> 31 / 34 -> 29 / 35 -> 30 / 36 -> 30 (5 us of each for the shorter front end).
// Four waves per workgroup once every CU gets two of them, else two waves for the finer grain (8 sequences of 333 tokens:
// 29 against 31 us), unless the finer grain spills into a round of its own (group 3, 32 heads, 2500 cached tokens, n = 677:
// 544 workgroups of two waves 141 us, 256 of four 105); d = 64 is faster with four throughout (40 against 47 us with the
// former loop).
int prefill_wide_waves(int head_dim, int group, int64_t units, int max_new, int max_seq_len, int num_cus)
{
    const int64_t cus = num_cus;
    auto items_of = [&](int tokens) { return units * ((max_new + tokens - 1) / tokens); };
    const int64_t items4 = items_of(256 / group);
    const bool even = max_seq_len >= 2 * (int64_t)max_new;
    if (group <= 4) {
        const int64_t items32 = items_of(32), waves32 = items32 * group;
        const bool thin = head_dim == 64 && group == 1;
        if (!even) {
            if (waves32 <= (head_dim == 64 ? 10 : group <= 2 ? 6 : 8) * cus) return 0;
        } else if (items32 < (thin ? 6 : group <= 3 ? 3 : 2) * cus && (waves32 <= (thin ? 6 : 4) * cus || items4 > cus)) {
            return 0;
        }
    }
    if (head_dim == 64 || items4 >= 2 * cus) return 4;
    return even && (items_of(128 / group) + 2 * cus - 1) / (2 * cus) > (items4 + cus - 1) / cus ? 4 : 2;
}

hipError_t launch_prefill_attn(const AttnArgs &a, int head_dim, int num_cus, hipStream_t stream)
{
    if (a.batch == 0 || a.max_new == 0) return hipSuccess;
    const int waves = prefill_wide_waves(head_dim, a.group, (int64_t)a.batch * a.num_kv_heads, a.max_new, a.max_seq_len, num_cus);
    if (waves == 0) return launch_prefill_split(a, head_dim, num_cus, stream);
    if (head_dim == 128) return waves == 2 ? launch_prefill_wide<128, 2>(a, num_cus, stream) : launch_prefill_wide<128, 4>(a, num_cus, stream);
    if (head_dim == 64) return launch_prefill_wide<64, 4>(a, num_cus, stream);
    return hipErrorInvalidValue;
}

}  // namespace orthrus
