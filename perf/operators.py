"""Performance cases of the operators around the decode step: drawing tokens, the consensus of filtered distributions,
page tables and slot maps from request lengths, and the store of packed K/V rows into the paged cache.

A case is a dict of plain values.  `kind` names the operator:

  sample   one token per logits row by temperature, top-k, top-p and min-p from a given uniform number
  verify   the lossless consensus of a block under each sequence's filters, and the commit into the cache
  tables   pages for the requests that grow, pages back from those that ended, the slots of the new tokens
  store    packed K/V rows of new tokens written to their slots in the paged cache

`own` false: `run` computes in elementary torch operations; true: it calls the framework.  Calls that change what they
are given (tables, lengths) get the values of before the call back first, so that every pass is the same one.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
P = 16                      # tokens per cache page
BIG = 3.4028234663852886e38  # the largest float
ONE_BELOW = 1.0 - 2.0 ** -24  # the largest float below one

# (temperature, top_k, top_p, min_p) of requests; sequence b takes entry b mod length
MIXES = {
    "nucleus": [(0.8, 0, 0.95, 0.0)],
    "chat": [(0.7, 0, 0.9, 0.0), (0.6, 20, 0.95, 0.0), (1.0, 50, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.05),
             (0.8, 40, 0.95, 0.05), (1.0, 0, 1.0, 0.0), (1.2, 0, 0.98, 0.02)],
    "plain": [(1.0, 0, 1.0, 0.0)],
    "topk": [(0.9, 40, 1.0, 0.0), (0.7, 200, 0.9, 0.0)],
    "warm": [(1.0, 0, 0.9, 0.0), (1.5, 0, 0.95, 0.0)],
}


def listed():
    heads = dict(hkv=8, d=128)
    return [
        # the smallest call: one row of a toy vocabulary, all launches and latency
        dict(name="sample_tiny", kind="sample", batch=1, K=1, vocab=512, dtype="f32", logits="peaked", mix="nucleus",
             logprob=1, pad=0),
        # an interactive user's block of drafts
        dict(name="sample_b1", kind="sample", batch=1, K=16, vocab=128256, dtype="f32", logits="peaked", mix="nucleus",
             logprob=0, pad=0),
        # plain decoding of a serving batch: one row a sequence, bf16 logits of a padded head, every request its own filters
        dict(name="sample_decode", kind="sample", batch=256, K=1, vocab=151669, dtype="bf16", logits="peaked", mix="chat",
             logprob=1, pad=267),
        # drafts of a large batch, every request its own filters
        dict(name="sample_b64", kind="sample", batch=64, K=16, vocab=151936, dtype="f32", logits="peaked", mix="chat",
             logprob=0, pad=0),
        # nearly flat rows at high temperatures: nuclei of tens of thousands of tokens
        dict(name="sample_flat", kind="sample", batch=8, K=32, vocab=151936, dtype="f32", logits="flat", mix="warm",
             logprob=0, pad=0),
        # batch 1, one block verified under a nucleus filter, 36 layers committed
        dict(name="verify_b1", kind="verify", batch=1, K=16, vocab=128256, dtype="f32", mix="nucleus", layers=36, lo=4096,
             hi=4096, **heads),
        # a large batch, every request its own filters
        dict(name="verify_b64", kind="verify", batch=64, K=16, vocab=151936, dtype="f32", mix="chat", layers=1, lo=200, hi=500,
             **heads),
        # one decode step of a serving batch: room for a block of 16 each, every eleventh request over
        dict(name="tables_decode", kind="tables", batch=64, lo=100, hi=4000, new_lo=16, new_hi=16, ended=11, short=0),
        # admission of long prompts, some on top of a cached prefix
        dict(name="tables_prompts", kind="tables", batch=48, lo=0, hi=2000, new_lo=500, new_hi=16000, ended=0, short=0),
        # single-token steps of a very large batch
        dict(name="tables_b4096", kind="tables", batch=4096, lo=1, hi=700, new_lo=1, new_hi=1, ended=17, short=0),
        # one decoded token of each of 256 sequences, K and V read where the fused projection left them
        dict(name="store_decode", kind="store", rows=256, layers=1, fused=1, hq=32, skip=0, **heads),
        # a packed batch of prompts, the tail of its buffer unused
        dict(name="store_prompts", kind="store", rows=30000, layers=1, fused=0, hq=32, skip=700, **heads),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above, sizes over their logarithm, trimmed until it costs less than the largest."""
    kind = rng.choice(["sample", "sample", "sample", "verify", "verify", "tables", "tables", "store"])
    if kind == "sample":
        c = dict(kind=kind, batch=_log(rng, 1, 256), K=rng.choice([1, 1, 1, 4, 8, 13, 16, 32]), vocab=_log(rng, 500, 160000),
                 dtype=rng.choice(["f32", "f32", "bf16", "f16"]), logits=rng.choice(["peaked", "peaked", "peaked", "flat"]),
                 mix=rng.choice(sorted(MIXES)), logprob=rng.randint(0, 1), pad=rng.choice([0, 0, rng.randint(1, 300)]))
        while c["batch"] > 1 and c["batch"] * c["K"] * c["vocab"] > 64 * 16 * 151936:
            c["batch"] //= 2
        return c
    if kind == "verify":
        hkv, d = rng.choice([(8, 128), (8, 128), (4, 128), (2, 64)])
        c = dict(kind=kind, batch=_log(rng, 1, 64), K=rng.choice([4, 8, 13, 16, 24, 32]), vocab=_log(rng, 500, 160000),
                 dtype=rng.choice(["f32", "f32", "bf16"]), mix=rng.choice(sorted(MIXES)), layers=rng.choice([1, 1, 2, 8, 36]),
                 lo=rng.randint(1, 300), hi=500, hkv=hkv, d=d)
        while c["batch"] > 1 and (c["batch"] * c["K"] * c["vocab"] > 64 * 16 * 151936 or c["batch"] * c["layers"] > 256):
            c["batch"] //= 2
        return c
    if kind == "tables":
        new = rng.choice([1, _log(rng, 2, 32), _log(rng, 100, 16000)])
        c = dict(kind=kind, batch=_log(rng, 1, 4096), lo=rng.choice([0, 1, 50]), hi=_log(rng, 60, 8000),
                 new_lo=max(1, new // rng.choice([1, 8])), new_hi=new, ended=rng.choice([0, 5, 16, 29]),
                 short=rng.choice([0, 0, 1]))
        while c["batch"] > 1 and c["batch"] * (c["hi"] + c["new_hi"]) > 3000000:
            c["batch"] //= 2
        return c
    hq, hkv, d = rng.choice([(32, 8, 128), (28, 4, 128), (16, 8, 128), (4, 2, 64)])
    c = dict(kind=kind, rows=_log(rng, 1, 30000), layers=rng.choice([1, 1, 2, 8, 36]), fused=rng.randint(0, 1), hq=hq, hkv=hkv,
             d=d, skip=0)
    c["skip"] = rng.choice([0, c["rows"] // 3])
    while c["layers"] > 1 and c["rows"] * c["layers"] > 30000:
        c["layers"] //= 2
    if c["layers"] > 1:
        c["fused"] = 0
    return c


def _spread(n, lo, hi):
    """n whole numbers from lo to hi, evenly spaced."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _table_lengths(c):
    """Cached and new lengths of a tables case; new is -1 for a request that ended."""
    B = c["batch"]
    old, new = _spread(B, c["lo"], c["hi"]), _spread(B, c["new_lo"], c["new_hi"])
    new = [new[(i * 7 + 3) % B] for i in range(B)]
    old = [old[(i * 5 + 1) % B] if B % 5 else old[i] for i in range(B)]
    if c["ended"]:
        new = [-1 if i % c["ended"] == 2 % c["ended"] else n for i, n in enumerate(new)]
    return old, new


def work(case):
    c = case
    if c["kind"] == "sample":
        n = c["batch"] * c["K"]
        return {"bytes": n * c["vocab"] * (4 if c["dtype"] == "f32" else 2) + n * (8 + 4 * c["logprob"]),
                "flops": 4 * n * c["vocab"]}
    if c["kind"] == "verify":
        n = c["batch"] * c["K"]
        commit = 2 * c["batch"] * 4 * c["layers"] * c["hkv"] * c["d"] * 4   # about four rows appended per sequence
        return {"bytes": 2 * n * c["vocab"] * (4 if c["dtype"] == "f32" else 2) + 12 * n + commit, "flops": 8 * n * c["vocab"]}
    if c["kind"] == "tables":
        old, new = _table_lengths(c)
        slots = sum(max(n, 0) for n in new)
        entries = sum((o + P - 1) // P if n < 0 else n // P + 2 for o, n in zip(old, new))
        return {"bytes": 4 * slots + 12 * entries + 20 * c["batch"], "flops": 2 * slots}
    rows = (c["rows"] - c["skip"]) * c["layers"]
    return {"bytes": rows * 8 * c["hkv"] * c["d"] + 4 * c["rows"], "flops": rows}


# ---------------------------------------------------------------------------------------------------------------
# what a program holds before the call

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 7919 + 23)


def _logits(g, rows, V, kind, pad=0):
    """Logits rows.  peaked: a bulk of N(0, 2) and a head of 96 tokens whose logits fall off like a language model's, from
    a certain next token to a broad choice (a row in ten keeps a nucleus of thousands); flat: the bulk alone."""
    x = torch.randn((rows, V + pad), generator=g, device=DEV) * 2
    if kind == "peaked":
        n = min(96, V)
        # one place in each of n stretches of the vocabulary, so that no place is taken twice; ranks in random order
        wide = V // n
        at = torch.arange(n, device=DEV)[None] * wide + torch.randint(0, wide, (rows, n), generator=g, device=DEV)
        top = 15 + 11 * torch.rand((rows, 1), generator=g, device=DEV)
        fall = 0.5 + 2 * torch.rand((rows, 1), generator=g, device=DEV)
        rank = torch.rand((rows, n), generator=g, device=DEV).argsort(1).float() + 1
        x.scatter_(1, at, top - fall * rank.log() + 0.3 * torch.randn((rows, n), generator=g, device=DEV))
    return x


_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _filters(c):
    m = MIXES[c["mix"]]
    rows = [m[b % len(m)] for b in range(c["batch"])]
    col = lambda i, t: torch.tensor([r[i] for r in rows], dtype=t, device=DEV)  # noqa: E731
    return col(0, torch.float32), col(1, torch.int32), col(2, torch.float32), col(3, torch.float32)


def _own_step(**kw):
    from paper_2605_12825_amd import runtime as rt
    full = dict(batch=1, num_q_heads=8, num_kv_heads=8, head_dim=128, block_k=1, page_size=P, max_pages_per_seq=1,
                max_seq_len=P, num_pages=1)
    full.update(kw)
    return rt.DecodeStep(**full)


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = dict(case=c)
    if c["kind"] == "sample":
        B, K, V = c["batch"], c["K"], c["vocab"]
        s["logits"] = _logits(g, B * K, V, c["logits"], c["pad"]).to(_DTYPES[c["dtype"]]).view(B, K, V + c["pad"])
        s["filters"] = _filters(c)
        s["u"] = torch.rand((B, K), generator=g, device=DEV)
        s["tokens"] = torch.zeros((B, K), dtype=torch.int32, device=DEV)
        s["logprob"] = torch.zeros((B, K), device=DEV) if c["logprob"] else None
        if own:
            s["step"] = _own_step(batch=B, block_k=K, vocab=V)
        return s
    if c["kind"] == "verify":
        return _prepare_verify(s, c, g)
    if c["kind"] == "tables":
        return _prepare_tables(s, c, g)
    N, H, d, L = c["rows"], c["hkv"], c["d"], c["layers"]
    bits = lambda *shape: torch.randn(shape, generator=g, dtype=torch.bfloat16, device=DEV).view(torch.int16)  # noqa: E731
    pages = (N * 5 // 4 + P - 1) // P + 1
    s["k_pool"], s["v_pool"] = bits(L, pages, H, P, d), bits(L, pages, H, P, d)
    if c["fused"]:
        x = bits(N, c["hq"] + 2 * H, d)
        s["fused"] = x
        s["k"], s["v"] = x[None, :, c["hq"]:c["hq"] + H], x[None, :, c["hq"] + H:]
    else:
        s["k"], s["v"] = bits(L, N, H, d), bits(L, N, H, d)
    # slots as a page table deals them out: runs of up to a page, in random places
    runs = torch.randperm(pages, generator=g, device=DEV)[:(N + P - 1) // P]
    s["slots"] = (runs[:, None] * P + torch.arange(P, device=DEV)[None]).reshape(-1)[:N].to(torch.int32)
    s["count"] = torch.tensor([N - c["skip"]], dtype=torch.int32, device=DEV)
    if own:
        row = (c["hq"] + 2 * H) * d if c["fused"] else H * d
        s["step"] = _own_step(num_q_heads=H, num_kv_heads=H, head_dim=d, num_pages=pages, num_layers=L, vocab=0,
                              pool_strides=(pages * H * P * d, H * P * d, P * d, d), block_strides=(0, 0, row, d, N * row))
    return s


def _prepare_verify(s, c, g):
    B, K, V, L, H, d = c["batch"], c["K"], c["vocab"], c["layers"], c["hkv"], c["d"]
    ar = _logits(g, B * K, V, "peaked")
    df = torch.randn((B * K, V), generator=g, device=DEV).mul_(0.3).add_(ar)
    t = _DTYPES[c["dtype"]]
    ar, df = ar.to(t), df.to(t)
    s["filters"] = _filters(c)
    rows = [f.repeat_interleave(K) for f in s["filters"]]
    # drafts as a sampler of the diffusion view draws them
    w, Z = _weights(df, *rows)
    s["draft"] = _draw(w, Z, torch.rand((B * K,), generator=g, device=DEV))[0].view(B, K).to(torch.int32)
    del w, Z
    s["ar"], s["df"] = ar.view(B, K, V), df.view(B, K, V)
    s["u"] = torch.rand((B, K), generator=g, device=DEV)
    s["gumbel"] = -torch.empty((B, V), device=DEV).exponential_(generator=g).log()
    lens = torch.tensor(_spread(B, c["lo"], c["hi"]), dtype=torch.int32, device=DEV)
    slots = (c["hi"] + K + P - 1) // P
    pages = B * slots + 1
    perm = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    s["page_table"] = perm[:B * slots].view(B, slots).contiguous()
    bits = lambda *shape: torch.randn(shape, generator=g, dtype=torch.bfloat16, device=DEV).view(torch.int16)  # noqa: E731
    s["k_pool"], s["v_pool"] = bits(L, pages, H, P, d), bits(L, pages, H, P, d)
    s["k"], s["v"] = bits(L, B, K, H, d), bits(L, B, K, H, d)
    s["lens0"], s["seq_lens"] = lens, lens.clone()
    s["acc"], s["ncm"], s["anchor"] = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(3))
    s["tokens"] = torch.zeros((B, K), dtype=torch.int32, device=DEV)
    if own:
        s["step"] = _own_step(batch=B, num_q_heads=H, num_kv_heads=H, head_dim=d, block_k=K, max_pages_per_seq=slots,
                              max_seq_len=slots * P, num_pages=pages, vocab=V, num_layers=L,
                              pool_strides=(pages * H * P * d, H * P * d, P * d, d))
    return s


def _prepare_tables(s, c, g):
    B = c["batch"]
    old, new = _table_lengths(c)
    width = (max(o + max(n, 0) for o, n in zip(old, new)) + P - 1) // P + 2
    held = [(o + P - 1) // P for o in old]
    need = [(o + max(n, 0) + P - 1) // P - h for o, n, h in zip(old, new, held)]
    free = sum(need) // 2 if c["short"] else sum(need) + 37
    pages = sum(held) + free + 11
    perm = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    lens = torch.tensor(held, device=DEV)
    start = lens.cumsum(0) - lens
    col = torch.arange(width, device=DEV)[None]
    table = torch.where(col < lens[:, None], perm[(start[:, None] + col).clamp(max=pages - 1)], -1).to(torch.int32)
    ring = torch.full((pages,), -1, dtype=torch.int32, device=DEV)
    head = pages // 3
    at = (head + torch.arange(free, device=DEV)) % pages
    ring[at] = perm[sum(held):sum(held) + free]
    state = torch.tensor([head, free], dtype=torch.int32, device=DEV)
    s["start"] = torch.cat([table.reshape(-1), ring, state])
    s["now"] = s["start"].clone()
    s["page_table"] = s["now"][:B * width].view(B, width)
    s["ring"], s["state"] = s["now"][B * width:B * width + pages], s["now"][B * width + pages:]
    s["old"], s["new"] = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in (old, new))
    s["pages"], s["bound"] = pages, width * P
    s["granted"] = torch.zeros(B, dtype=torch.int32, device=DEV)
    s["starts"] = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    s["slots"] = torch.full((sum(max(n, 0) for n in new) + 5,), -1, dtype=torch.int32, device=DEV)
    if own:
        s["step"] = _own_step(batch=B, max_pages_per_seq=width, max_seq_len=width * P, num_pages=pages)
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass

def run(s):
    c = s["case"]
    if c["kind"] == "sample":
        if own:
            s["step"].sample_tokens(s["logits"], *s["filters"], s["u"], s["tokens"], s["logprob"],
                                    logits_stride_row=c["vocab"] + c["pad"])
        else:
            R, V = c["batch"] * c["K"], c["vocab"]
            w, Z = _weights(s["logits"].view(R, -1)[:, :V], *[f.repeat_interleave(c["K"]) for f in s["filters"]])
            token, lp = _draw(w, Z, s["u"].view(R))
            s["tokens"].copy_(token.view(s["tokens"].shape))
            if s["logprob"] is not None:
                s["logprob"].copy_(lp.view(s["logprob"].shape))
        return [s["tokens"]] + ([s["logprob"]] if s["logprob"] is not None else [])
    if c["kind"] == "verify":
        s["seq_lens"].copy_(s["lens0"])
        if own:
            s["step"].filtered_consensus_commit(s["ar"], s["df"], *s["filters"], s["draft"], s["u"], s["gumbel"], s["k"], s["v"],
                                                s["k_pool"], s["v_pool"], s["page_table"], s["seq_lens"], s["acc"], s["ncm"],
                                                s["tokens"], s["anchor"])
        else:
            _plain_verify(s, c)
        return [s["acc"], s["ncm"], s["tokens"], s["anchor"], s["seq_lens"], s["k_pool"], s["v_pool"]]
    if c["kind"] == "tables":
        s["now"].copy_(s["start"])
        if own:
            s["step"].update_page_tables(s["old"], s["new"], s["page_table"], s["ring"], s["state"], s["granted"], s["starts"],
                                         s["slots"])
        else:
            _plain_tables(s)
        return [s["page_table"], s["ring"], s["state"], s["granted"], s["starts"], s["slots"]]
    if own:
        s["step"].store_kv(s["k"], s["v"], s["slots"], s["k_pool"], s["v_pool"], s["count"])
    else:
        # rows that are not stored go to a spare row behind the pool's own
        slots = s["slots"].long()
        page, off = slots // P, slots % P
        use = (torch.arange(c["rows"], device=DEV) < s["count"])[:, None, None]
        for l in range(c["layers"]):
            for x, pool in ((s["k"], s["k_pool"]), (s["v"], s["v_pool"])):
                pool[l][page, :, off] = torch.where(use, x[l], pool[l][page, :, off])
    return [s["k_pool"], s["v_pool"]]


def _weights(x, T, top_k, top_p, min_p):
    """Weights exp((x - max) / T) of the tokens that the row's filters keep, 0 elsewhere, and their sum.  64 bits: a
    token next to a cut, or next to the uniform number, is decided by the last bits of sums over the vocabulary."""
    V = x.shape[1]
    x = x.float()
    x = torch.where(x.isnan(), -math.inf, x).clamp(max=BIG)
    greedy = ~(T > 0)
    T = torch.where(greedy, 1.0, T).double()[:, None]
    top_k = torch.where(greedy, 1, top_k).long()[:, None]
    top = x.amax(1, keepdim=True)
    w = torch.where(x > -math.inf, ((x.double() - top.double()) / T).exp(), 0.0)
    order = x.sort(dim=1, descending=True, stable=True).indices     # equal logits: the lower index first
    w = w.gather(1, order)
    rank = torch.arange(V, device=x.device)[None]
    w = torch.where((top_k > 0) & (rank >= top_k), 0.0, w)
    run_sum = w.cumsum(1)
    before = torch.cat([torch.zeros_like(run_sum[:, :1]), run_sum[:, :-1]], 1)
    p = top_p.double()[:, None]
    p = torch.where(greedy[:, None] | p.isnan(), 1.0, p)
    w = torch.where((p < 1) & (rank > 0) & (before >= p * run_sum[:, -1:]), 0.0, w)
    m = min_p.double()[:, None]
    m = torch.where(greedy[:, None] | m.isnan(), 0.0, m).clamp(max=1.0)
    w = torch.where(w >= m, w, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, w)
    return w, w.sum(1)


def _draw(w, Z, u):
    """The first token in index order whose running sum exceeds u times the sum, and its log-probability."""
    u = u.double().nan_to_num(0.0).clamp(0.0, ONE_BELOW)
    token = ((w.cumsum(1) > (u * Z)[:, None]) & (w > 0)).to(torch.uint8).argmax(1)
    lp = (w.gather(1, token[:, None])[:, 0] / Z).log()
    return torch.where(Z > 0, token, -1), torch.where(Z > 0, lp, -math.inf).float()


def _plain_verify(s, c):
    B, K, V = c["batch"], c["K"], c["vocab"]
    rows = [f.repeat_interleave(K) for f in s["filters"]]
    wp, Zp = _weights(s["ar"].view(B * K, V), *rows)
    wq, Zq = _weights(s["df"].view(B * K, V), *rows)
    Zp, Zq = Zp.view(B, K), Zq.view(B, K)
    x = s["draft"].long()
    inside = (x >= 0) & (x < V)
    at = x.clamp(0, V - 1).view(B * K, 1)
    px = wp.gather(1, at).view(B, K) / Zp
    qx = torch.where(Zq > 0, wq.gather(1, at).view(B, K) / Zq, 0.0)
    keep = inside & (s["u"].double() * qx < px)
    acc = keep.long().cumprod(1).sum(1)
    m = (acc + 1).clamp(max=K)
    j = acc.clamp(max=K - 1)
    row = torch.arange(B, device=DEV) * K + j
    p = wp[row] / Zp.gather(1, j[:, None])
    q = torch.where(Zq.gather(1, j[:, None]) > 0, wq[row] / Zq.gather(1, j[:, None]), 0.0)
    r = p - q
    r = torch.where((r > 0).any(1, keepdim=True), r, p)
    score = torch.where(r > 0, r.clamp(min=0).log() + s["gumbel"].double(), -math.inf)
    repl = torch.where((p > 0).any(1), score.argmax(1), -1)
    k = torch.arange(K, device=DEV)[None]
    tokens = torch.where(k < acc[:, None], x, torch.where(k == acc[:, None], repl[:, None], -1))
    s["acc"].copy_(acc)
    s["ncm"].copy_(m)
    s["tokens"].copy_(tokens)
    s["anchor"].copy_(torch.where(acc < K, repl, x[:, K - 1]))
    # the first m rows of every sequence's block enter the cache
    pos = s["lens0"].long()[:, None] + k
    page = s["page_table"].long().gather(1, pos // P)
    off = pos % P
    use = (k < m[:, None])[..., None, None]
    for l in range(c["layers"]):
        for new, pool in ((s["k"], s["k_pool"]), (s["v"], s["v_pool"])):
            pool[l][page, :, off] = torch.where(use, new[l], pool[l][page, :, off])
    s["seq_lens"].copy_(s["lens0"] + m)


def _plain_tables(s):
    table, ring, state = s["page_table"], s["ring"], s["state"]
    B, width = table.shape
    N, L, n = s["pages"], s["old"].long(), s["new"].long()
    head, free = state[0].long(), state[1].long()
    col = torch.arange(width, device=DEV)[None]
    mapped = (table >= 0) & (table < N)
    ended = n < 0
    first, last = L // P, (L + n - 1) // P
    torn = (L % P != 0) & ~mapped.gather(1, first.clamp(0, width - 1)[:, None])[:, 0] & (n > 0)
    valid = ~ended & (L >= 0) & (L + n <= s["bound"]) & ~torn
    missing = (valid & (n > 0))[:, None] & (col >= first[:, None]) & (col <= last[:, None]) & ~mapped
    count = missing.sum(1)
    total = count.cumsum(0)
    granted = valid & ((count == 0) | (total <= free))
    rank = (total - count)[:, None] + missing.cumsum(1) - 1
    page = ring[(head + rank.clamp(min=0)) % N]
    take = missing & granted[:, None]
    back = ended[:, None] & mapped
    order = back.sum(1).cumsum(0) - back.sum(1)
    place = (head + free + order[:, None] + back.cumsum(1) - 1) % N
    ring2 = torch.cat([ring, ring[:1]])
    ring2[torch.where(back, place, N).reshape(-1)] = table.reshape(-1)
    table.copy_(torch.where(take, page, torch.where(back, -1, table)))
    ring.copy_(ring2[:N])
    taken = torch.where(granted, count, 0).sum()
    state.copy_(torch.stack([(head + taken) % N, free - taken + back.sum()]))
    s["granted"].copy_(torch.where(granted, n, 0))
    s["starts"][1:] = s["granted"].cumsum(0)
    flat = torch.arange(s["slots"].numel(), device=DEV)
    b = torch.searchsorted(s["starts"][1:].contiguous(), flat.int(), right=True).clamp(max=B - 1)
    pos = L[b] + flat - s["starts"][b]
    slot = table[b, (pos // P).clamp(0, width - 1)] * P + pos % P
    s["slots"].copy_(torch.where(flat < s["starts"][-1], slot, s["slots"]))


# ---------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, with numpy on the host, one row or request after another

def exact(case, seed):
    if case["kind"] in ("sample", "verify") and case["batch"] * case["K"] * case["vocab"] > 6e7 and (
            case["mix"] in ("warm", "plain") or case.get("logits") == "flat"):
        return None        # wide cuts of hundreds of rows: half a minute here
    s = prepare(case, seed)
    c = s["case"]
    h = {k: v.cpu() for k, v in s.items() if isinstance(v, torch.Tensor)}
    f = [t.cpu().numpy() for t in s["filters"]] if "filters" in s else None
    h = {k: (v.float() if v.dtype in (torch.bfloat16, torch.float16) else v).numpy() for k, v in h.items()}
    s.clear()
    if c["kind"] == "sample":
        return _exact_sample(c, h, f)
    if c["kind"] == "verify":
        return _exact_verify(c, h, f)
    if c["kind"] == "tables":
        return _exact_tables(h, h["ring"].size)
    for t in range(c["rows"] - c["skip"]):
        page, off = divmod(int(h["slots"][t]), P)
        h["k_pool"][:, page, :, off] = h["k"][:, t]
        h["v_pool"][:, page, :, off] = h["v"][:, t]
    return [h["k_pool"], h["v_pool"]]


def _row(x, T, k, p, m):
    """Indices that a row's filters keep, ascending, and their weights."""
    x = x.astype(np.float64)
    x[np.isnan(x)] = -np.inf
    np.minimum(x, BIG, out=x)
    live = np.flatnonzero(x > -np.inf)
    if live.size == 0:
        return live, x[live]
    top = x.max()
    if not T > 0:
        return np.array([int(np.argmax(x))]), np.ones(1)
    T = float(T)
    k = int(k) if 0 < k < x.size else x.size
    p = float(p)
    cut_p = p < 1
    keep = live
    if k < live.size or cut_p:
        total = None if k < live.size else float(np.sum(np.exp((x[live] - top) / T)))
        size = min(live.size, k if k < live.size else 1024)
        while True:
            # everything at least as large as the size-th largest, in order
            edge = np.partition(x[live], live.size - size)[live.size - size]
            some = live[x[live] >= edge]
            some = some[np.lexsort((some, -x[some]))]
            mass = np.cumsum(np.exp((x[some[:k]] - top) / T))
            if total is None:
                total = float(mass[-1])
            if not cut_p:
                keep = some[:k]
                break
            n = int(np.searchsorted(mass, p * total, side="left")) + 1   # shortest prefix with at least that mass
            if n <= mass.size or size == live.size or k <= size:
                keep = some[:max(1, min(n, mass.size))]
                break
            size = min(live.size, size * 16)
    w = np.exp((x[keep] - top) / T)
    if m > 0:
        keep = keep[w >= min(float(m), 1.0)]
    keep = np.sort(keep)
    return keep, np.exp((x[keep] - top) / T)


def _exact_sample(c, h, f):
    B, K, V = c["batch"], c["K"], c["vocab"]
    tokens, lp = np.full((B, K), -1, np.int32), np.full((B, K), -np.inf)
    for b in range(B):
        for k in range(K):
            keep, w = _row(h["logits"][b, k, :V], *[a[b] for a in f])
            if not w.size:
                continue
            sums = np.cumsum(w)
            u = min(max(float(h["u"][b, k]), 0.0), ONE_BELOW)
            i = min(int(np.searchsorted(sums, u * sums[-1], side="right")), w.size - 1)
            tokens[b, k], lp[b, k] = keep[i], math.log(w[i] / sums[-1]) if w[i] > 0 else -np.inf
    return [tokens] + ([lp] if c["logprob"] else [])


def _exact_verify(c, h, f):
    B, K = c["batch"], c["K"]
    acc, ncm, anchor = (np.zeros(B, np.int32) for _ in range(3))
    tokens, lens = np.full((B, K), -1, np.int32), h["lens0"].copy()
    for b in range(B):
        for k in range(K):
            x = int(h["draft"][b, k])
            ip, wp = _row(h["ar"][b, k], *[a[b] for a in f])
            iq, wq = _row(h["df"][b, k], *[a[b] for a in f])
            p, q = np.zeros(c["vocab"]), np.zeros(c["vocab"])
            p[ip], q[iq] = wp / wp.sum(), wq / wq.sum()
            if float(h["u"][b, k]) * q[x] < p[x]:
                tokens[b, k] = anchor[b] = x
                acc[b] += 1
                continue
            r = p[ip] - q[ip]
            if not np.any(r > 0):
                r = p[ip]
            score = np.full(r.size, -np.inf)
            score[r > 0] = np.log(r[r > 0]) + h["gumbel"][b, ip[r > 0]].astype(np.float64)
            tokens[b, k] = anchor[b] = ip[int(np.argmax(score))] if r.size else -1
            break
        ncm[b] = min(acc[b] + 1, K)
        for i in range(ncm[b]):
            pos = int(lens[b]) + i
            page = h["page_table"][b, pos // P]
            h["k_pool"][:, page, :, pos % P] = h["k"][:, b, i]
            h["v_pool"][:, page, :, pos % P] = h["v"][:, b, i]
        lens[b] += ncm[b]
    return [acc, ncm, tokens, anchor, lens, h["k_pool"], h["v_pool"]]


def _exact_tables(h, N):
    table, ring, (head, free) = h["page_table"].copy(), h["ring"].copy(), [int(v) for v in h["state"]]
    B, width = table.shape
    granted, starts, slots = np.zeros(B, np.int32), np.zeros(B + 1, np.int32), h["slots"].copy()
    wanted, taken, back = 0, 0, []
    for b in range(B):
        L, n = int(h["old"][b]), int(h["new"][b])
        row = table[b]
        starts[b + 1] = starts[b]
        if n < 0:
            for e in range(width):
                if 0 <= row[e] < N:
                    back.append(row[e])
                    row[e] = -1
            continue
        if L < 0 or L + n > width * P or (n > 0 and L % P and not 0 <= row[L // P] < N):
            continue
        need = [e for e in range(L // P, (L + n + P - 1) // P) if not 0 <= row[e] < N] if n else []
        wanted += len(need)
        if need and wanted > free:
            continue
        for e in need:
            row[e] = ring[(head + taken) % N]
            taken += 1
        granted[b] = n
        for i in range(n):
            slots[starts[b] + i] = row[(L + i) // P] * P + (L + i) % P
        starts[b + 1] += n
    for i, page in enumerate(back):
        ring[(head + free + i) % N] = page
    return [table, ring, np.array([(head + taken) % N, free - taken + len(back)], np.int32), granted, starts, slots]
