"""Performance cases of the operators for drafts that branch and requests with rules of their own: attention of a tree of
drafted tokens over the paged cache, the greedy consensus of such a tree with its commit, and the rules (penalties for
repeated tokens, biases, allowed tokens) that a request's logits go through before a token is taken from them.

A case is a dict of plain values.  `kind` names the operator:

  attn     every node of a sequence's tree attends the cache, its ancestors and itself
  walk     from the root down to the child that holds the node's greedy token; the path's K/V rows enter the cache
  logits   repetition, presence and frequency penalties by a request's history and a node's path, biases, allowed tokens

A tree is given by parents[b][i]: the node that node i follows, -1 for the root (node 0, the anchor) and for unused nodes, which
see and follow the root alone.
`own` false: `run` computes in elementary torch operations; true: it calls the framework.  The consensus changes lengths:
it gets those of before the call back first, so that every pass is the same one.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
P = 16   # tokens per cache page

# (repetition, presence, frequency) of requests; sequence b takes entry b mod length
PENALTIES = [(1.1, 0.0, 0.0), (1.0, 0.5, 0.3), (1.0, 0.0, 0.0), (1.25, 0.4, 0.2), (0.9, -0.3, 0.1)]


def listed():
    h8, h28 = dict(hq=32, hkv=8, d=128), dict(hq=28, hkv=4, d=128)
    return [
        # the smallest call: a toy model's tree of 8 nodes, launches and latency
        dict(name="attn_tiny", kind="attn", batch=1, nodes=8, depth=4, used=0, lo=128, hi=128, splits=0, lse=1, hq=4, hkv=2, d=64),
        # an interactive user's tree over a middling context
        dict(name="attn_b1", kind="attn", batch=1, nodes=32, depth=8, used=0, lo=4096, hi=4096, splits=0, lse=0, **h8),
        # long contexts, small trees: the cache's stream
        dict(name="attn_long", kind="attn", batch=4, nodes=16, depth=6, used=0, lo=32768, hi=32768, splits=0, lse=0, **h8),
        # a serving batch with the largest trees: the matrix products
        dict(name="attn_batch", kind="attn", batch=64, nodes=64, depth=8, used=1, lo=1000, hi=2500, splits=0, lse=0, **h8),
        # contexts of very different lengths, shared out evenly
        dict(name="attn_ragged", kind="attn", batch=16, nodes=32, depth=8, used=1, lo=512, hi=8192, splits=-1, lse=0, **h28),
        # one request's tree, its path into the caches of 36 layers
        dict(name="walk_b1", kind="walk", batch=1, nodes=32, depth=8, vocab=128256, dtype="f32", pad=0, layers=36, lo=4096,
             hi=4096, hkv=8, d=128),
        # a serving batch's trees
        dict(name="walk_b64", kind="walk", batch=64, nodes=64, depth=8, vocab=151936, dtype="f32", pad=0, layers=1, lo=200,
             hi=500, hkv=8, d=128),
        # a middling batch, bf16 logits of a padded output head
        dict(name="walk_b8", kind="walk", batch=8, nodes=48, depth=6, vocab=151669, dtype="bf16", pad=267, layers=8, lo=100,
             hi=900, hkv=8, d=128),
        # the smallest call: one row of a toy vocabulary
        dict(name="logits_tiny", kind="logits", batch=1, rows=1, tree=0, vocab=512, dtype="f32", pad=0, lo=100, hi=100,
             penalties=1, bias=8, masked=1, inplace=0),
        # plain decoding of a serving batch: every request its penalties, some a grammar, bf16 logits of a padded head
        dict(name="logits_decode", kind="logits", batch=256, rows=1, tree=0, vocab=151669, dtype="bf16", pad=267, lo=50, hi=8000,
             penalties=1, bias=50, masked=4, inplace=0),
        # the rows of a batch's trees, each node with its own path
        dict(name="logits_tree", kind="logits", batch=32, rows=32, tree=1, vocab=151936, dtype="f32", pad=0, lo=500, hi=30000,
             penalties=1, bias=300, masked=3, inplace=0),
        # grammars alone, in place: what is not allowed is struck out
        dict(name="logits_grammar", kind="logits", batch=64, rows=16, tree=0, vocab=128256, dtype="f32", pad=0, lo=0, hi=0,
             penalties=0, bias=0, masked=1, inplace=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above, sizes over their logarithm, trimmed until it costs less than the largest."""
    kind = rng.choice(["attn", "attn", "attn", "walk", "walk", "logits", "logits"])
    if kind == "attn":
        hq, hkv, d = rng.choice([(32, 8, 128), (32, 8, 128), (28, 4, 128), (16, 8, 128), (4, 2, 64), (8, 8, 128), (40, 8, 128), (8, 2, 64)])
        n = rng.choice([1, 2, 5, 8, 13, 16, 24, 32, 33, 48, 63, 64])
        hi = _log(rng, 16, 40000)
        c = dict(kind=kind, batch=_log(rng, 1, 64), nodes=n, depth=rng.randint(1, min(n, 12)), used=rng.randint(0, 1),
                 lo=rng.choice([0, 1, hi // 8, hi // 2, hi]), hi=hi, splits=rng.choice([0, 0, 0, -1]), lse=rng.randint(0, 1),
                 hq=hq, hkv=hkv, d=d)
        while c["batch"] > 1 and (c["batch"] * hi * hq * max(n, 8) * d > 64 * 1750 * 32 * 64 * 128 or c["batch"] * hi * hkv * d > 4 * 32768 * 8 * 128):
            c["batch"] //= 2
        return c
    if kind == "walk":
        hkv, d = rng.choice([(8, 128), (8, 128), (4, 128), (2, 64)])
        n = rng.choice([1, 2, 7, 16, 24, 32, 48, 60, 64])
        c = dict(kind=kind, batch=_log(rng, 1, 64), nodes=n, depth=rng.randint(1, min(n, 12)), vocab=_log(rng, 500, 160000),
                 dtype=rng.choice(["f32", "f32", "bf16", "f16"]), pad=rng.choice([0, 0, rng.randint(1, 300)]),
                 layers=rng.choice([1, 1, 2, 8, 36]), lo=rng.randint(0, 300), hi=500, hkv=hkv, d=d)
        while c["batch"] > 1 and (c["batch"] * n * c["vocab"] > 64 * 64 * 151936 or c["batch"] * c["layers"] > 256):
            c["batch"] //= 2
        return c
    rows = rng.choice([1, 1, 1, 4, 8, 16, 32, 64])
    hi = _log(rng, 1, 30000)
    c = dict(kind=kind, batch=_log(rng, 1, 256), rows=rows, tree=rng.randint(0, 1), vocab=_log(rng, 500, 160000),
             dtype=rng.choice(["f32", "f32", "bf16", "f16"]), pad=rng.choice([0, 0, rng.randint(1, 300)]), lo=rng.choice([0, hi // 10, hi]),
             hi=hi, penalties=rng.choice([1, 1, 0]), bias=rng.choice([0, 10, 300]), masked=rng.choice([0, 1, 3]), inplace=0)
    if not c["penalties"]:
        c["bias"], c["inplace"], c["masked"] = 0, 1, 1
    while c["batch"] > 1 and c["batch"] * rows * c["vocab"] > 32 * 32 * 151936:
        c["batch"] //= 2
    return c


def _spread(n, lo, hi):
    """n whole numbers from lo to hi, evenly spaced, in a fixed mixed order."""
    v = [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]
    random.Random(n).shuffle(v)
    return v


def _bytes(c):
    return 4 if c["dtype"] == "f32" else 2


def work(case):
    c = case
    if c["kind"] == "attn":
        L = _spread(c["batch"], c["lo"], c["hi"])
        rows = c["batch"] * c["nodes"]
        return {"bytes": 4 * sum(L) * c["hkv"] * c["d"] + 4 * rows * (c["hq"] + c["hkv"]) * c["d"] + 4 * c["lse"] * rows * c["hq"],
                "flops": 4 * c["hq"] * c["d"] * c["nodes"] * (sum(L) + c["batch"] * c["depth"])}
    if c["kind"] == "walk":
        # the rows of the path, half the depth on average, and their K/V once read and once written
        n = c["batch"] * (c["depth"] + 1) / 2
        return {"bytes": n * c["vocab"] * _bytes(c) + 8 * n * c["layers"] * c["hkv"] * c["d"] + 8 * c["batch"] * c["nodes"],
                "flops": n * c["vocab"]}
    n = c["batch"] * c["rows"]
    tight = (n // c["masked"]) if c["masked"] else 0        # rows with a grammar: one logit in 32 is looked at
    value = c["vocab"] * _bytes(c)
    read = (n - tight) * value * (0 if c["inplace"] else 1) + tight * (value / 32 if not c["inplace"] else 0) + tight * c["vocab"] / 8
    write = (tight if c["inplace"] else n) * value
    return {"bytes": read + write + 4 * sum(_spread(c["batch"], c["lo"], c["hi"])) * c["penalties"], "flops": 4 * n * c["vocab"]}


# ---------------------------------------------------------------------------------------------------------------
# what a program holds before the call

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 7919 + 37)


_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _trees(batch, nodes, depth, used, seed):
    """Parents and levels of random trees of at most `depth` levels, and a path from the root in each: (parents, paths).
    `used`: every other tree leaves some of its nodes unused."""
    rng = random.Random(seed * 31 + 7)
    parents, paths = [], []
    for b in range(batch):
        n = rng.randint(max(1, nodes // 2), nodes) if used and b % 2 else nodes
        up, level = [-1], [0]
        for i in range(1, n):
            # the first nodes make a chain as deep as the tree may be; the others follow an early node or the last one
            k = i - 1 if i < depth else min(rng.randrange(i), rng.randrange(i))
            while level[k] + 1 >= depth and k > 0:
                k = up[k]
            ok = level[k] + 1 < depth
            up.append(k if ok else -1)
            level.append(level[k] + 1 if ok else 0)
        path = [0]
        for _ in range(rng.randint(0, depth - 1)):
            below = [i for i in range(1, n) if up[i] == path[-1]]
            if not below:
                break
            path.append(rng.choice(below))
        parents.append(up + [-1] * (nodes - n))
        paths.append(path)
    return parents, paths


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _own_step(**kw):
    from paper_2605_12825_amd import runtime as rt
    full = dict(batch=1, num_q_heads=8, num_kv_heads=8, head_dim=128, block_k=1, page_size=P, max_pages_per_seq=1,
                max_seq_len=P, num_pages=1)
    full.update(kw)
    return rt.DecodeStep(**full)


def _paged(s, c, g, room):
    """A paged cache whose pages lie anywhere, room for `room` more tokens a sequence."""
    B, H, d = c["batch"], c["hkv"], c["d"]
    lens = _spread(B, c["lo"], c["hi"])
    slots = (c["hi"] + room + P - 1) // P
    held = [(n + room + P - 1) // P for n in lens]
    pages = sum(held) + 1
    perm = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    n = torch.tensor(held, device=DEV)
    start = n.cumsum(0) - n
    col = torch.arange(slots, device=DEV)[None]
    s["page_table"] = torch.where(col < n[:, None], perm[(start[:, None] + col).clamp(max=pages - 1)], -1).to(torch.int32)
    s["lens0"] = _i32(lens)
    s["seq_lens"] = s["lens0"].clone()
    layers = c.get("layers", 1)
    normal = lambda *shape: torch.randn(shape, generator=g, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    s["k_pool"], s["v_pool"] = normal(layers, pages, H, P, d), normal(layers, pages, H, P, d)
    return pages, slots, normal


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = dict(case=c)
    if c["kind"] == "attn":
        B, N, H, d = c["batch"], c["nodes"], c["hkv"], c["d"]
        parents, _ = _trees(B, N, c["depth"], c["used"], seed)
        s["parents"] = _i32(parents)
        pages, slots, normal = _paged(s, c, g, 0)
        s["q"], s["k"], s["v"] = normal(B, N, c["hq"], d), normal(B, N, H, d), normal(B, N, H, d)
        s["out"] = torch.zeros((B, N, c["hq"], d), dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.zeros((B, c["hq"], N), device=DEV) if c["lse"] else None
        if own:
            s["step"] = _own_step(batch=B, num_q_heads=c["hq"], num_kv_heads=H, head_dim=d, max_pages_per_seq=max(slots, 1),
                                  max_seq_len=c["hi"], num_pages=pages, num_splits=c["splits"])
        return s
    if c["kind"] == "walk":
        return _prepare_walk(s, c, g, seed)
    return _prepare_logits(s, c, g, seed)


def _prepare_walk(s, c, g, seed):
    B, N, V, L, H, d = c["batch"], c["nodes"], c["vocab"], c["layers"], c["hkv"], c["d"]
    parents, paths = _trees(B, N, c["depth"], 0, seed)
    s["parents"] = _i32(parents)
    s["tokens"] = torch.randint(0, V, (B, N), generator=g, device=DEV).to(torch.int32)
    x = torch.randn((B * N, V + c["pad"]), generator=g, device=DEV).mul_(2)
    # every row has a certain next token: on the path the next node's, elsewhere any
    sure = torch.randint(0, V, (B, N), generator=g, device=DEV)
    at = [(b, p[i], p[i + 1]) for b, p in enumerate(paths) for i in range(len(p) - 1)]
    if at:
        b, i, j = torch.tensor(at, device=DEV).T
        sure[b, i] = s["tokens"][b, j].long()
    x.scatter_(1, sure.view(-1, 1), 16 + 4 * torch.rand((B * N, 1), generator=g, device=DEV))
    s["logits"] = x.to(_DTYPES[c["dtype"]]).view(B, N, V + c["pad"])
    del x
    pages, slots, normal = _paged(s, c, g, c["depth"])
    s["k"], s["v"] = normal(L, B, N, H, d), normal(L, B, N, H, d)
    s["acc"], s["ncm"], s["anchor"] = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(3))
    s["path"], s["emitted"] = (torch.zeros((B, N), dtype=torch.int32, device=DEV) for _ in range(2))
    if own:
        s["step"] = _own_step(batch=B, num_q_heads=H, num_kv_heads=H, head_dim=d, max_pages_per_seq=slots, max_seq_len=slots * P,
                              num_pages=pages, vocab=V, num_layers=L, pool_strides=(pages * H * P * d, H * P * d, P * d, d))
    return s


def _prepare_logits(s, c, g, seed):
    B, R, V = c["batch"], c["rows"], c["vocab"]
    t = _DTYPES[c["dtype"]]
    s["logits"] = torch.randn((B, R, V + c["pad"]), generator=g, device=DEV).mul_(3).to(t)
    s["out"] = s["logits"] if c["inplace"] else torch.zeros((B, R, V + c["pad"]), dtype=t, device=DEV)
    # text repeats itself: tokens thin out as they do in a language
    words = lambda *shape: (V * torch.rand(shape, generator=g, device=DEV) ** 4).long().clamp(max=V - 1).to(torch.int32)  # noqa: E731
    width = max(c["hi"], 1)
    lens = _spread(B, c["lo"], c["hi"])
    s["history"], s["history_lens"] = words(B, width), _i32(lens)
    s["prompt_lens"] = _i32([n * 3 // 5 for n in lens])
    s["tokens"] = words(B, R)
    s["parents"] = _i32(_trees(B, R, min(R, 8), 0, seed)[0]) if c["tree"] else None
    pen = [PENALTIES[b % len(PENALTIES)] for b in range(B)]
    s["penalties"] = [torch.tensor([p[i] for p in pen], device=DEV) if c["penalties"] else None for i in range(3)]
    counts = [c["bias"] if b % 3 == 0 else 0 for b in range(B)]
    s["bias_starts"] = _i32([sum(counts[:b]) for b in range(B + 1)]) if c["bias"] else None
    total = sum(counts)
    # a request's biased tokens lie in a stretch each of the vocabulary, so that none comes twice
    wide = V // max(c["bias"], 1)
    place = torch.arange(total, device=DEV) % max(c["bias"], 1)
    s["bias_tokens"] = (place * wide + torch.randint(0, wide, (total,), generator=g, device=DEV)).to(torch.int32) if c["bias"] else None
    s["bias_values"] = torch.randn((total,), generator=g, device=DEV) * 5 if c["bias"] else None
    s["masks"] = s["mask_rows"] = None
    if c["masked"]:
        # every row of every masked-th sequence has its own mask of allowed tokens, one in 32 of them
        who = [b for b in range(B) if b % c["masked"] == 0]
        bits = torch.randint(-2 ** 31, 2 ** 31, (5, len(who) * R, (V + 31) // 32), generator=g, device=DEV)
        s["masks"] = (bits[0] & bits[1] & bits[2] & bits[3] & bits[4]).to(torch.int32)
        rows = torch.full((B, R), -1, dtype=torch.int32, device=DEV)
        rows[who] = torch.arange(len(who) * R, device=DEV).view(-1, R).to(torch.int32)
        s["mask_rows"] = rows
    if own:
        from paper_2605_12825_amd import runtime as rt
        s["step"] = _own_step(batch=B, vocab=V)
        use = c["penalties"]
        s["rules"] = rt.LogitRules(history=s["history"] if use else None, history_lens=s["history_lens"] if use else None,
                                   prompt_lens=s["prompt_lens"] if use else None, repetition=s["penalties"][0],
                                   presence=s["penalties"][1], frequency=s["penalties"][2], bias_starts=s["bias_starts"],
                                   bias_tokens=s["bias_tokens"], bias_values=s["bias_values"], masks=s["masks"],
                                   mask_rows=s["mask_rows"])
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass

def run(s):
    c = s["case"]
    if c["kind"] == "attn":
        if own:
            s["step"].tree_attn(s["parents"], s["q"], s["k"], s["v"], s["k_pool"][0], s["v_pool"][0], s["page_table"], s["seq_lens"],
                                s["out"], s["lse"])
        else:
            _plain_attn(s, c)
        return [s["out"]] + ([s["lse"]] if c["lse"] else [])
    if c["kind"] == "walk":
        s["seq_lens"].copy_(s["lens0"])
        if own:
            s["step"].tree_consensus_commit(s["logits"], s["parents"], s["tokens"], s["k"], s["v"], s["k_pool"], s["v_pool"],
                                            s["page_table"], s["seq_lens"], s["acc"], s["ncm"], s["path"], s["emitted"],
                                            s["anchor"], max_path=c["depth"], logits_stride_row=c["vocab"] + c["pad"])
        else:
            _plain_walk(s, c)
        return [s["acc"], s["ncm"], s["path"], s["emitted"], s["anchor"], s["seq_lens"], s["k_pool"], s["v_pool"]]
    if own:
        s["step"].process_logits(s["logits"], s["rules"], tokens=s["tokens"] if c["penalties"] else None, parents=s["parents"],
                                 out=s["out"], logits_stride_row=c["vocab"] + c["pad"], out_stride_row=c["vocab"] + c["pad"])
    else:
        _plain_logits(s, c)
    return [s["out"]]


def _ancestors(parents):
    """[B, N, N]: whether node j is on the path from the root to node i, i itself included; for unused nodes the root alone."""
    B, N = parents.shape
    i = torch.arange(N, device=parents.device)
    up = parents.long()
    up = torch.where((up >= 0) & (up < i[None]), up, -1)
    step = (up[:, :, None] == i) | (i[:, None] == i)
    on = torch.linalg.matrix_power(step.double(), max(N - 1, 1)) > 0
    return torch.where(on[:, :, :1], on, i == 0)


def _plain_attn(s, c):
    B, N, Hq, H, d = c["batch"], c["nodes"], c["hq"], c["hkv"], c["d"]
    G, S = Hq // H, c["hi"]
    pos = torch.arange(S, device=DEV)
    page = s["page_table"].long().clamp(min=0)[:, pos // P]
    rows = lambda pool, new: torch.cat([pool[0][page, :, pos % P].float(), new.float()], 1).transpose(1, 2).contiguous()  # noqa: E731
    k, v = rows(s["k_pool"], s["k"]), rows(s["v_pool"], s["v"])                                  # [B, H, S + N, d]
    q = s["q"].float().view(B, N, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * N, d).contiguous()
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d)
    seen = torch.cat([(pos < s["seq_lens"].long()[:, None])[:, None].expand(B, N, S), _ancestors(s["parents"])], 2)
    score = score.view(B, H, G, N, S + N).masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(4, keepdim=True)
    w = score.sub_(top).exp_()
    total = w.sum(4, keepdim=True)
    o = torch.matmul(w.view(B, H, G * N, S + N), v).view(B, H, G, N, d) / total
    s["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(B, N, Hq, d))
    if c["lse"]:
        s["lse"].copy_((top + total.log())[..., 0].reshape(B, Hq, N))


def _plain_walk(s, c):
    B, N, V = c["batch"], c["nodes"], c["vocab"]
    sure = s["logits"][..., :V].float().argmax(2)
    i = torch.arange(N, device=DEV)
    up, token = s["parents"].long(), s["tokens"].long()
    follows = (up >= 0) & (up < i)
    right = follows & (token == sure.gather(1, up.clamp(min=0)))
    # of siblings with the same token the first
    twin = (up[:, :, None] == up[:, None, :]) & (token[:, :, None] == token[:, None, :]) & (i[:, None] > i)
    right = right & ~(twin & right[:, None, :]).any(2)
    right[:, 0] = True
    on = _ancestors(s["parents"])
    level = on.sum(2) - 1
    kept = ~(on & ~right[:, None, :]).any(2) & on[:, i, i] & (level < c["depth"])
    m = kept.sum(1)
    at = torch.where(kept, level, N)
    put = lambda x: torch.full((B, N + 1), -1, dtype=torch.long, device=DEV).scatter_(1, at, x)[:, :N]  # noqa: E731
    path, emitted = put(i.expand(B, N).contiguous()), put(sure)
    s["acc"].copy_(m - 1)
    s["ncm"].copy_(m)
    s["path"].copy_(path)
    s["emitted"].copy_(emitted)
    s["anchor"].copy_(emitted.gather(1, m[:, None] - 1)[:, 0])
    k = torch.arange(c["depth"], device=DEV)[None]
    pos = s["lens0"].long()[:, None] + k
    page, off = s["page_table"].long().gather(1, pos // P), pos % P
    use = (k < m[:, None])[None, :, :, None, None]
    b = torch.arange(B, device=DEV)[:, None]
    for new, pool in ((s["k"], s["k_pool"]), (s["v"], s["v_pool"])):
        pool[:, page, :, off] = torch.where(use, new[:, b, path[:, :c["depth"]].clamp(min=0)], pool[:, page, :, off].movedim(2, 0)).movedim(0, 2)
    s["seq_lens"].copy_(s["lens0"] + m)


def _plain_logits(s, c):
    B, R, V = c["batch"], c["rows"], c["vocab"]
    x = s["logits"][..., :V].float()
    if c["penalties"]:
        pos = torch.arange(s["history"].shape[1], device=DEV)
        used, prompt = pos < s["history_lens"][:, None], pos < s["prompt_lens"][:, None]
        h = s["history"].long()
        count = lambda take: torch.zeros((B, V + 1), device=DEV).scatter_add_(1, torch.where(take, h, V), torch.ones_like(h, dtype=torch.float32))  # noqa: E731
        chain = s["parents"] if s["parents"] is not None else (torch.arange(R, device=DEV, dtype=torch.int32) - 1).expand(B, R)
        on = _ancestors(chain)
        out = count(used & ~prompt)[:, None].repeat(1, R, 1)
        out.scatter_add_(2, torch.where(on, s["tokens"].long()[:, None, :], V), torch.ones((B, R, R), device=DEV))
        out = out[..., :V]
        seen = (out > 0) | (count(used & prompt)[:, None, :V] > 0)
        rep, pres, freq = (t[:, None, None] for t in s["penalties"])
        x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
        x = x - freq * out - pres * (out > 0)
    if c["bias"]:
        n = s["bias_starts"].long()
        owner = torch.searchsorted(n[1:].contiguous(), torch.arange(s["bias_tokens"].numel(), device=DEV), right=True)
        add = torch.zeros((B, V), device=DEV)
        add[owner, s["bias_tokens"].long()] = s["bias_values"]
        x = x + add[:, None]
    if c["masked"]:
        bit = (s["masks"][:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
        allowed = bit.view(s["masks"].shape[0], -1)[:, :V].bool()
        row = s["mask_rows"].long()
        x = torch.where((row < 0)[..., None] | allowed[row.clamp(min=0)], x, -math.inf)
    s["out"][..., :V].copy_(x)


# ---------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, with numpy on the host, one sequence after another

def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    h = {k: (v.float() if v.dtype in (torch.bfloat16, torch.float16) else v).cpu().numpy() for k, v in s.items() if isinstance(v, torch.Tensor)}
    h["penalties"] = [None if t is None else t.cpu().numpy().astype(np.float64) for t in s.get("penalties", [])]
    s.clear()
    return {"attn": _exact_attn, "walk": _exact_walk, "logits": _exact_logits}[c["kind"]](c, h)


def _path(up, i):
    """The nodes from the root down to i; of an unused node the root."""
    path = [i]
    while 0 <= up[path[-1]] < path[-1]:
        path.append(int(up[path[-1]]))
    return path[::-1] if path[-1] == 0 else [0]


def _exact_attn(c, h):
    B, N, Hq, H, d = c["batch"], c["nodes"], c["hq"], c["hkv"], c["d"]
    G = Hq // H
    out, lse = np.zeros((B, N, Hq, d)), np.zeros((B, Hq, N))
    for b in range(B):
        L = int(h["seq_lens"][b])
        pages = h["page_table"][b, :(L + P - 1) // P]
        hidden = np.ones((N, N), bool)
        for i in range(N):
            hidden[i, _path(h["parents"][b], i)] = False
        for n in range(H):
            k, v = (np.concatenate([h[pool][0][pages, n].reshape(-1, d)[:L], h[new][b, :, n]]).astype(np.float64)
                    for pool, new in (("k_pool", "k"), ("v_pool", "v")))
            x = h["q"][b, :, n * G:(n + 1) * G].astype(np.float64).reshape(N * G, d) @ k.T / math.sqrt(d)
            x[:, L:][np.repeat(hidden, G, axis=0)] = -np.inf
            top = x.max(1, keepdims=True)
            np.exp(np.subtract(x, top, out=x), out=x)
            total = x.sum(1, keepdims=True)
            out[b, :, n * G:(n + 1) * G] = (x @ v / total).reshape(N, G, d)
            lse[b, n * G:(n + 1) * G] = (top + np.log(total)).reshape(N, G).T
    return [out] + ([lse] if c["lse"] else [])


def _exact_walk(c, h):
    B, N, V = c["batch"], c["nodes"], c["vocab"]
    acc, ncm, anchor = (np.zeros(B, np.int32) for _ in range(3))
    path, emitted = (np.full((B, N), -1, np.int32) for _ in range(2))
    lens = h["lens0"].copy()
    for b in range(B):
        node, m = 0, 0
        while True:
            t = int(np.argmax(h["logits"][b, node, :V]))
            path[b, m], emitted[b, m], anchor[b] = node, t, t
            m += 1
            below = [i for i in range(node + 1, N) if h["parents"][b, i] == node and h["tokens"][b, i] == t]
            if m == c["depth"] or not below:
                break
            node = below[0]
        acc[b], ncm[b] = m - 1, m
        for i in range(m):
            pos = int(lens[b]) + i
            page = h["page_table"][b, pos // P]
            h["k_pool"][:, page, :, pos % P] = h["k"][:, b, path[b, i]]
            h["v_pool"][:, page, :, pos % P] = h["v"][:, b, path[b, i]]
        lens[b] += m
    return [acc, ncm, path, emitted, anchor, lens, h["k_pool"].astype(np.float64), h["v_pool"].astype(np.float64)]


def _exact_logits(c, h):
    B, R, V = c["batch"], c["rows"], c["vocab"]
    out = h["out"].astype(np.float64)
    for b in range(B):
        n, n0 = int(h["history_lens"][b]), int(h["prompt_lens"][b])
        text = h["history"][b]
        prompt, written = np.bincount(text[:n0], minlength=V), np.bincount(text[n0:n], minlength=V)
        for r in range(R):
            x = h["logits"][b, r, :V].astype(np.float64)
            if c["penalties"]:
                rep, pres, freq = (float(t[b]) for t in h["penalties"])
                times = written.copy()
                for i in (_path(h["parents"][b], r) if c["tree"] else range(r + 1)):
                    times[h["tokens"][b, i]] += 1
                at = np.flatnonzero((times > 0) | (prompt > 0))
                y = x[at]
                y = np.where(y > 0, y / rep, y * rep)
                x[at] = y - freq * times[at] - pres * (times[at] > 0)
            if c["bias"]:
                i, j = int(h["bias_starts"][b]), int(h["bias_starts"][b + 1])
                x[h["bias_tokens"][i:j]] += h["bias_values"][i:j].astype(np.float64)
            if c["masked"] and h["mask_rows"][b, r] >= 0:
                words = np.ascontiguousarray(h["masks"][h["mask_rows"][b, r]])
                x[np.unpackbits(words.view(np.uint8), bitorder="little")[:V] == 0] = -np.inf
            out[b, r, :V] = x
    return [out]
