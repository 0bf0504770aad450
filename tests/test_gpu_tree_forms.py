"""GPU tests of the tree operators' further forms, each of which asserts that its case reaches it: attention at every wave count, start order,
partition, kind of load and number of row groups; consensus level by level and by whole scans, every size of a workgroup's piece; rows of
which a mask leaves nothing; strided rows, other pages, the largest vocabulary; calls that are refused."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_trees import LSE_TOL, U, _TYPES, _bits, _cache, _check_attn, _f, _rt, _tree
from test_tree_routes_cpu import attn_form, consensus_form

pytestmark = pytest.mark.gpu


class _Rows:
    """Logits on the device as the oracle takes them, a row at a time."""

    def __init__(self, x, V):
        self.x, self.shape = x, (x.shape[0], x.shape[1], V)

    def __getitem__(self, at):
        return self.x[at][:self.shape[2]].float().cpu().numpy()


def _logits(seed, B, N, V, parents, tokens, kind, pad=0, offset=0, stop=0.15):
    """Rows of small numbers with one large one each: where a path goes on the next node's token, elsewhere any.  A path ends at its
    leaves, and at a node with probability `stop`.  Padding is larger than everything.  Also the planted paths."""
    rng = np.random.default_rng(seed)
    flat = torch.randn(B * N * (V + pad) + offset, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(_TYPES[kind])
    x = flat[offset:].view(B, N, V + pad)
    x[..., V:] = 50.0
    sure, paths = rng.integers(0, V, (B, N)), []
    for b in range(B):
        node, path = 0, [0]
        while True:
            below = [i for i in range(node + 1, N) if parents[b, i] == node and 0 <= tokens[b, i] < V]
            if not below or rng.random() < stop:
                break
            child = int(rng.choice(below))
            sure[b, node] = tokens[b, child]
            node = child
            path.append(node)
        paths.append(path)
    at = torch.from_numpy(sure).cuda()[..., None]
    x.scatter_(2, at, torch.full(at.shape, 12.0, dtype=x.dtype, device="cuda"))
    return rng, x, paths


def _trees(seed, B, N, depth, V):
    rng = np.random.default_rng(seed)
    parents = np.array([_tree(rng, N, depth, 0.1) for _ in range(B)], np.int64).astype(np.int32)
    return parents, rng.integers(0, V, (B, N)).astype(np.int32)


def _consensus(x, V, parents, tokens, max_path, kv=None, table=None, lens=None, strides=None, views=None):
    """The call and the oracle's answer, compared.  kv: numpy rows [layers, B, N, H, d] and pools; `views`: where the rows lie on the
    device instead, with the step's strides."""
    rt, (B, N), P = _rt(), parents.shape, 16 if kv is None else kv["kp"].shape[3]
    H, d, layers = (1, 64, 1) if kv is None else (kv["k"].shape[3], kv["k"].shape[4], kv["k"].shape[0])
    step = rt.DecodeStep(batch=B, num_q_heads=H, num_kv_heads=H, head_dim=d, block_k=1, page_size=P, max_pages_per_seq=1 if table is None else table.shape[1],
                         max_seq_len=0, vocab=V, num_layers=layers, num_pages=1 if kv is None else kv["kp"].shape[1], block_strides=strides,
                         pool_strides=None if kv is None else (kv["kp"].shape[1] * H * P * d, H * P * d, P * d, d))
    i32 = dict(dtype=torch.int32, device="cuda")
    r = {n: torch.full((B,), -7, **i32) for n in ("accept_len", "num_committed", "next_anchor")}
    r.update({n: torch.full((B, N), -7, **i32) for n in ("path_nodes", "out_tokens")})
    up = rt.to_device_bits
    dv = {k: up(v) for k, v in (kv or {}).items()}
    if views:
        dv["k"], dv["v"] = views
    t, l = (None, None) if table is None else (up(table), up(lens))
    step.tree_consensus_commit(x, up(parents), up(tokens), dv.get("k"), dv.get("v"), dv.get("kp"), dv.get("vp"), t, l, r["accept_len"], r["num_committed"],
                               r["path_nodes"], r["out_tokens"], r["next_anchor"], max_path=max_path, logits_stride_row=x.shape[2])
    torch.cuda.synchronize()
    args = {}
    if kv:
        kp, vp, n = kv["kp"].copy(), kv["vp"].copy(), lens.copy()
        args = dict(k_blk_ar=kv["k"], v_blk_ar=kv["v"], k_pool=kp, v_pool=vp, page_table=table, seq_lens=n)
    want = oracle.tree_consensus_commit(_Rows(x, V), parents, tokens, max_path or N, **args)
    for k, v in r.items():
        np.testing.assert_array_equal(v.cpu().numpy(), want[k], err_msg=k)
    assert step.device_error() == want["status"]
    if kv:
        for k, v in ((dv["kp"], kp), (dv["vp"], vp), (l, n)):
            np.testing.assert_array_equal(rt.bits_to_numpy(k), v)
    step.close()
    return want


def _kv(rng, layers, B, N, lens, room, P=16, H=2, d=64):
    kp, vp, table = _cache(rng, B, H, d, lens, P, room=room, layers=layers)
    return dict(kp=kp, vp=vp, k=_bits(rng, layers, B, N, H, d), v=_bits(rng, layers, B, N, H, d)), table


# (batch, nodes, depth, vocabulary, longest path): a few rows, scanned; the last two are walked, with small and with large pieces
_DEAD = [(12, 30, 9, 5000, None, ("scan", 2048)), (12, 30, 9, 5000, 4, ("scan", 2048)), (40, 64, 9, 40000, 5, ("walk", 2048)),
         (64, 40, 9, 70000, 6, ("walk", 8192))]


@pytest.mark.parametrize("B,N,depth,V,max_path,form", _DEAD)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_a_row_of_which_nothing_is_left_ends_the_path(B, N, depth, V, max_path, form, kind):
    """At the root, on the way and at the last node, with children that hold token 0 (and -1) below it: none is followed or committed, and
    there is no next anchor.  One logit that is left, the lowest number of the type or a NaN among -inf, is a token as any."""
    assert consensus_form(B, N, V, max_path, kind) == form
    parents, tokens = _trees(B + V, B, N, depth, V)
    rng, x, paths = _logits(B, B, N, V, parents, tokens, kind, stop=0.02)
    dead, alive = {}, {}
    for b in range(B):
        if b % 4 == 3:
            continue
        path = paths[b][:max_path]
        node = (path[0], path[len(path) // 2], path[-1])[b % 3]
        x[b, node] = -torch.inf
        for i in np.flatnonzero(parents[b] == node):
            tokens[b, i] = (0, -1)[i % 2] if i > node else tokens[b, i]
        if b % 5 == 4:   # something is left
            v, value = int(rng.integers(1, V)), (float("nan"), torch.finfo(_TYPES[kind]).min)[b % 2]
            x[b, node, v] = value
            alive[b] = v
        else:
            dead[b] = node
    lens = rng.integers(0, 50, B).astype(np.int32)
    kv, table = _kv(rng, 2, B, N, lens, N)
    want = _consensus(x, V, parents, tokens, max_path, kv, table, lens)
    assert dead and alive and want["status"] == 0
    ended = [b for b, node in dead.items() if want["path_nodes"][b, want["accept_len"][b]] == node]
    assert len(ended) > len(dead) // 2
    for b in range(B):
        assert (want["next_anchor"][b] == -1) == (b in ended), b
    for b in ended:
        assert want["out_tokens"][b, want["accept_len"][b]] == 0 and want["num_committed"][b] == want["accept_len"][b] + 1


# ---------------------------------------------------------------------------------------------------------------
# consensus

@pytest.mark.parametrize("kind,B,N,depth,V,max_path,pad,offset,form", [
    ("f32", 24, 64, 12, 50001, 8, 0, 0, ("walk", 2048)), ("f32", 24, 64, 12, 50001, 7, 3, 1, ("walk", 2048)), ("bf16", 24, 64, 12, 100003, 8, 5, 3, ("walk", 2048)),
    ("f16", 30, 64, 9, 90001, 2, 0, 1, ("walk", 2048)), ("f32", 40, 64, 4, 20011, 1, 1, 2, ("walk", 2048)),
    ("f32", 64, 64, 12, 70001, 8, 2, 1, ("walk", 8192)), ("bf16", 64, 64, 14, 70001, 12, 0, 0, ("walk", 8192)), ("f16", 64, 64, 12, 70001, 6, 267, 5, ("walk", 8192)),
    ("f32", 64, 64, 64, 120001, 32, 0, 0, ("walk", 8192)), ("bf16", 64, 48, 6, 66001, 6, 3, 7, ("walk", 8192)),
    ("f32", 16, 33, 9, 70001, None, 1, 0, ("scan", 8192)), ("bf16", 16, 33, 9, 70001, None, 3, 1, ("scan", 4096)), ("f16", 40, 64, 20, 20011, 19, 0, 3, ("scan", 4096)),
    ("f32", 24, 16, 5, 3001, 5, 0, 1, ("scan", 2048)), ("bf16", 24, 16, 5, 3001, 5, 1, 0, ("scan", 2048)),
])
def test_paths_by_every_form(kind, B, N, depth, V, max_path, pad, offset, form):
    """Paths of every length up to the limit and past it, rows at odd places, K/V rows into two layers' caches; sequences without a page for
    what they would append keep their caches and lengths."""
    assert consensus_form(B, N, V, max_path, kind) == form
    parents, tokens = _trees(V + N, B, N, depth, V)
    if depth == 64:   # chains with side branches: paths of all lengths
        parents = np.array([[-1] + [max(0, i - 1) if i % 9 or b % 2 else max(0, i - 4) for i in range(1, N)] for b in range(B)], np.int32)
    rng, x, paths = _logits(V, B, N, V, parents, tokens, kind, pad, offset, stop=1.2 / depth if depth > 2 else 0.3)
    lens = rng.integers(0, 60, B).astype(np.int32)
    kv, table = _kv(rng, 2, B, N, lens, N)
    table[3, (lens[3] + 15) // 16:] = -1               # no page to go on in
    table[7, lens[7] // 16] = kv["kp"].shape[1]        # a page that the pool does not have
    lens[9], lens[11] = -1, 2 ** 31 - 5                # lengths that no table holds
    want = _consensus(x, V, parents, tokens, max_path, kv, table, lens)
    m = want["accept_len"] + 1
    longest = min(max_path or N, max(map(len, paths)))
    assert want["status"] == -4 and want["num_committed"][[7, 9, 11]].tolist() == [0, 0, 0]
    assert m.max() == longest and (longest < 3 or len(set(m.tolist())) > 2), np.bincount(m)


@pytest.mark.parametrize("form,B,N,V,max_path", [("walk", 24, 64, 50001, 5), ("scan", 5, 20, 3001, 20)])
@pytest.mark.parametrize("P,layer_gap", [(16, 0), (32, 64), (128, 0)])
def test_committed_rows_are_read_where_the_projection_left_them(form, B, N, V, max_path, P, layer_gap):
    """The K/V parts of fused rows, layers without and with a gap between them, into pages of several sizes."""
    assert consensus_form(B, N, V, max_path)[0] == form
    rt, H, Hq, d, L = _rt(), 2, 3, 64, 3
    parents, tokens = _trees(P, B, N, 9, V)
    rng, x, _ = _logits(P + 1, B, N, V, parents, tokens, "f32", stop=0.1)
    lens = rng.integers(0, 300, B).astype(np.int32)
    kv, table = _kv(rng, L, B, N, lens, N, P, H, d)
    row = (Hq + 2 * H) * d
    fused = torch.full((L, B * N * row + layer_gap), 0x7fc0, dtype=torch.int16, device="cuda")
    parts = fused[:, :B * N * row].unflatten(1, (B, N, Hq + 2 * H, d))
    k, v = parts[..., Hq:Hq + H, :], parts[..., Hq + H:, :]
    k.copy_(rt.to_device_bits(kv["k"]))
    v.copy_(rt.to_device_bits(kv["v"]))
    want = _consensus(x, V, parents, tokens, max_path, kv, table, lens, (0, 0, row, d, B * N * row + layer_gap if layer_gap else 0), (k, v))
    assert want["status"] == 0 and want["num_committed"].max() > 3


@pytest.mark.parametrize("kind,B,N,max_path,form", [("f32", 2, 3, None, ("scan", 2048)), ("bf16", 8, 64, 6, ("walk", 8192)), ("f32", 3, 64, 5, ("walk", 2048)),
                                                    ("f16", 5, 8, None, ("scan", 4096))])
def test_the_largest_vocabulary(kind, B, N, max_path, form):
    V = 1 << 20
    assert consensus_form(B, N, V, max_path, kind) == form
    parents, tokens = _trees(B, B, N, 7, V)
    tokens[:, 1::2] |= V - 1024       # many among the last
    tokens[:, -1] = V - 1
    _, x, _ = _logits(B + 1, B, N, V, parents, tokens, kind, stop=0.05)
    want = _consensus(x, V, parents, tokens, max_path)
    assert want["out_tokens"].max() > V - 1025


@pytest.mark.parametrize("form,B,N,V,max_path", [("walk", 24, 64, 50001, 6), ("scan", 5, 20, 3001, 20)])
def test_a_recorded_consensus_takes_the_logits_and_trees_of_each_replay(form, B, N, V, max_path):
    """With eager work in between; the paths of one replay leave nothing to the next."""
    assert consensus_form(B, N, V, max_path)[0] == form
    from paper_2605_12825_amd import binding
    rt, H, d = _rt(), 2, 64
    step = rt.DecodeStep(batch=B, num_q_heads=H, num_kv_heads=H, head_dim=d, block_k=1, page_size=16, max_pages_per_seq=1, max_seq_len=0, num_pages=1, vocab=V)
    i32 = dict(dtype=torch.int32, device="cuda")
    r = {n: torch.zeros((B,), **i32) for n in ("accept_len", "num_committed", "next_anchor")}
    r.update({n: torch.zeros((B, N), **i32) for n in ("path_nodes", "out_tokens")})
    x, up, held = torch.zeros((B, N, V), device="cuda"), torch.zeros((B, N), **i32), torch.zeros((B, N), **i32)
    stream = torch.cuda.Stream()
    step.reserve(tree_nodes=N)
    torch.cuda.synchronize()
    binding.orthrus_graph_begin(step.ctx, stream)
    step.tree_consensus_commit(x, up, held, None, None, None, None, None, None, r["accept_len"], r["num_committed"], r["path_nodes"], r["out_tokens"],
                               r["next_anchor"], max_path=max_path, stream=stream)
    g = binding.orthrus_graph_end(step.ctx, stream)
    for i, stop in enumerate((0.02, 0.9, 0.3, 1.0, 0.05)):
        parents, tokens = _trees(i, B, N, 8, V)
        _, y, _ = _logits(i, B, N, V, parents, tokens, "f32", stop=stop)
        x.copy_(y)
        up.copy_(torch.from_numpy(parents))
        held.copy_(torch.from_numpy(tokens))
        torch.cuda.synchronize()
        binding.orthrus_graph_launch(g, stream)
        torch.cuda.synchronize()
        want = oracle.tree_consensus_commit(_Rows(x, V), parents, tokens, max_path)
        for k, v in r.items():
            np.testing.assert_array_equal(v.cpu().numpy(), want[k], err_msg="%s %d" % (k, i))
        (y * 2).sum()
    binding.orthrus_graph_destroy(g)
    step.close()


# ---------------------------------------------------------------------------------------------------------------
# calls that are refused, before anything is launched

def test_each_operand_on_another_device_is_refused():
    rt, B, N, H, d, V = _rt(), 2, 9, 2, 64, 500
    step = rt.DecodeStep(batch=B, num_q_heads=H, num_kv_heads=H, head_dim=d, block_k=1, page_size=16, max_pages_per_seq=4, max_seq_len=60, num_pages=8,
                         vocab=V, pool_strides=(8 * H * 16 * d, H * 16 * d, 16 * d, d))
    on = dict(device="cuda")
    rows = lambda *n: torch.zeros(n, dtype=torch.bfloat16, **on)  # noqa: E731
    ints = lambda *n: torch.zeros(n, dtype=torch.int32, **on)  # noqa: E731
    attn = dict(parents=ints(B, N), q=rows(B, N, H, d), k_blk=rows(B, N, H, d), v_blk=rows(B, N, H, d), k_pool=rows(8, H, 16, d), v_pool=rows(8, H, 16, d),
                page_table=ints(B, 4), seq_lens=ints(B), out=rows(B, N, H, d), lse=torch.zeros((B, H, N), **on))
    walk = dict(ar_logits=torch.zeros((B, N, V), **on), parents=ints(B, N), node_tokens=ints(B, N), k_blk_ar=rows(1, B, N, H, d), v_blk_ar=rows(1, B, N, H, d),
                k_pool=rows(1, 8, H, 16, d), v_pool=rows(1, 8, H, 16, d), page_table=ints(B, 4), seq_lens=ints(B), accept_len=ints(B), num_committed=ints(B),
                path_nodes=ints(B, N), out_tokens=ints(B, N), next_anchor=ints(B))
    for call, args in ((step.tree_attn, attn), (step.tree_consensus_commit, walk)):
        for _ in range(2):     # before and after a call of the same sizes
            for name in args:
                with pytest.raises(ValueError, match="%s must be on cuda:0, not on cpu" % name):
                    call(**dict(args, **{name: args[name].cpu()}))
            call(**args)
    rules = rt.LogitRules(repetition=torch.ones(B, **on))
    x, fed = torch.zeros((B, N, V), **on), ints(B, N)
    for kw in (dict(logits=x.cpu(), rules=rt.LogitRules(repetition=torch.ones(B))), dict(logits=x, rules=rt.LogitRules(repetition=torch.ones(B))),
               dict(logits=x, rules=rules, tokens=fed.cpu()), dict(logits=x, rules=rules, tokens=fed, parents=fed.cpu()), dict(logits=x, rules=rules, out=x.cpu())):
        with pytest.raises(ValueError):
            step.process_logits(**kw)
    step.process_logits(x, rules, fed, fed)
    torch.cuda.synchronize()
    assert step.device_error() == 0
    step.close()


def test_a_first_call_within_a_recording_is_refused():
    """On the stream that is recorded, whatever torch's current one is; after reserve() the same call is recorded."""
    from paper_2605_12825_amd import binding
    rt, B, N, H, d, V = _rt(), 2, 9, 2, 64, 500
    step = rt.DecodeStep(batch=B, num_q_heads=H, num_kv_heads=H, head_dim=d, block_k=1, page_size=16, max_pages_per_seq=4, max_seq_len=60, num_pages=8,
                         vocab=V, num_splits=2)
    rng = np.random.default_rng(1)
    up = rt.to_device_bits
    q, k, v = up(_bits(rng, B, N, H, d)), up(_bits(rng, B, N, H, d)), up(_bits(rng, B, N, H, d))
    kp, vp = up(_bits(rng, 8, H, 16, d)), up(_bits(rng, 8, H, 16, d))
    parents = up(np.array([_tree(rng, N)] * B, np.int32))
    table, lens = torch.arange(8, dtype=torch.int32, device="cuda").view(B, 4), torch.tensor([60, 17], dtype=torch.int32, device="cuda")
    out, x, rules = torch.zeros_like(q), torch.ones((B, N, V), device="cuda"), rt.LogitRules(repetition=torch.full((B,), 2.0, device="cuda"))
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for first in (True, False):
        binding.orthrus_graph_begin(step.ctx, stream)
        try:
            step.process_logits(x, rules, parents.clamp(min=0) if first else None, stream=stream)    # (needs no workspace)
            if first:
                for handle in (stream, stream.cuda_stream):
                    with pytest.raises(RuntimeError, match="reserve"):
                        step.tree_attn(parents, q, k, v, kp, vp, table, lens, out, stream=handle)
            else:
                step.tree_attn(parents, q, k, v, kp, vp, table, lens, out, stream=stream)
        finally:
            g = binding.orthrus_graph_end(step.ctx, stream)
        if first:
            binding.orthrus_graph_destroy(g)
            step.reserve(tree_nodes=N)
    step.tree_attn(parents, q, k, v, kp, vp, table, lens, out)
    torch.cuda.synchronize()
    want = out.clone()
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        binding.orthrus_graph_launch(g, stream)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    binding.orthrus_graph_destroy(g)
    step.close()


# ---------------------------------------------------------------------------------------------------------------
# attention: ((64-row kernel, waves, order, non-temporal, row groups), (Hq, H, d, nodes, batch, longest, splits, layers))

_FORMS = [
    ((False, 1, 'balanced', 0, 1), (1, 1, 64, 1, 20, 131, -1, 1)), ((False, 1, 'balanced', 1, 1), (2, 2, 64, 1, 6, 400, -1, 300)),
    ((False, 1, 'by size', 0, 1), (2, 2, 64, 2, 520, 131, 2, 1)), ((False, 1, 'by size', 1, 1), (1, 1, 64, 1, 520, 260, 3, 300)),
    ((False, 1, 'plain', 0, 1), (1, 1, 64, 2, 9, 131, 1, 1)), ((False, 1, 'plain', 1, 1), (4, 4, 64, 1, 9, 200, 0, 300)),
    ((False, 2, 'balanced', 0, 1), (1, 1, 64, 33, 6, 131, -1, 1)), ((False, 2, 'balanced', 1, 1), (1, 1, 64, 33, 9, 520, -1, 300)),
    ((False, 2, 'by size', 0, 1), (1, 1, 64, 33, 384, 131, 3, 1)), ((False, 2, 'by size', 1, 1), (2, 2, 64, 33, 200, 131, 3, 300)),
    ((False, 2, 'plain', 0, 1), (1, 1, 64, 33, 6, 131, 0, 1)), ((False, 2, 'plain', 1, 1), (1, 1, 64, 33, 9, 520, 3, 300)),
    ((False, 3, 'balanced', 0, 1), (2, 1, 64, 33, 6, 131, -1, 1)), ((False, 3, 'balanced', 1, 1), (2, 1, 64, 33, 9, 520, -1, 300)),
    ((False, 3, 'by size', 0, 1), (4, 2, 64, 33, 200, 131, 2, 1)), ((False, 3, 'by size', 1, 1), (2, 1, 64, 33, 384, 131, 3, 300)),
    ((False, 3, 'plain', 0, 1), (2, 1, 64, 33, 6, 131, 3, 1)), ((False, 3, 'plain', 1, 1), (2, 1, 64, 33, 9, 520, 0, 300)),
    ((False, 4, 'balanced', 0, 1), (3, 1, 64, 33, 6, 131, -1, 1)), ((False, 4, 'balanced', 1, 1), (6, 2, 64, 33, 9, 260, -1, 300)),
    ((False, 4, 'balanced', 0, 2), (7, 1, 64, 33, 6, 131, -1, 1)), ((False, 4, 'by size', 0, 1), (3, 1, 64, 33, 200, 131, 3, 1)),
    ((False, 4, 'by size', 1, 1), (3, 1, 64, 33, 200, 131, 3, 300)), ((False, 4, 'plain', 0, 1), (2, 1, 64, 49, 6, 131, 3, 1)),
    ((False, 4, 'plain', 1, 1), (3, 1, 64, 33, 9, 520, 3, 300)), ((False, 5, 'balanced', 0, 1), (3, 1, 64, 48, 6, 131, -1, 1)),
    ((False, 5, 'balanced', 1, 1), (4, 1, 64, 33, 9, 520, -1, 300)), ((False, 5, 'balanced', 0, 2), (7, 1, 64, 38, 6, 131, -1, 1)),
    ((False, 5, 'balanced', 0, 3), (16, 2, 64, 58, 6, 131, -1, 1)), ((False, 5, 'by size', 0, 1), (4, 1, 64, 33, 200, 131, 3, 1)),
    ((False, 5, 'by size', 1, 1), (4, 1, 64, 33, 200, 131, 3, 300)), ((False, 5, 'by size', 0, 2), (16, 2, 64, 33, 64, 131, 3, 1)),
    ((False, 5, 'plain', 0, 1), (4, 1, 64, 33, 6, 131, 2, 1)), ((False, 5, 'plain', 1, 1), (6, 2, 64, 43, 9, 260, 0, 300)),
    ((False, 5, 'plain', 0, 2), (8, 1, 64, 33, 6, 131, 2, 1)), ((False, 6, 'balanced', 0, 1), (5, 1, 64, 33, 6, 131, -1, 1)),
    ((False, 6, 'balanced', 1, 1), (5, 1, 64, 33, 9, 520, -1, 300)), ((False, 6, 'balanced', 0, 2), (7, 1, 64, 48, 6, 131, -1, 1)),
    ((False, 6, 'balanced', 0, 3), (8, 1, 64, 64, 6, 131, -1, 1)), ((False, 6, 'by size', 0, 1), (10, 2, 64, 33, 64, 131, 3, 1)),
    ((False, 6, 'by size', 1, 1), (10, 2, 64, 33, 64, 131, 3, 300)), ((False, 6, 'by size', 0, 2), (7, 1, 64, 48, 64, 131, 3, 1)),
    ((False, 6, 'plain', 0, 1), (5, 1, 64, 33, 6, 131, 0, 1)), ((False, 6, 'plain', 1, 1), (5, 1, 64, 33, 9, 520, 0, 300)),
    ((False, 6, 'plain', 0, 2), (7, 1, 64, 48, 6, 131, 1, 1)), ((False, 7, 'balanced', 0, 1), (5, 1, 64, 41, 6, 131, -1, 1)),
    ((False, 7, 'balanced', 1, 1), (5, 1, 64, 41, 6, 1024, -1, 300)), ((False, 7, 'balanced', 0, 2), (8, 1, 64, 54, 6, 131, -1, 1)),
    ((False, 7, 'by size', 0, 1), (8, 2, 64, 50, 64, 200, 3, 1)), ((False, 7, 'by size', 1, 1), (5, 1, 64, 41, 128, 200, 3, 300)),
    ((False, 7, 'by size', 0, 2), (8, 1, 64, 51, 64, 131, 3, 1)), ((False, 7, 'plain', 0, 1), (4, 1, 64, 53, 6, 131, 3, 1)),
    ((False, 7, 'plain', 1, 1), (4, 1, 64, 49, 9, 520, 2, 300)), ((False, 7, 'plain', 0, 2), (7, 1, 64, 62, 6, 131, 0, 1)),
    ((False, 8, 'by size', 0, 1), (7, 1, 64, 33, 128, 131, 3, 1)), ((False, 8, 'by size', 1, 1), (7, 1, 64, 33, 128, 131, 3, 300)),
    ((False, 8, 'by size', 0, 2), (8, 1, 64, 63, 64, 131, 3, 1)), ((False, 8, 'plain', 0, 1), (5, 1, 64, 46, 6, 131, 0, 1)),
    ((False, 8, 'plain', 1, 1), (20, 4, 64, 45, 9, 131, 2, 300)), ((False, 8, 'plain', 0, 2), (8, 1, 64, 63, 6, 131, 0, 1)),
    ((True, 2, 'by size', 0, 1), (2, 1, 64, 58, 768, 260, 0, 1)), ((True, 2, 'by size', 1, 1), (6, 2, 64, 38, 384, 260, 0, 300)),
    ((True, 4, 'by size', 0, 1), (5, 1, 64, 48, 384, 520, 0, 1)), ((True, 4, 'by size', 1, 1), (5, 1, 64, 48, 384, 520, 0, 300)),
    ((True, 4, 'by size', 0, 2), (8, 1, 64, 62, 200, 520, 0, 1)), ((True, 4, 'plain', 0, 1), (5, 1, 64, 48, 256, 1024, 0, 1)),
    ((True, 4, 'plain', 1, 1), (10, 2, 64, 48, 128, 1024, 0, 300)), ((True, 4, 'plain', 0, 2), (16, 2, 64, 63, 64, 1024, 0, 1)),
    ((False, 1, 'balanced', 0, 1), (1, 1, 128, 1, 9, 260, -1, 1)), ((False, 1, 'balanced', 1, 1), (1, 1, 128, 1, 6, 1024, -1, 300)),
    ((False, 1, 'by size', 0, 1), (1, 1, 128, 1, 520, 200, 2, 1)), ((False, 1, 'by size', 1, 1), (1, 1, 128, 1, 512, 200, 3, 300)),
    ((False, 1, 'plain', 0, 1), (1, 1, 128, 1, 9, 131, 1, 1)), ((False, 1, 'plain', 1, 1), (1, 1, 128, 1, 6, 400, 0, 300)),
    ((False, 2, 'balanced', 0, 1), (1, 1, 128, 33, 6, 131, -1, 1)), ((False, 2, 'balanced', 1, 1), (1, 1, 128, 33, 9, 260, -1, 300)),
    ((False, 2, 'by size', 0, 1), (1, 1, 128, 33, 300, 131, 3, 1)), ((False, 2, 'by size', 1, 1), (1, 1, 128, 33, 300, 131, 3, 300)),
    ((False, 2, 'plain', 0, 1), (1, 1, 128, 33, 6, 131, 0, 1)), ((False, 2, 'plain', 1, 1), (1, 1, 128, 33, 9, 260, 3, 300)),
    ((False, 3, 'balanced', 0, 1), (2, 1, 128, 33, 6, 131, -1, 1)), ((False, 3, 'balanced', 1, 1), (2, 1, 128, 33, 9, 260, -1, 300)),
    ((False, 3, 'by size', 0, 1), (2, 1, 128, 33, 300, 131, 3, 1)), ((False, 3, 'by size', 1, 1), (2, 1, 128, 34, 300, 131, 3, 300)),
    ((False, 3, 'plain', 0, 1), (2, 1, 128, 33, 6, 131, 0, 1)), ((False, 3, 'plain', 1, 1), (2, 1, 128, 33, 9, 260, 0, 300)),
    ((False, 4, 'balanced', 0, 1), (3, 1, 128, 33, 6, 131, -1, 1)), ((False, 4, 'balanced', 1, 1), (3, 1, 128, 33, 9, 260, -1, 300)),
    ((False, 4, 'balanced', 0, 2), (7, 1, 128, 33, 6, 131, -1, 1)), ((False, 4, 'by size', 0, 1), (2, 1, 128, 62, 200, 131, 3, 1)),
    ((False, 4, 'by size', 1, 1), (4, 2, 128, 49, 128, 131, 3, 300)), ((False, 4, 'plain', 0, 1), (2, 1, 128, 49, 6, 131, 0, 1)),
    ((False, 4, 'plain', 1, 1), (3, 1, 128, 33, 9, 260, 0, 300)), ((False, 5, 'balanced', 0, 1), (4, 1, 128, 33, 6, 131, -1, 1)),
    ((False, 5, 'balanced', 1, 1), (4, 1, 128, 33, 9, 260, -1, 300)), ((False, 5, 'balanced', 0, 2), (8, 1, 128, 33, 6, 131, -1, 1)),
    ((False, 5, 'balanced', 0, 3), (8, 1, 128, 59, 6, 131, -1, 1)), ((False, 5, 'by size', 0, 1), (4, 1, 128, 33, 200, 131, 3, 1)),
    ((False, 5, 'by size', 1, 1), (4, 1, 128, 33, 200, 131, 3, 300)), ((False, 5, 'by size', 0, 2), (8, 1, 128, 33, 128, 131, 3, 1)),
    ((False, 5, 'plain', 0, 1), (4, 1, 128, 33, 6, 131, 0, 1)), ((False, 5, 'plain', 1, 1), (4, 1, 128, 33, 9, 260, 2, 300)),
    ((False, 5, 'plain', 0, 2), (8, 1, 128, 33, 6, 131, 0, 1)), ((False, 6, 'balanced', 0, 1), (5, 1, 128, 33, 6, 131, -1, 1)),
    ((False, 6, 'balanced', 1, 1), (5, 1, 128, 33, 9, 260, -1, 300)), ((False, 6, 'balanced', 0, 2), (7, 1, 128, 48, 6, 131, -1, 1)),
    ((False, 6, 'balanced', 0, 3), (8, 1, 128, 64, 6, 131, -1, 1)), ((False, 6, 'by size', 0, 1), (4, 1, 128, 44, 128, 131, 3, 1)),
    ((False, 6, 'by size', 1, 1), (5, 1, 128, 33, 128, 131, 3, 300)), ((False, 6, 'by size', 0, 2), (7, 1, 128, 48, 64, 131, 3, 1)),
    ((False, 6, 'plain', 0, 1), (3, 1, 128, 54, 6, 131, 3, 1)), ((False, 6, 'plain', 1, 1), (5, 1, 128, 33, 9, 260, 0, 300)),
    ((False, 6, 'plain', 0, 2), (7, 1, 128, 48, 6, 131, 3, 1)), ((False, 7, 'balanced', 0, 1), (8, 2, 128, 50, 6, 131, -1, 1)),
    ((False, 7, 'balanced', 1, 1), (4, 1, 128, 54, 6, 400, -1, 300)), ((False, 7, 'balanced', 0, 2), (7, 1, 128, 57, 6, 131, -1, 1)),
    ((False, 7, 'by size', 0, 1), (4, 1, 128, 49, 128, 131, 3, 1)), ((False, 7, 'by size', 1, 1), (4, 1, 128, 50, 128, 200, 3, 300)),
    ((False, 7, 'by size', 0, 2), (7, 1, 128, 64, 64, 131, 3, 1)), ((False, 7, 'plain', 0, 1), (5, 1, 128, 39, 6, 131, 3, 1)),
    ((False, 7, 'plain', 1, 1), (5, 1, 128, 39, 9, 260, 1, 300)), ((False, 7, 'plain', 0, 2), (8, 1, 128, 54, 6, 131, 1, 1)),
    ((False, 8, 'by size', 0, 1), (5, 1, 128, 45, 128, 131, 3, 1)), ((False, 8, 'by size', 1, 1), (4, 1, 128, 57, 128, 131, 3, 300)),
    ((False, 8, 'by size', 0, 2), (8, 1, 128, 63, 64, 131, 3, 1)), ((False, 8, 'plain', 0, 1), (5, 1, 128, 45, 6, 131, 1, 1)),
    ((False, 8, 'plain', 1, 1), (7, 1, 128, 33, 9, 260, 0, 300)), ((False, 8, 'plain', 0, 2), (8, 1, 128, 63, 6, 131, 1, 1)),
    ((True, 2, 'by size', 0, 1), (2, 1, 128, 61, 896, 131, 0, 1)), ((True, 2, 'by size', 1, 1), (3, 1, 128, 41, 900, 131, 0, 300)),
    ((True, 2, 'plain', 0, 1), (12, 4, 128, 40, 128, 131, 1, 1)), ((True, 2, 'plain', 1, 1), (4, 2, 128, 60, 256, 131, 0, 300)),
    ((True, 4, 'by size', 0, 1), (5, 1, 128, 48, 300, 2048, 0, 1)), ((True, 4, 'by size', 1, 1), (5, 1, 128, 48, 300, 2048, 0, 300)),
    ((True, 4, 'by size', 0, 2), (8, 1, 128, 60, 200, 2048, 0, 1)),
]
_PAGES = 400


@pytest.mark.parametrize("form,args", _FORMS, ids=["%s-%d-%s-%d-%d-d%d" % (("wide" if f[0] else "32",) + f[1:] + (a[2],)) for f, a in _FORMS])
def test_attention_by_every_form(form, args):
    """A few of the sequences, with lengths from none on, against the oracle, all of them against another partition; unused nodes' memory
    holds NaN."""
    Hq, H, d, N, B, longest, splits, layers = args
    assert attn_form(*args, _PAGES * 16)[:5] == form
    rt, rng = _rt(), np.random.default_rng(B + N + Hq)
    lens = rng.integers(0, longest + 1, B).astype(np.int32)
    some = sorted({0, 1, 2, B // 2, B - 1})
    lens[some] = [0, 1, min(33, longest), longest, min(64, longest)]
    x = dict(q=_bits(rng, B, N, Hq, d), k=_bits(rng, B, N, H, d), v=_bits(rng, B, N, H, d), kp=_bits(rng, _PAGES, H, 16, d), vp=_bits(rng, _PAGES, H, 16, d),
             table=rng.integers(0, _PAGES, (B, (longest + 15) // 16)).astype(np.int32), lens=lens)
    parents = np.array([_tree(rng, N, 9, 0.1) for _ in range(B)], np.int64).astype(np.int32)
    bad = dict(x, k=x["k"].copy(), v=x["v"].copy())
    for b in range(0, B, 3):
        for i in range(1, N):
            if i not in oracle.tree_path(parents[b], i):
                bad["k"][b, i] = bad["v"][b, i] = 0x7fc0

    def call(x, splits, layers):
        step = rt.DecodeStep(batch=B, num_q_heads=Hq, num_kv_heads=H, head_dim=d, block_k=1, page_size=16, max_pages_per_seq=x["table"].shape[1],
                             max_seq_len=longest, num_pages=_PAGES, num_splits=splits, num_layers=layers)
        dv = {k: rt.to_device_bits(v) for k, v in x.items()}
        out = torch.full((B, N, Hq, d), 0x7fc0, dtype=torch.int16, device="cuda")
        lse = torch.full((B, Hq, N), float("nan"), device="cuda")
        args = (rt.to_device_bits(parents), dv["q"], dv["k"], dv["v"], dv["kp"], dv["vp"], dv["table"], dv["lens"])
        step.tree_attn(*args, out, lse)
        torch.cuda.synchronize()
        assert step.device_error() == 0
        again = torch.zeros_like(out)
        step.tree_attn(*args, again)
        torch.cuda.synchronize()
        assert torch.equal(out, again)
        step.close()
        return _f(rt.bits_to_numpy(out)).astype(np.float64), lse.cpu().numpy()

    got, lse = call(bad, splits, layers)
    part = {k: v if k in ("kp", "vp") else v[some] for k, v in x.items()}
    _check_attn(part, parents[some], got[some], lse[some])
    other, lse2 = call(x, 1 if splits == 2 else 2, 1)
    # two roundings of each, of weights and outputs of order one
    assert np.abs(got - other).max() <= 4 * U * max(1.0, np.abs(other).max()) and np.abs(lse - lse2).max() <= 2 * LSE_TOL
