"""GPU tests of the tree operators' further forms: consensus level by level and by whole scans, both sizes of a workgroup's piece, against
the oracle; rows of which a mask leaves nothing."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_trees import _TYPES, _bits, _cache, _rt, _tree

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
_DEAD = [(12, 30, 9, 5000, None), (12, 30, 9, 5000, 4), (40, 64, 9, 40000, 5), (64, 40, 9, 70000, 6)]


@pytest.mark.parametrize("B,N,depth,V,max_path", _DEAD)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_a_row_of_which_nothing_is_left_ends_the_path(B, N, depth, V, max_path, kind):
    """At the root, on the way and at the last node, with children that hold token 0 (and -1) below it: none is followed or committed, and
    there is no next anchor.  One logit that is left, the lowest number of the type or a NaN among -inf, is a token as any."""
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
