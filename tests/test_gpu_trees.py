"""GPU tests of orthrus_tree_attn and orthrus_tree_consensus_commit against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
from orthrus_inputs import bf16_bits_to_f32

pytestmark = pytest.mark.gpu

# A weight is rounded to bf16 before the value product and the output to bf16 after it: half a step, 2^-8, of each.  Scores are
# 32-bit sums of d = 128 products: with N(0, 1) rows at most 128 * 2^-24 * 110 / sqrt(128) = 8e-5 off, so weights and their sum
# each by that factor: 2e-4 = 0.05 * 2^-8 together.
U = 2.0 ** -8
LSE_TOL = 8e-5 + 1.2e-4 + 2e-5   # scores, up to 2100 additions in a lane at 2^-24 each, the exponential and the logarithm


def _rt():
    from paper_2605_12825_amd import runtime
    return runtime


def _bits(rng, *shape):
    return (rng.standard_normal(shape).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def _f(bits):
    return bf16_bits_to_f32(bits)


def _tree(rng, N, depth=64, unused=0.0):
    up, level = [-1], [0]
    for i in range(1, N):
        k = int(rng.integers(max(0, i - 6), i))
        while level[k] + 1 >= depth and k > 0:
            k = up[k] if up[k] >= 0 else 0
        if level[k] + 1 >= depth or rng.random() < unused:
            up.append(int(rng.choice([-1, i, i + 3, 1 << 30, -(1 << 31)])))
            level.append(0)
        else:
            up.append(k)
            level.append(level[k] + 1)
    return up


def _cache(rng, B, H, d, lens, P, room=0, layers=None):
    width = (int(max(lens)) + room + P - 1) // P + 1
    held = [(int(n) + room + P - 1) // P for n in lens]
    pages = sum(held) + 2
    perm, at = rng.permutation(pages).astype(np.int32), 0
    table = np.full((B, width), -1, np.int32)
    for b, n in enumerate(held):
        table[b, :n] = perm[at:at + n]
        at += n
    shape = (pages, H, P, d) if layers is None else (layers, pages, H, P, d)
    return _bits(rng, *shape), _bits(rng, *shape), table


def _attn(x, parents, splits, P, bound=None, want_lse=True, strides=None, step=None):
    B, N, Hq, d = x["q"].shape
    H, rt = x["k"].shape[2], _rt()
    step = step or rt.DecodeStep(batch=B, num_q_heads=Hq, num_kv_heads=H, head_dim=d, block_k=1, page_size=P,
                                 max_pages_per_seq=x["table"].shape[1], max_seq_len=int(x["lens"].max()) if bound is None else bound,
                                 num_pages=x["kp"].shape[0], num_splits=splits, block_strides=strides)
    dv = {k: rt.to_device_bits(v) for k, v in x.items()}
    out = torch.full((B, N, Hq, d), 0x7fc0, dtype=torch.int16, device="cuda")
    lse = torch.full((B, Hq, N), float("nan"), device="cuda") if want_lse else None
    step.tree_attn(rt.to_device_bits(np.asarray(parents, np.int32)), dv["q"], dv["k"], dv["v"], dv["kp"], dv["vp"], dv["table"], dv["lens"],
                   out, lse)
    torch.cuda.synchronize()
    err = step.device_error()
    return _f(rt.bits_to_numpy(out)).astype(np.float64), None if lse is None else lse.cpu().numpy(), err, step


def _check_attn(x, parents, got, lse):
    d = x["q"].shape[3]
    want, size, want_lse = oracle.tree_attn(1 / np.sqrt(d), np.asarray(parents), *[_f(x[n]) for n in ("q", "k", "v", "kp", "vp")],
                                            x["table"], x["lens"])
    off = np.abs(got - want) - (1.06 * U * size + 1.01 * U * np.abs(want) + 1e-6)
    assert np.isfinite(got).all() and off.max() <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))
    if lse is not None:
        assert np.abs(lse - want_lse).max() <= LSE_TOL


def _inputs(seed, N, Hq, H, d, lens, P):
    rng = np.random.default_rng(seed)
    B = len(lens)
    kp, vp, table = _cache(rng, B, H, d, lens, P)
    return rng, dict(q=_bits(rng, B, N, Hq, d), k=_bits(rng, B, N, H, d), v=_bits(rng, B, N, H, d), kp=kp, vp=vp, table=table,
                     lens=np.array(lens, np.int32))


@pytest.mark.parametrize("splits", [0, 1, 3, -1])
@pytest.mark.parametrize("N,Hq,H,d", [(1, 2, 2, 64), (1, 8, 1, 128), (5, 4, 2, 64), (8, 8, 2, 128), (24, 8, 2, 128), (31, 3, 1, 128),
                                      (32, 2, 1, 64), (33, 2, 2, 128), (40, 5, 1, 128), (64, 1, 1, 128), (64, 3, 1, 64), (48, 4, 1, 128),
                                      (63, 4, 1, 128), (64, 8, 1, 128), (40, 10, 1, 64)])
def test_trees_over_a_cache(N, Hq, H, d, splits):
    """Every wave count, one and two tiles of nodes, one and two row groups; lengths around the tiles' and pages' ends."""
    lens = [0, 1, 31, 32, 33, 200] if N <= 40 else [0, 33, 97]
    rng, x = _inputs(N * 100 + Hq, N, Hq, H, d, lens, 16)
    parents = [_tree(rng, N, unused=0.1) for _ in lens]
    got, lse, err, step = _attn(x, parents, splits, 16)
    assert err == 0
    _check_attn(x, parents, got, lse)
    again = _attn(x, parents, splits, 16, want_lse=False, step=step)[0]
    np.testing.assert_array_equal(got, again)      # the same bits, with and without the second output
    step.close()


@pytest.mark.parametrize("shape", ["chain", "star", "comb"])
@pytest.mark.parametrize("N", [17, 64])
def test_extreme_trees(shape, N):
    up = {"chain": list(range(-1, N - 1)), "star": [-1] + [0] * (N - 1), "comb": [-1] + [max(0, (i - 1) // 2 * 2) for i in range(1, N)]}[shape]
    _, x = _inputs(7, N, 4, 2, 128, [5, 300], 32)
    got, lse, err, step = _attn(x, [up, up], 0, 32)
    assert err == 0
    _check_attn(x, [up, up], got, lse)
    step.close()


def test_long_and_ragged_batches():
    for splits in (0, -1):
        rng, x = _inputs(11, 16, 8, 2, 128, [4000, 3, 1777, 0, 250], 64)
        parents = [_tree(rng, 16, 5) for _ in range(5)]
        got, lse, err, step = _attn(x, parents, splits, 64, bound=4096)
        assert err == 0
        _check_attn(x, parents, got, lse)
        step.close()


def test_empty_caches():
    for N in (1, 33, 64):
        rng, x = _inputs(12, N, 4, 2, 64, [0, 0], 16)
        parents = [_tree(rng, N) for _ in range(2)]
        for splits in (0, 2, -1):
            got, lse, err, step = _attn(x, parents, splits, 16)
            assert err == 0
            _check_attn(x, parents, got, lse)
            step.close()


def test_many_short_sequences_start_by_size():
    rng, x = _inputs(13, 8, 2, 2, 64, list(np.random.default_rng(3).integers(0, 60, 500)), 16)
    parents = [_tree(rng, 8, 4, 0.2) for _ in range(500)]
    got, lse, err, step = _attn(x, parents, 1, 16)
    assert err == 0
    _check_attn(x, parents, got, lse)
    step.close()


@pytest.mark.parametrize("splits", [0, -1])
def test_what_unused_nodes_hold_is_not_read(splits):
    """NaN and infinities in the rows of unused nodes, whose own rows see the cache and the root, in pages behind the length and in
    pages of nobody."""
    N = 40
    rng, x = _inputs(17, N, 4, 1, 128, [0, 20, 70], 16)
    parents = [_tree(rng, N, 6, 0.4) for _ in range(3)]
    want = _attn(x, parents, splits, 16)[0]
    bad = {k: v.copy() for k, v in x.items()}
    for b in range(3):
        for i in range(N):
            if i and i not in oracle.tree_path(parents[b], i):
                bad["k"][b, i], bad["v"][b, i] = rng.choice([0x7fc0, 0x7f80, 0xff80]), rng.choice([0x7fc0, 0x7f80, 0xff80])
    mapped = {}
    for b, n in enumerate([0, 20, 70]):
        for s in range((n + 15) // 16):
            mapped[int(x["table"][b, s])] = min(16, n - 16 * s)
    for page in range(x["kp"].shape[0]):
        bad["kp"][page, :, mapped.get(page, 0):] = bad["vp"][page, :, mapped.get(page, 0):] = 0x7fc0
    got, lse, err, _ = _attn(bad, parents, splits, 16)
    assert err == 0
    np.testing.assert_array_equal(got, want)
    _check_attn(x, parents, got, lse)


def test_rows_read_where_the_projection_left_them():
    rt = _rt()
    B, N, Hq, H, d, P = 2, 33, 4, 2, 64, 16
    rng, x = _inputs(19, N, Hq, H, d, [40, 9], P)
    parents = np.array([_tree(rng, N) for _ in range(B)], np.int32)
    fused = np.concatenate([x["q"], x["k"], x["v"]], axis=2)     # [B, N, Hq + 2H, d]
    f = rt.to_device_bits(fused)
    row = (Hq + 2 * H) * d
    step = rt.DecodeStep(batch=B, num_q_heads=Hq, num_kv_heads=H, head_dim=d, block_k=1, page_size=P, max_pages_per_seq=x["table"].shape[1],
                         max_seq_len=40, num_pages=x["kp"].shape[0], block_strides=(row, d, row, d, 0))
    out = torch.zeros((B, N, Hq, d), dtype=torch.int16, device="cuda")
    dv = {k: rt.to_device_bits(v) for k, v in x.items()}
    step.tree_attn(rt.to_device_bits(parents), f[:, :, :Hq], f[:, :, Hq:Hq + H], f[:, :, Hq + H:], dv["kp"], dv["vp"], dv["table"],
                   dv["lens"], out)
    torch.cuda.synchronize()
    _check_attn(x, parents, _f(rt.bits_to_numpy(out)).astype(np.float64), None)
    step.close()


def test_bad_pages_and_lengths_are_reported_and_nothing_is_read_out_of_bounds():
    N = 9
    rng, x = _inputs(23, N, 4, 2, 64, [50, 40, 30], 16)
    parents = [_tree(rng, N) for _ in range(3)]
    x["table"][1, 0] = 1 << 29
    x["table"][2, 1] = -4
    for splits in (0, 2, -1):
        got, _, err, step = _attn(x, parents, splits, 16)
        assert err == -4 and np.isfinite(got).all()
        good = {k: v[:1] if k in ("q", "k", "v", "table", "lens") else v for k, v in x.items()}
        _check_attn(good, parents[:1], got[:1], None)
        step.close()
    rng, x = _inputs(29, N, 4, 2, 64, [50, 40], 16)
    lens = x["lens"].copy()
    x["lens"] = np.array([-3, 1 << 30], np.int32)
    got, _, err, step = _attn(x, parents[:2], 0, 16, bound=40)
    assert err == -4 and np.isfinite(got).all()
    x["lens"] = np.array([0, 40], np.int32)      # what such lengths count as
    _check_attn(x, parents[:2], got, None)
    step.close()
    assert lens.tolist() == [50, 40]


# ---------------------------------------------------------------------------------------------------------------
# consensus

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _walk_inputs(seed, B, N, V, depth, kind="f32", unused=0.1):
    """Logits whose largest value is planted: along a random path the next node's token, elsewhere any."""
    rng = np.random.default_rng(seed)
    parents = np.array([_tree(rng, N, depth, unused) for _ in range(B)], np.int64).astype(np.int32)
    tokens = rng.integers(0, V, (B, N)).astype(np.int32)
    tokens[rng.random((B, N)) < 0.05] = rng.choice([-1, V, -(1 << 31)])
    x = rng.standard_normal((B, N, V)).astype(np.float32)
    for b in range(B):
        node = 0
        for i in range(N):
            x[b, i, rng.integers(V)] = 9
        while True:
            below = [i for i in range(node + 1, N) if parents[b, i] == node and 0 <= tokens[b, i] < V]
            if not below or rng.random() < 0.15:
                break
            child = int(rng.choice(below))
            x[b, node, tokens[b, child]] = 12
            node = child
    return rng, parents, tokens, torch.from_numpy(x).to(_TYPES[kind]).float().numpy()


def _walk(x, parents, tokens, max_path, kind="f32", pad=0, offset=0, kv=None, table=None, lens=None, P=16, layers=1):
    rt = _rt()
    B, N, V = x.shape
    H, d = (kv["k"].shape[3], kv["k"].shape[4]) if kv else (1, 64)
    step = rt.DecodeStep(batch=B, num_q_heads=H, num_kv_heads=H, head_dim=d, block_k=1, page_size=P,
                         max_pages_per_seq=1 if table is None else table.shape[1], max_seq_len=0, vocab=V, num_layers=layers,
                         num_pages=1 if kv is None else kv["kp"].shape[1],
                         pool_strides=None if kv is None else (kv["kp"].shape[1] * H * P * d, H * P * d, P * d, d))
    flat = torch.full((B * N * (V + pad) + offset,), 50.0, dtype=_TYPES[kind], device="cuda")   # padding is never looked at
    logits = flat[offset:].view(B, N, V + pad)
    logits[..., :V] = torch.from_numpy(x).cuda().to(_TYPES[kind])
    i32 = dict(dtype=torch.int32, device="cuda")
    r = {n: torch.full((B,), -7, **i32) for n in ("accept_len", "num_committed", "next_anchor")}
    r.update({n: torch.full((B, N), -7, **i32) for n in ("path_nodes", "out_tokens")})
    dv = {k: rt.to_device_bits(v) for k, v in (kv or {}).items()}
    t, l = (None, None) if table is None else (rt.to_device_bits(table), rt.to_device_bits(lens))
    step.tree_consensus_commit(logits, rt.to_device_bits(parents), rt.to_device_bits(tokens), dv.get("k"), dv.get("v"), dv.get("kp"),
                               dv.get("vp"), t, l, r["accept_len"], r["num_committed"], r["path_nodes"], r["out_tokens"], r["next_anchor"],
                               max_path=max_path, logits_stride_row=V + pad)
    torch.cuda.synchronize()
    got = {k: v.cpu().numpy() for k, v in r.items()}
    got["status"] = step.device_error()
    if kv:
        got["kp"], got["vp"], got["lens"] = rt.bits_to_numpy(dv["kp"]), rt.bits_to_numpy(dv["vp"]), l.cpu().numpy()
    step.close()
    return got


def _check_walk(x, parents, tokens, max_path, got, kv=None, table=None, lens=None):
    N = x.shape[1]
    args = {}
    if kv:
        kp, vp, l = kv["kp"].copy(), kv["vp"].copy(), lens.copy()
        args = dict(k_blk_ar=kv["k"], v_blk_ar=kv["v"], k_pool=kp, v_pool=vp, page_table=table, seq_lens=l)
    want = oracle.tree_consensus_commit(x, parents, tokens, min(max_path or N, N), **args)
    for k, v in want.items():
        np.testing.assert_array_equal(got[k], v, err_msg=k)
    if kv:
        for k, v in (("kp", kp), ("vp", vp), ("lens", l)):
            np.testing.assert_array_equal(got[k], v, err_msg=k)
    return want


@pytest.mark.parametrize("B,N,V,depth", [(1, 1, 1, 1), (1, 2, 3, 2), (3, 64, 511, 64), (2, 33, 2047, 9), (1, 17, 2049, 17), (2, 5, 8193, 5),
                                         (4, 64, 40001, 3), (40, 24, 16411, 2), (70, 48, 4099, 6), (1, 8, 151936, 8), (9, 60, 70000, 2)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_paths(B, N, V, depth, kind):
    """Both ways to the path (every row scanned; level by level), few and many chunks; rows that are not 16-byte aligned."""
    rng, parents, tokens, x = _walk_inputs(B * N + V, B, N, V, depth, kind)
    for max_path, pad, offset in ((None, 0, 0), (depth, 5, 1), (max(1, depth - 1), 267, 3)):
        got = _walk(x, parents, tokens, max_path, kind, pad, offset)
        _check_walk(x, parents, tokens, max_path, got)


def test_special_logits_ties_and_twins():
    B, N, V = 6, 12, 5000
    rng, parents, tokens, x = _walk_inputs(5, B, N, V, 6, unused=0)
    x[0] = -np.inf                                     # nothing: token 0
    x[1, 0, [4000, 31, 999]] = np.nan                  # the first NaN
    x[2, 0, :] = 3.0                                   # ties: the lowest index
    x[3, 0, :] = -0.0
    x[3, 0, 17] = 0.0                                  # the same value
    x[4, 0, [70, 4999]] = np.inf
    tokens[2, 3], parents[2, 3] = 0, 0
    tokens[2, 5], parents[2, 5] = 0, 0                 # twins: the first of them
    tokens[1, 1], parents[1, 1] = 31, 0
    got = _walk(x, parents, tokens, None)
    want = _check_walk(x, parents, tokens, None, got)
    assert want["out_tokens"][0, 0] == 0 and want["out_tokens"][1, 0] == 31 and want["out_tokens"][3, 0] == 0 and want["out_tokens"][4, 0] == 70


@pytest.mark.parametrize("layers,B,N,depth,V", [(1, 3, 8, 4, 700), (5, 2, 64, 40, 900), (2, 50, 48, 3, 9000)])
def test_the_path_enters_every_layers_cache(layers, B, N, depth, V):
    H, d, P = 2, 64, 16
    rng, parents, tokens, x = _walk_inputs(31 + layers, B, N, V, depth)
    lens = rng.integers(0, 60, B).astype(np.int32)
    kp, vp, table = _cache(rng, B, H, d, lens, P, room=depth, layers=layers)
    kv = dict(kp=kp, vp=vp, k=_bits(rng, layers, B, N, H, d), v=_bits(rng, layers, B, N, H, d))
    table[1, (lens[1] + P - 1) // P:] = -1             # no page to go on in
    if B > 2:
        table[2, lens[2] // P] = kp.shape[1]           # a page that the pool does not have
    got = _walk(x, parents, tokens, depth, kv=kv, table=table, lens=lens, P=P, layers=layers)
    _check_walk(x, parents, tokens, depth, got, kv, table, lens)
    assert got["status"] in (0, -4)
    bad = lens.copy()
    bad[0], bad[1] = -1, 2 ** 31 - 5                   # lengths that no table holds
    got = _walk(x, parents, tokens, depth, kv=kv, table=table, lens=bad, P=P, layers=layers)
    want = _check_walk(x, parents, tokens, depth, got, kv, table, bad)
    assert want["status"] == -4 and want["num_committed"][0] == 0 and want["num_committed"][1] == 0


@pytest.mark.parametrize("Hq,H,d,N,B,lo,hi", [(2, 2, 128, 56, 300, 128, 140), (2, 1, 128, 64, 520, 128, 170), (4, 1, 128, 64, 257, 1920, 1930),
                                              (8, 1, 64, 32, 320, 520, 540), (4, 1, 64, 63, 257, 890, 920), (2, 1, 64, 64, 704, 250, 260),
                                              (8, 1, 64, 64, 160, 512, 560)])
def test_the_64_row_kernel(Hq, H, d, N, B, lo, hi):
    """Launches that take it (units over CUs, rows that fill its waves, lengths from its rule on), both sides of its limits; a few of the
    sequences, with lengths from none on, against the oracle, the other ones against the 32-row kernel at two splits."""
    rng = np.random.default_rng(B)
    lens = rng.integers(lo, hi + 1, B).astype(np.int32)
    some = [0, 1, 7, B // 2, B - 1]
    lens[some[:4]] = [0, 1, 33, 64]
    pages = 400
    x = dict(q=_bits(rng, B, N, Hq, d), k=_bits(rng, B, N, H, d), v=_bits(rng, B, N, H, d), kp=_bits(rng, pages, H, 16, d),
             vp=_bits(rng, pages, H, 16, d), table=rng.integers(0, pages, (B, (hi + 15) // 16)).astype(np.int32), lens=lens)
    parents = np.array([_tree(rng, N, 9, 0.1) for _ in range(B)], np.int64).astype(np.int32)
    bad = x["v"].copy()
    for b in range(0, B, 9):
        for i in range(1, N):
            if i not in oracle.tree_path(parents[b], i):
                bad[b, i] = 0x7fc0
    got, lse, err, step = _attn(dict(x, v=bad), parents, 0, 16, bound=hi)
    assert err == 0
    step.close()
    part = {k: v if k in ("kp", "vp") else v[some] for k, v in x.items()}
    _check_attn(part, parents[some], got[some], lse[some])
    other, lse2, _, step = _attn(x, parents, 2, 16, bound=hi)
    step.close()
    # two roundings of each, of weights and outputs of order one
    assert np.abs(got - other).max() <= 4 * U * max(1.0, np.abs(other).max()) and np.abs(lse - lse2).max() <= 2 * LSE_TOL


@pytest.mark.parametrize("over", [-64, 64])
def test_rows_of_the_block_gigabytes_apart(over):
    """Offsets of the last rows on both sides of 31 bits."""
    N, Hq, H, d, P = 64, 3, 1, 64, 16
    rng, x = _inputs(61, N, Hq, H, d, [37], P)
    parents = [_tree(rng, N)]
    rt, row = _rt(), (1 << 24) + over
    step = rt.DecodeStep(batch=1, num_q_heads=Hq, num_kv_heads=H, head_dim=d, block_k=1, page_size=P, max_pages_per_seq=x["table"].shape[1],
                         max_seq_len=37, num_pages=x["kp"].shape[0], block_strides=(0, 0, row, d, 0))
    dv = {k: rt.to_device_bits(v) for k, v in x.items()}
    far = torch.empty(N * row, dtype=torch.int16, device="cuda")
    k, v = (far[at:].as_strided((1, N, H, d), (N * row, row, d, 1)) for at in (0, 1024))
    k.copy_(dv["k"].view(torch.int16))
    v.copy_(dv["v"].view(torch.int16))
    out = torch.zeros((1, N, Hq, d), dtype=torch.int16, device="cuda")
    step.tree_attn(rt.to_device_bits(np.asarray(parents, np.int32)), dv["q"], k, v, dv["kp"], dv["vp"], dv["table"], dv["lens"], out)
    torch.cuda.synchronize()
    assert step.device_error() == 0
    _check_attn(x, parents, _f(rt.bits_to_numpy(out)).astype(np.float64), None)
    step.close()


def test_a_recorded_call_keeps_its_workspace_when_a_larger_one_is_made():
    rt = _rt()
    from paper_2605_12825_amd import binding as B_
    rng, x = _inputs(71, 8, 4, 2, 128, [300, 900], 16)
    parents = [_tree(rng, 8) for _ in range(2)]
    step = rt.DecodeStep(batch=2, num_q_heads=4, num_kv_heads=2, head_dim=128, block_k=1, page_size=16, max_pages_per_seq=x["table"].shape[1],
                         max_seq_len=900, num_pages=x["kp"].shape[0], num_splits=4)
    dv = {k: rt.to_device_bits(v) for k, v in x.items()}
    up = rt.to_device_bits(np.asarray(parents, np.int32))
    out = torch.zeros((2, 8, 4, 128), dtype=torch.int16, device="cuda")
    step.reserve(tree_nodes=8)
    stream = torch.cuda.Stream()
    args = (up, dv["q"], dv["k"], dv["v"], dv["kp"], dv["vp"], dv["table"], dv["lens"], out)
    step.tree_attn(*args)
    torch.cuda.synchronize()
    want = out.clone()
    torch.cuda.synchronize()
    B_.orthrus_graph_begin(step.ctx, stream)
    step.tree_attn(*args, stream=stream)
    g = B_.orthrus_graph_end(step.ctx, stream)
    first = step.tree_attn_ws
    place, size = first.data_ptr(), first.numel()
    del first
    for N in (40, 64):   # each larger than the one before
        _, y = _inputs(N, N, 4, 2, 128, [300, 900], 16)
        dy = {k: rt.to_device_bits(y[k]) for k in ("q", "k", "v")}
        step.tree_attn(rt.to_device_bits(np.asarray([_tree(rng, N)] * 2, np.int32)), dy["q"], dy["k"], dy["v"], dv["kp"], dv["vp"], dv["table"], dv["lens"],
                       torch.zeros((2, N, 4, 128), dtype=torch.int16, device="cuda"))
    torch.cuda.synchronize()
    others = [torch.full((size,), 77, dtype=torch.uint8, device="cuda") for _ in range(6)]
    assert not any(t.data_ptr() < place + size and place < t.data_ptr() + t.numel() for t in others)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        B_.orthrus_graph_launch(g, stream)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(bool((t == 77).all()) for t in others)
    B_.orthrus_graph_destroy(g)
    step.close()


@pytest.mark.parametrize("splits", [16, 17, 40, -1])
def test_more_pieces_than_are_merged_at_once(splits):
    _, x = _inputs(81, 20, 2, 1, 128, [3000, 0, 100, 1, 1500], 16)
    parents = [list(range(-1, 19))] * 5
    for b in range(5) if splits < 0 else [None]:
        y = x if b is None else {k: v if k in ("kp", "vp") else v[b:b + 1] for k, v in x.items()}
        up = parents if b is None else parents[:1]
        got, lse, err, step = _attn(y, up, splits, 16, bound=3000)
        assert err == 0
        _check_attn(y, up, got, lse)
        step.close()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_many_rows_scanned_at_odd_places(kind):
    B, N, V = 9, 60, 69997
    rng, parents, tokens, x = _walk_inputs(91, B, N, V, 12, kind)
    for pad, offset in ((3, 0), (6, 5)):
        _check_walk(x, parents, tokens, None, _walk(x, parents, tokens, None, kind, pad, offset))
