"""GPU tests of orthrus_logits_process against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu

_TYPES = {"f32": (torch.float32, 0.0, 0.0), "bf16": (torch.bfloat16, 2.0 ** -8, 0.0), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -25)}


def _rt():
    from paper_2605_12825_amd import runtime
    return runtime


def _dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _rules(rng, B, R, V, hist=60, bias=True, masks=True, penalties=True):
    r = {}
    if penalties:
        r["history"] = rng.integers(0, V, (B, hist)).astype(np.int32)
        if B:
            r["history"][:, ::5] = r["history"][:, :1]                        # the same token many times
            r["history"][:, 3::11] = rng.choice([-1, V, 1 << 30, -(1 << 31)])   # no token
        r["history_lens"] = rng.integers(0, hist + 1, B).astype(np.int32)
        r["prompt_lens"] = (r["history_lens"] * rng.random(B)).astype(np.int32)
        r["repetition"] = rng.choice([1.0, 1.1, 0.7, 2.0], B).astype(np.float32)
        r["presence"] = rng.choice([0.0, 0.5, -0.25], B).astype(np.float32)
        r["frequency"] = rng.choice([0.0, 0.3, -0.1], B).astype(np.float32)
    if bias:
        n = rng.integers(0, 30, B)
        r["bias_starts"] = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        r["bias_tokens"] = rng.integers(-1, V + 1, int(n.sum())).astype(np.int32)
        if n.sum() > 1:
            r["bias_tokens"][1::3] = r["bias_tokens"][0::3][:r["bias_tokens"][1::3].size]   # a token twice: the last one counts
        r["bias_values"] = (rng.standard_normal(int(n.sum())) * 3).astype(np.float32)
    if masks:
        r["masks"] = rng.integers(-2 ** 31, 2 ** 31, (4, (V + 31) // 32 + 1)).astype(np.int32)
        r["masks"][1] = 0            # allows nothing
        r["masks"][2] = -1           # everything
        r["mask_rows"] = rng.choice([-1, 0, 1, 2, 3, 4, -(1 << 31)], (B, R)).astype(np.int32)
    return r


def _run(x, rules, tokens, parents, kind, pad=0, offset=0, in_place=False, stream=None):
    rt = _rt()
    B, R, V = x.shape
    step = rt.DecodeStep(batch=B, num_q_heads=1, num_kv_heads=1, head_dim=64, block_k=1, page_size=16, max_pages_per_seq=1, max_seq_len=0,
                         num_pages=1, vocab=V)
    flat = torch.full((B * R * (V + pad) + offset,), 7.0, dtype=_TYPES[kind][0], device="cuda")
    logits = flat[offset:].view(B, R, V + pad)
    logits[..., :V] = x.cuda()
    out = logits if in_place else torch.full((B, R, V + pad + 1), 3.0, dtype=_TYPES[kind][0], device="cuda")
    r = rt.LogitRules(**{k: _dev(v) for k, v in rules.items()})
    step.process_logits(logits, r, _dev(tokens), _dev(parents), out=None if in_place else out, logits_stride_row=V + pad,
                        out_stride_row=V + pad + 1)
    torch.cuda.synchronize()
    step.close()
    assert (flat[:offset] == 7).all() and (logits[..., V:] == 7).all()
    if not in_place:
        assert (out[..., V:] == 3).all() and torch.equal(logits[..., :V].cpu().view(torch.uint8), x.view(torch.uint8))   # (bits: NaN too)
    return out[..., :V].cpu()


def _check(x, got, kind, rules, tokens, parents):
    want, size = oracle.process_logits(x.float().numpy(), tokens, parents, **rules)
    _, u, least = _TYPES[kind]
    g = got.double().numpy()
    plain = size == 0
    # untouched logits keep their bits, struck out ones are -inf
    kept = torch.where(torch.from_numpy(np.isneginf(want)), torch.full_like(x, -np.inf), x)
    same = (got.view(torch.int32 if kind == "f32" else torch.int16) == kept.view(torch.int32 if kind == "f32" else torch.int16)).numpy()
    assert same[plain].all()
    fin = np.isfinite(want) & ~plain
    over = np.abs(want) > float(torch.finfo(_TYPES[kind][0]).max)
    tol = 1.01 * 2.0 ** -24 * size + 1.01 * u * np.abs(want) + least
    off = np.abs(g - want)
    assert (off[fin & ~over] <= tol[fin & ~over]).all(), (off - tol)[fin & ~over].max()
    odd = ~np.isfinite(want) & ~plain
    np.testing.assert_array_equal(g[odd], want[odd])
    return want


@pytest.mark.parametrize("B,R,V", [(1, 1, 1), (1, 1, 31), (2, 3, 33), (3, 1, 512), (2, 64, 700), (1, 33, 8191), (5, 2, 8192), (1, 16, 8193),
                                   (3, 7, 20011), (1, 4, 40000)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tree", [0, 1])
def test_rules(B, R, V, kind, tree):
    rng = np.random.default_rng(B * 1000 + R * 10 + V + tree)
    x = torch.from_numpy(rng.standard_normal((B, R, V)).astype(np.float32) * 4).to(_TYPES[kind][0])
    rules = _rules(rng, B, R, V)
    tokens = rng.integers(-1, V + 1, (B, R)).astype(np.int32)
    tokens[:, R // 2:] = tokens[:, :1]                     # the same token again on a path
    parents = np.array([[-1] + [int(rng.integers(-1, i + 1)) for i in range(1, R)] for _ in range(B)], np.int32) if tree else None
    for in_place, pad, offset in ((False, 0, 0), (True, 3, 1), (False, 2, 5), (True, 0, 0)):
        got = _run(x, rules, tokens, parents, kind, pad, offset, in_place)
        _check(x, got, kind, rules, tokens, parents)


@pytest.mark.parametrize("only", ["penalties", "bias", "masks", "nothing"])
@pytest.mark.parametrize("in_place", [False, True])
def test_one_rule_alone(only, in_place):
    rng = np.random.default_rng(5)
    B, R, V = 4, 3, 9001
    x = torch.from_numpy(rng.standard_normal((B, R, V)).astype(np.float32))
    rules = _rules(rng, B, R, V, bias=only == "bias", masks=only == "masks", penalties=only == "penalties")
    for tokens in (None, rng.integers(0, V, (B, R)).astype(np.int32)):
        got = _run(x, rules, tokens, None, "f32", in_place=in_place)
        _check(x, got, "f32", rules, tokens, None)
        if only == "nothing":
            assert torch.equal(got, x)


def test_odd_penalties_and_logits():
    rng = np.random.default_rng(6)
    B, R, V = 8, 2, 3000
    x = torch.from_numpy(rng.standard_normal((B, R, V)).astype(np.float32))
    x[:, 0, ::3], x[:, 1, ::3] = float("nan"), float("-inf")
    x[:, :, 1::7] = float("inf")
    x[:, :, 2::5] = 0.0
    rules = _rules(rng, B, R, V, hist=700)
    rules["repetition"] = np.array([np.nan, np.inf, 0, -1, 1.5, 1.5, 1, 1e-3], np.float32)
    rules["presence"] = np.array([1, 0, np.nan, np.inf, 0, -np.inf, 0, 1e30], np.float32)
    rules["frequency"] = np.array([0, np.nan, 2, 0, np.inf, 1, 0, -1e30], np.float32)
    tokens = rng.integers(0, V, (B, R)).astype(np.int32)
    got = _run(x, rules, tokens, None, "f32")
    want = _check(x, got, "f32", rules, tokens, None)
    assert np.isnan(want).any()


def test_histories_of_all_lengths():
    """None, one token, all of it the same, longer than the row, negative, the prompt longer than the text."""
    rng = np.random.default_rng(7)
    V, hist = 20000, 5000
    lens = np.array([0, 1, hist, hist, hist + 9, -4, 511, 513], np.int32)
    B = len(lens)
    rules = _rules(rng, B, 1, V, hist=hist, bias=False, masks=False)
    rules["history_lens"], rules["prompt_lens"] = lens, np.array([0, 5, 0, hist, 100, 3, -1, 512], np.int32)
    rules["history"][2] = 77
    rules["repetition"][:], rules["presence"][:], rules["frequency"][:] = 1.3, 0.5, 0.01
    x = torch.from_numpy(rng.standard_normal((B, 1, V)).astype(np.float32))
    got = _run(x, rules, None, None, "f32")
    want = _check(x, got, "f32", rules, None, None)
    assert abs(got[2, 0, 77].item() - want[2, 0, 77]) < 1e-4 and want[2, 0, 77] < -45


def test_biases_outside_the_list():
    rng = np.random.default_rng(8)
    B, V = 5, 300
    x = torch.from_numpy(rng.standard_normal((B, 1, V)).astype(np.float32))
    rules = dict(bias_starts=np.array([-5, 3, 2, 9, 400, 2], np.int32), bias_tokens=rng.integers(0, V, 12).astype(np.int32),
                 bias_values=np.arange(12).astype(np.float32))
    _check(x, _run(x, rules, None, None, "f32"), "f32", rules, None, None)


def test_long_texts_and_many_biases():
    """Texts whose tokens may stand there more often than 15 bits count, and more biases than 16 bits number: two words a token."""
    rng = np.random.default_rng(10)
    B, V, hist = 3, 9000, 40000
    x = torch.from_numpy(rng.standard_normal((B, 2, V)).astype(np.float32))
    rules = _rules(rng, B, 2, V, hist=hist, bias=False)
    rules["history"][0] = 8999
    rules["history_lens"], rules["prompt_lens"] = np.array([hist, hist, 33000], np.int32), np.array([100, 39000, 0], np.int32)
    rules["frequency"][:], rules["repetition"][:], rules["presence"][:] = 0.001, 1.2, 0.1
    rules["mask_rows"][:] = -1
    tokens = rng.integers(0, V, (B, 2)).astype(np.int32)
    for biases in (False, True):
        if biases:
            rules["bias_starts"] = np.array([0, 66000, 66000, 70000], np.int32)
            rules["bias_tokens"] = rng.integers(0, V, 70000).astype(np.int32)
            rules["bias_values"] = rng.standard_normal(70000).astype(np.float32)
        for in_place in (False, True):
            want = _check(x, _run(x, rules, tokens, None, "f32", in_place=in_place), "f32", rules, tokens, None)
    short = {k: v for k, v in rules.items() if k not in ("history", "history_lens", "prompt_lens")}   # biases alone ask for them too
    _check(x, _run(x, short, tokens, None, "f32"), "f32", short, tokens, None)
    assert want[0, 0, 8999] < -35


@pytest.mark.parametrize("kind,in_place,pad", [("f32", False, 0), ("f32", True, 3), ("bf16", False, 1)])
def test_more_logits_than_the_last_level_cache_holds(kind, in_place, pad):
    """Several rows to a workgroup and accesses that go past the caches: the bits of the same sequences in small calls."""
    rt = _rt()
    rng = np.random.default_rng(11)
    B, R, V = 32, 32, 150001
    rules, tokens = _rules(rng, B, R, V, hist=500), rng.integers(0, V, (B, R)).astype(np.int32)
    parents = np.array([[-1] + [int(rng.integers(0, i)) for i in range(1, R)] for _ in range(B)], np.int32)
    make = lambda n: rt.DecodeStep(batch=n, num_q_heads=1, num_kv_heads=1, head_dim=64, block_k=1, page_size=16, max_pages_per_seq=1,  # noqa: E731
                                   max_seq_len=0, num_pages=1, vocab=V)
    x = torch.randn((B, R, V + pad), generator=torch.Generator("cuda").manual_seed(3), device="cuda").to(_TYPES[kind][0])
    part, big, small = {}, make(B), make(2)
    for b in (0, 6, 30):
        r = {k: v[b:b + 2] if k not in ("bias_starts", "bias_tokens", "bias_values", "masks") else v for k, v in rules.items()}
        r["bias_starts"] = rules["bias_starts"][b:b + 3]
        part[b] = torch.zeros((2, R, V + pad), dtype=x.dtype, device="cuda")
        small.process_logits(x[b:b + 2], rt.LogitRules(**{k: _dev(v) for k, v in r.items()}), _dev(tokens[b:b + 2]), _dev(parents[b:b + 2]),
                             out=part[b], logits_stride_row=V + pad, out_stride_row=V + pad)
    out = None if in_place else torch.zeros_like(x)
    big.process_logits(x, rt.LogitRules(**{k: _dev(v) for k, v in rules.items()}), _dev(tokens), _dev(parents), out=out, logits_stride_row=V + pad,
                       out_stride_row=V + pad)
    torch.cuda.synchronize()
    words = torch.int32 if kind == "f32" else torch.int16
    for b, want in part.items():
        assert torch.equal((x if in_place else out)[b:b + 2, :, :V].view(words), want[..., :V].view(words)), b
    big.close()
    small.close()


def test_many_rows_and_rules_on_two_streams_and_replayed():
    """Two calls at once, each in place on logits of its own, with tensors of rules shared; then the same from a graph, five times
    with eager work in between."""
    rt = _rt()
    rng = np.random.default_rng(9)
    B, R, V = 6, 32, 30000
    xs = [torch.from_numpy(rng.standard_normal((B, R, V)).astype(np.float32)) for _ in range(2)]
    rules, tokens = _rules(rng, B, R, V, hist=3000), rng.integers(0, V, (B, R)).astype(np.int32)
    step = rt.DecodeStep(batch=B, num_q_heads=1, num_kv_heads=1, head_dim=64, block_k=1, page_size=16, max_pages_per_seq=1, max_seq_len=0,
                         num_pages=1, vocab=V)
    r, t = rt.LogitRules(**{k: _dev(v) for k, v in rules.items()}), _dev(tokens)
    d, streams = [x.cuda() for x in xs], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for x, s in zip(d, streams):
        step.process_logits(x, r, t, stream=s)
    torch.cuda.synchronize()
    for x, y in zip(xs, d):
        _check(x, y.cpu(), "f32", rules, tokens, None)
    fresh, out = xs[0].cuda(), torch.zeros_like(d[0])
    from paper_2605_12825_amd import binding as B_
    torch.cuda.synchronize()
    B_.orthrus_graph_begin(step.ctx, streams[0])
    step.process_logits(fresh, r, t, out=out, stream=streams[0])
    g = B_.orthrus_graph_end(step.ctx, streams[0])
    for i in range(5):
        out.zero_()
        torch.cuda.synchronize()
        B_.orthrus_graph_launch(g, streams[0])
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int32), d[0].view(torch.int32)), i
        (fresh * 2).sum()
    B_.orthrus_graph_destroy(g)
    step.close()
