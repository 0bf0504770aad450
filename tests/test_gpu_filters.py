"""GPU tests of orthrus_sample_tokens and orthrus_filtered_consensus_commit against the fp64 oracle.

Tokens and lengths must be identical.  Kernel and oracle both sum weights in 64 bits or more; what parts them is the polynomial
of the weights (4e-14), the fixed point (2^-40 of the largest weight, summed over the vocabulary) and the rounding of sums of
64-bit numbers: below 1e-10 of the sum for every row here, while a uniform number or a cut lies on average 1e-6 and more away from where
it would change a token.  (Where sums are equal by construction, in rows of equal logits, both are exact.)
A log-probability is rounded to fp32 once: half a step, 2^-24 of it, and 1e-9 of the probability.
"""
import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
#        temperature, top_k, top_p, min_p
FILTERS = [(1.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.0, 50, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (0.8, 40, 0.95, 0.05),
           (1.3, 0, 1.0, 0.02), (1.0, 3000, 0.8, 0.0), (2.0, 0, 0.97, 0.001), (0.05, 7, 0.5, 0.0), (1.0, 1, 1.0, 0.0),
           (0.9, 0, 0.999999, 0.0)]


def _rt():
    from paper_2605_12825_amd import runtime
    return runtime


def _step(B, K, V, **kw):
    full = dict(batch=B, num_q_heads=2, num_kv_heads=2, head_dim=64, block_k=K, page_size=16, max_pages_per_seq=4,
                max_seq_len=64, num_pages=8, vocab=V)
    full.update(kw)
    return _rt().DecodeStep(**full)


def _logits(seed, B, K, V, kind="peaked"):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((B, K, V)).astype(np.float32) * 2
    if kind == "peaked":
        n = min(V, 60)
        for r in x.reshape(-1, V):
            at = rng.permutation(V)[:n]
            r[at] = rng.uniform(13, 24) - rng.uniform(0.5, 2.0) * np.log(1 + np.arange(n)) + 0.2 * rng.standard_normal(n)
    return x


def _filters(rows, drop=()):
    cols = [np.array([f[i] for f in rows], dtype=t) for i, t in enumerate((np.float32, np.int32, np.float32, np.float32))]
    return [None if i in drop else c for i, c in enumerate(cols)]


def _dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _sample(x, filters, u, stride=0, want_lp=True, off=0):
    """x: torch tensor of logits [B,K,V] (host); returns tokens, log-probabilities and the step's device error."""
    B, K, V = x.shape
    step = _step(B, K, V)
    if stride or off:
        buf = torch.full((B * K * (stride or V) + off + 8,), 55.0, dtype=x.dtype)
        view = buf[off:off + B * K * (stride or V)].view(B * K, stride or V)
        view[:, :V] = x.view(B * K, V)
        dev = buf.cuda()[off:]
    else:
        dev = x.cuda()
    tokens = torch.full((B, K), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((B, K), 7.0, device="cuda") if want_lp else None
    step.sample_tokens(dev, *[_dev(f) for f in filters], _dev(u), tokens, lp, logits_stride_row=stride)
    torch.cuda.synchronize()
    assert step.device_error() == 0
    step.close()
    return tokens.cpu().numpy(), None if lp is None else lp.cpu().numpy()


def _check(x, filters, u, **kw):
    tokens, lp = _sample(x, filters, u, **kw)
    want, want_lp, _ = oracle.sample_tokens(x.float().numpy(), *filters, u)
    np.testing.assert_array_equal(tokens, want)
    if lp is not None:
        live = want >= 0
        assert (lp[~live] == -np.inf).all()
        assert np.all(np.abs(lp[live] - want_lp[live]) <= np.abs(want_lp[live]) * 2.0 ** -24 + 1e-9)
    return tokens


@pytest.mark.parametrize("vocab", [1, 2, 5, 63, 64, 511, 2049, 8191, 8193, 40001, 128256, 151936])
@pytest.mark.parametrize("kind", ["peaked", "flat"])
def test_every_filter_at_every_size(vocab, kind):
    B = len(FILTERS)
    x = torch.from_numpy(_logits(vocab, B, 2, vocab, kind))
    u = np.random.default_rng(vocab + 1).random((B, 2)).astype(np.float32)
    _check(x, _filters(FILTERS), u)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("vocab", [7, 1000, 32003, 151669])
@pytest.mark.parametrize("kind", ["peaked", "flat"])
def test_half_types_with_their_many_ties(dtype, vocab, kind):
    B = len(FILTERS)
    x = torch.from_numpy(_logits(vocab + 3, B, 2, vocab, kind)).to(TYPES[dtype])
    u = np.random.default_rng(vocab + 2).random((B, 2)).astype(np.float32)
    _check(x, _filters(FILTERS), u)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("stride,off", [(0, 1), (0, 3), (1003, 0), (1001, 5), (1024, 2)])
def test_strided_and_unaligned_rows(dtype, stride, off):
    B = len(FILTERS)
    x = torch.from_numpy(_logits(stride + off, B, 3, 1001)).to(TYPES[dtype])
    u = np.random.default_rng(stride).random((B, 3)).astype(np.float32)
    _check(x, _filters(FILTERS), u, stride=stride, off=off)


@pytest.mark.parametrize("batch,K", [(1, 1), (1, 32), (7, 13), (300, 1), (40, 16)])
def test_batches(batch, K):
    x = torch.from_numpy(_logits(batch, batch, K, 3001))
    u = np.random.default_rng(K).random((batch, K)).astype(np.float32)
    _check(x, _filters([FILTERS[b % len(FILTERS)] for b in range(batch)]), u)


@pytest.mark.parametrize("drop", [(1,), (2,), (3,), (1, 2, 3)])
def test_filters_that_are_not_given(drop):
    B = len(FILTERS)
    x = torch.from_numpy(_logits(77, B, 1, 5003))
    u = np.random.default_rng(78).random((B, 1)).astype(np.float32)
    _check(x, _filters(FILTERS, drop), u, want_lp=False)


def test_filter_values_outside_their_ranges():
    nan, inf = float("nan"), float("inf")
    rows = [(nan, 0, 1, 0), (-3, 5, .5, .1), (inf, 0, 1, 0), (1e-30, 0, 1, 0), (1e30, 0, .5, 0), (1, -4, 1, 0), (1, 10 ** 9, 1, 0),
            (1, 0, nan, 0), (1, 0, 0, 0), (1, 0, -1, 0), (1, 0, 2, 0), (1, 0, 1, nan), (1, 0, 1, -1), (1, 0, 1, 1), (1, 0, 1, 9),
            (1, 700, .3, 1e-8), (1e-45, 0, .9, 0)]
    x = torch.from_numpy(_logits(5, len(rows), 2, 701))
    u = np.random.default_rng(6).random((len(rows), 2)).astype(np.float32)
    _check(x, _filters(rows), u)


def test_uniform_numbers_at_and_outside_their_ends():
    us = [0.0, -0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, np.nan, np.inf, -np.inf, 2.0 ** -149]
    B = len(FILTERS)
    x = torch.from_numpy(np.repeat(_logits(8, B, 1, 9001), len(us), axis=1))
    _check(x, _filters(FILTERS), np.tile(np.array(us, np.float32), (B, 1)))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("gap,T", [(18.5, 0.3), (22.0, 0.5), (45.0, 1.0)])
@pytest.mark.parametrize("off", [0, 1, 3])
def test_unfiltered_draws_next_to_chunks_that_weigh_next_to_nothing(dtype, gap, T, off):
    """Every logit but the planted ones is 40 T to 41 T below the largest (0.2 T more or less for the types' rounding): e^-39.8 < 2^-57,
    so none has an amount in a fixed point of 50 bits, though 2048 of them together have, e^-41.2 * 2048 > 2^-49.  What is drawn is
    a planted token, wherever in the row it stands and however small the uniform number."""
    V, rng = 40001, np.random.default_rng(int(gap) + off)
    x = (gap - rng.uniform(40, 41, (5, 1, V)) * T).astype(np.float32)
    x[0, 0, 20007] = gap
    x[1, 0, :3 * 2048] = -np.inf                     # masked, then next to nothing, then the token
    x[1, 0, 39000] = gap
    x[2, 0, [100, 30000]] = gap                      # half of the sum at either, stretches of next to nothing between them
    x[3, 0, V - 1] = gap
    x[4, 0, :] = -np.inf
    x[4, 0, :2048] = gap - 40 * T                    # one stretch of next to nothing, the token at the end of the next
    x[4, 0, 4000] = gap
    us = np.array([0.0, -1.0, np.nan, 2.0 ** -149, 2.0 ** -50, 0.25, 0.5, 1.0], np.float32)
    f = [np.full(5, T, np.float32), None, None, None]
    t = torch.from_numpy(np.repeat(x, us.size, axis=1)).to(TYPES[dtype])
    tokens, lp = _sample(t, f, np.tile(us, (5, 1)), off=off)
    want = np.tile(np.array([20007, 39000, 100, V - 1, 4000], np.int32)[:, None], (1, us.size))
    want[2, us >= 0.5] = 30000
    np.testing.assert_array_equal(tokens, want)
    half = np.log(0.5)
    assert np.all(np.abs(lp[[0, 1, 3, 4]]) <= 1e-9) and np.all(np.abs(lp[2] - half) <= -half * 2.0 ** -24 + 1e-9)


@pytest.mark.parametrize("vocab", [1, 64, 1024, 9001, 65536])
@pytest.mark.parametrize("value", [0.0, -3.25, np.finfo(np.float32).min, np.inf])
def test_rows_of_equal_logits(vocab, value):
    """Sums that meet their targets exactly: the shortest prefix and the strict comparison decide."""
    rows = [(1.0, 0, 1.0, 0.0), (1.0, 0, 0.5, 0.0), (1.0, 17, 1.0, 0.0), (0.3, 0, 0.25, 1.0), (1.0, 16, 0.5, 0.0), (0.0, 0, 1.0, 0.0),
            (1.0, vocab // 2, 0.75, 0.0)]
    x = torch.full((len(rows), 5, vocab), value)
    u = np.tile(np.array([0.0, 0.25, 0.5, 0.75, 0.999], np.float32), (len(rows), 1))
    _check(x, _filters(rows), u)


def test_masked_infinite_and_nan_logits():
    B, V = len(FILTERS), 4099
    x = _logits(12, B, 9, V)
    rng = np.random.default_rng(13)
    low = np.finfo(np.float32).min
    for b in range(B):
        x[b, 0] = -np.inf                                     # nothing left
        x[b, 1] = -np.inf; x[b, 1, rng.integers(V)] = -3.0    # one left
        x[b, 2, rng.permutation(V)[:V - 20]] = -np.inf        # twenty left
        x[b, 3, rng.permutation(V)[:V - 20]] = low            # masked with the lowest value
        x[b, 4] = low; x[b, 4, :3] = -np.inf                  # nothing but the lowest value
        x[b, 5, rng.permutation(V)[:300]] = np.nan
        x[b, 6] = np.nan
        x[b, 7, rng.permutation(V)[:3]] = np.inf
        x[b, 8, rng.permutation(V)[:V // 2]] = 0.0
        x[b, 8, rng.permutation(V)[:V // 2]] = -0.0           # equal to the zeros
    u = rng.random((B, 9)).astype(np.float32)
    tokens = _check(torch.from_numpy(x), _filters(FILTERS), u)
    assert (tokens[:, 0] == -1).all() and (tokens[:, 6] == -1).all() and (tokens[:, [1, 2, 3, 4, 5, 7, 8]] >= 0).all()


def test_low_tokens_hold_the_nucleus():
    """Vocabularies list frequent tokens first: everything that is kept lies in one stretch of the row."""
    B, V = len(FILTERS), 151936
    x = _logits(21, B, 1, V, "flat")
    x[:, :, :3000] += 14
    u = np.random.default_rng(22).random((B, 1)).astype(np.float32)
    _check(torch.from_numpy(x), _filters(FILTERS), u)


def test_the_same_call_twice_and_rows_alone_or_together():
    B, K, V = len(FILTERS), 16, 30011
    x = torch.from_numpy(_logits(31, B, K, V))
    u = np.random.default_rng(32).random((B, K)).astype(np.float32)
    f = _filters(FILTERS)
    a, la = _sample(x, f, u)
    b, lb = _sample(x, f, u)
    np.testing.assert_array_equal(a, b)
    np.testing.assert_array_equal(la, lb)
    for i in (0, 4, 7):
        c, lc = _sample(x[i:i + 1, 3:4].contiguous(), [v[i:i + 1] for v in f], u[i:i + 1, 3:4])
        assert c[0, 0] == a[i, 3] and lc[0, 0] == la[i, 3]


@pytest.mark.parametrize("vocab,dtype,off", [(1 << 20, "f32", 3), (1 << 20, "bf16", 7), (300007, "f16", 1)])
@pytest.mark.parametrize("kind", ["peaked", "flat"])
def test_the_largest_vocabularies(vocab, dtype, off, kind):
    x = torch.from_numpy(_logits(41, len(FILTERS), 1, vocab, kind)).to(TYPES[dtype])
    u = np.random.default_rng(42).random((len(FILTERS), 1)).astype(np.float32)
    _check(x, _filters(FILTERS), u, off=off)


@pytest.mark.parametrize("batch,vocab", [(65535, 40), (20000, 1801)])
def test_as_many_sequences_as_a_call_takes(batch, vocab):
    """Sequence b repeats sequence b mod 52: the oracle answers for those."""
    few = 52
    rows = [FILTERS[b % len(FILTERS)] for b in range(few)]
    x = torch.from_numpy(_logits(43, few, 1, vocab))
    u = np.random.default_rng(44).random((few, 1)).astype(np.float32)
    f = _filters(rows)
    want, _, _ = oracle.sample_tokens(x.numpy(), *f, u)
    again = np.arange(batch) % few
    tokens, _ = _sample(x[torch.from_numpy(again)], [v[again] for v in f], u[again])
    np.testing.assert_array_equal(tokens, want[again])
    c = _case(45, few, 1, vocab, rows)
    want = oracle.filtered_consensus_commit(c["ar"].numpy(), c["df"].numpy(), *c["f"], c["draft"], c["u"], c["gumbel"])
    assert want["margin"] > 1e-8
    many = {k: c[k][again] for k in ("draft", "u", "gumbel")}
    many.update(ar=c["ar"][torch.from_numpy(again)], df=c["df"][torch.from_numpy(again)], f=[v[again] for v in c["f"]])
    got, err = _consensus(many)
    assert err == 0
    for k in ("accept_len", "num_committed", "out_tokens", "next_anchor"):
        np.testing.assert_array_equal(got[k], want[k][again], err_msg=k)


def test_rows_farther_apart_than_32_bits_count():
    B, K, V, stride = 2, 10, 40001, (1 << 27) + 8
    x = torch.from_numpy(_logits(46, B, K, V)).to(torch.bfloat16)
    u = np.random.default_rng(47).random((B, K)).astype(np.float32)
    f = _filters([FILTERS[1], FILTERS[0]])
    want, _ = _sample(x, f, u)
    buf = torch.empty((B * K - 1) * stride + V, dtype=torch.bfloat16, device="cuda")
    for r in range(B * K):
        buf[r * stride:r * stride + V] = x.view(B * K, V)[r].cuda()
    step = _step(B, K, V)
    tokens = torch.full((B, K), -7, dtype=torch.int32, device="cuda")
    step.sample_tokens(buf, *[_dev(v) for v in f], _dev(u), tokens, None, logits_stride_row=stride)
    torch.cuda.synchronize()
    step.close()
    np.testing.assert_array_equal(tokens.cpu().numpy(), want)


# ---- the consensus

def _case(seed, B, K, V, rows, kind="peaked", noise=0.4, dtype="f32"):
    rng = np.random.default_rng(seed)
    ar = _logits(seed, B, K, V, kind)
    df = ar + noise * rng.standard_normal(ar.shape).astype(np.float32)
    t = TYPES[dtype]
    ar, df = torch.from_numpy(ar).to(t), torch.from_numpy(df).to(t)
    f = _filters(rows)
    draft, _, _ = oracle.sample_tokens(df.float().numpy(), *f, rng.random((B, K)))
    return dict(ar=ar, df=df, f=f, draft=draft, u=rng.random((B, K)).astype(np.float32),
                gumbel=rng.gumbel(size=(B, V)).astype(np.float32))


def _consensus(c, commit=None, in_place=False, stride=0):
    B, K, V = c["ar"].shape
    kw = {}
    if commit is not None:
        L, pages, H, P, d = commit["k_pool"].shape
        kw = dict(num_q_heads=H, num_kv_heads=H, head_dim=d, max_pages_per_seq=commit["page_table"].shape[1],
                  max_seq_len=commit["page_table"].shape[1] * P, num_pages=pages, num_layers=L,
                  pool_strides=(pages * H * P * d, H * P * d, P * d, d))
    step = _step(B, K, V, **kw)
    place = lambda x: x.cuda()  # noqa: E731
    if stride:
        def place(x):
            buf = torch.full((B * K, stride), 60.0, dtype=x.dtype)
            buf[:, :V] = x.view(B * K, V)
            return buf.cuda()
    D = _rt().to_device_bits
    draft = _dev(c["draft"])
    acc, ncm, anchor = (torch.full((B,), -7, dtype=torch.int32, device="cuda") for _ in range(3))
    toks = draft if in_place else torch.full((B, K), -7, dtype=torch.int32, device="cuda")
    cm = {k: D(v) for k, v in commit.items()} if commit is not None else {}
    names = ("k_blk", "v_blk", "k_pool", "v_pool", "page_table", "seq_lens")
    step.filtered_consensus_commit(place(c["ar"]), place(c["df"]), *[_dev(v) for v in c["f"]], draft, _dev(c["u"]), _dev(c["gumbel"]),
                                   *[cm.get(n) for n in names], acc, ncm, toks, anchor, logits_stride_row=stride)
    torch.cuda.synchronize()
    err = step.device_error()
    step.close()
    got = dict(accept_len=acc, num_committed=ncm, out_tokens=toks, next_anchor=anchor)
    got = {k: v.cpu().numpy() for k, v in got.items()}
    for n in ("k_pool", "v_pool", "seq_lens"):
        if n in cm:
            got[n] = _rt().bits_to_numpy(cm[n])
    return got, err


def _check_consensus(c, **kw):
    want = oracle.filtered_consensus_commit(c["ar"].float().numpy(), c["df"].float().numpy(), *c["f"], c["draft"], c["u"], c["gumbel"])
    assert want["margin"] > 1e-8     # no decision nearer to its border than any of the sides can tell
    got, err = _consensus(c, **kw)
    assert err == 0
    for k in ("accept_len", "num_committed", "out_tokens", "next_anchor"):
        np.testing.assert_array_equal(got[k], want[k], err_msg=k)
    return got


@pytest.mark.parametrize("vocab", [1, 3, 64, 1000, 8193, 40001, 151936])
@pytest.mark.parametrize("kind", ["peaked", "flat"])
def test_consensus_at_every_size(vocab, kind):
    _check_consensus(_case(vocab, len(FILTERS), 3, vocab, FILTERS, kind))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("K", [1, 8, 32])
def test_consensus_of_half_types(dtype, K):
    _check_consensus(_case(K, len(FILTERS), K, 2003, FILTERS, dtype=dtype), stride=2008)


@pytest.mark.parametrize("vocab", [4526, 9001, 40001, 151936])
def test_consensus_where_top_k_is_all_that_stands_above_a_level(vocab):
    """Eight rows of logits in steps and, for every level with 65 to 1790 logits at and above it, a sequence whose top-k is that number:
    whatever level a row's lists go down to, one sequence keeps exactly what they hold.  Its draft, a token below, is never kept."""
    rng = np.random.default_rng(vocab)
    rows, top_k, draft = [], [], []
    for row in np.floor(rng.exponential(size=(8, vocab)) * 4).astype(np.float32):
        counts = [(t, int((row >= t).sum())) for t in range(1, int(row.max()))]
        for t, n in counts:
            if 65 <= n <= 1790:
                rows.append(row)
                top_k.append(n)
                draft.append(np.flatnonzero(row == t - 1)[0])
    B = len(rows)
    ar = torch.from_numpy(np.stack(rows)[:, None])
    c = dict(ar=ar, df=ar, f=[np.full(B, 20.0, np.float32), np.array(top_k, np.int32), None, None], draft=np.array(draft, np.int32)[:, None],
             u=np.full((B, 1), 0.25, np.float32), gumbel=rng.gumbel(size=(B, vocab)).astype(np.float32))
    got = _check_consensus(c)
    assert B >= 80 and (got["accept_len"] == 0).all()


def test_consensus_of_equal_views_keeps_every_draft():
    c = _case(41, len(FILTERS), 6, 3000, FILTERS, noise=0.0)
    got = _check_consensus(c)
    assert (got["accept_len"] == 6).all()


def test_drafts_outside_the_vocabulary_outside_the_support_and_empty_rows():
    B, K, V = len(FILTERS), 4, 1500
    c = _case(43, B, K, V, FILTERS)
    c["draft"][::3, 0] = [-1, V, -2 ** 31, 2 ** 31 - 1][:len(c["draft"][::3])] * 1
    c["draft"][1::3, 1] = 0                       # hardly ever kept by anybody
    c["ar"][2, 0] = -float("inf")                 # nothing to emit
    c["df"][5, :] = -float("inf")                 # q is zero everywhere: every draft that p allows is kept
    c["ar"][8, 1] = float("nan")
    want = oracle.filtered_consensus_commit(c["ar"].numpy(), c["df"].numpy(), *c["f"], c["draft"], c["u"], c["gumbel"])
    got, err = _consensus(c)
    assert err == 0 and got["out_tokens"][2, 0] == -1 and got["next_anchor"][2] == -1
    for k in ("accept_len", "num_committed", "out_tokens", "next_anchor"):
        np.testing.assert_array_equal(got[k], want[k], err_msg=k)


@pytest.mark.parametrize("layers", [1, 3])
@pytest.mark.parametrize("in_place", [False, True])
def test_consensus_commit_and_capacity(layers, in_place):
    B, K, V, H, P, d, pages = len(FILTERS), 8, 900, 2, 16, 64, 60
    c = _case(47, B, K, V, FILTERS)
    rng = np.random.default_rng(48)
    bits = lambda *s: rng.integers(0, 1 << 16, s, dtype=np.uint16)  # noqa: E731
    table = rng.permutation(pages)[:B * 3].reshape(B, 3).astype(np.int32)
    lens = rng.integers(0, 2 * P, B).astype(np.int32)
    table[3, 1:] = -1
    lens[3] = P                                   # its next page is not mapped
    lens[6] = 3 * P                               # its table is full
    cm = dict(k_pool=bits(layers, pages, H, P, d), v_pool=bits(layers, pages, H, P, d), page_table=table, seq_lens=lens,
              k_blk=bits(layers, B, K, H, d), v_blk=bits(layers, B, K, H, d))
    got, err = _consensus(c, commit=cm, in_place=in_place)
    want = oracle.filtered_consensus_commit(c["ar"].numpy(), c["df"].numpy(), *c["f"], c["draft"], c["u"], c["gumbel"],
                                            cm["k_blk"], cm["v_blk"], cm["k_pool"], cm["v_pool"], table, lens)
    assert err == -4 == want["status"] and got["num_committed"][3] == 0 == got["num_committed"][6]
    for k in ("accept_len", "num_committed", "out_tokens", "next_anchor"):
        np.testing.assert_array_equal(got[k], want[k], err_msg=k)
    for k in ("k_pool", "v_pool", "seq_lens"):    # (the oracle has updated them in place)
        np.testing.assert_array_equal(got[k], cm[k], err_msg=k)


def test_without_filters_the_decisions_are_those_of_the_sampling_consensus():
    B, K, V = 6, 8, 5000
    c = _case(51, B, K, V, [(0.8, 0, 1.0, 0.0)] * B)
    got = _check_consensus(c)
    step = _step(B, K, V)
    acc, ncm, anchor = (torch.full((B,), -7, dtype=torch.int32, device="cuda") for _ in range(3))
    toks = torch.full((B, K), -7, dtype=torch.int32, device="cuda")
    step.sampling_consensus_commit(0.8, c["ar"].cuda(), c["df"].cuda(), _dev(c["draft"]), _dev(c["u"]), _dev(c["gumbel"]), None, None,
                                   None, None, None, None, acc, ncm, toks, anchor)
    torch.cuda.synchronize()
    step.close()
    for k, v in (("accept_len", acc), ("num_committed", ncm), ("out_tokens", toks), ("next_anchor", anchor)):
        np.testing.assert_array_equal(got[k], v.cpu().numpy(), err_msg=k)


def test_consensus_of_the_largest_vocabulary():
    _check_consensus(_case(48, 4, 2, 1 << 20, [FILTERS[0], FILTERS[1], FILTERS[4], FILTERS[2]]))


@pytest.mark.parametrize("K,dtype", [(4, "f32"), (13, "f32"), (32, "bf16")])
def test_consensus_in_two_stages(K, dtype):
    """More logits than the last-level cache holds: the later rows are gone through only where the first drafts were all kept.
    The rows behind a lost draft hold NaN, which nothing may read anything from."""
    V = 151936 if dtype == "f32" else 160001
    B = (220 << 20) // (2 * K * V * (4 if dtype == "f32" else 2)) + 1
    rows = [FILTERS[b % len(FILTERS)] for b in range(B)]
    c = _case(61 + K, B, K, V, rows, noise=0.25, dtype=dtype)
    first = (3 * K + 7) // 8
    c["draft"][1, first - 1] = -1       # lost at the last row of the first stage
    if B > 2:
        c["draft"][2, first:first + 1] = -1   # at the first of the second
    got = _check_consensus(c)
    for b in range(B):
        c["ar"][b, got["accept_len"][b] + 1:] = float("nan")
        c["df"][b, got["accept_len"][b] + 1:] = float("nan")
    again, err = _consensus(c)
    assert err == 0
    for k in got:
        np.testing.assert_array_equal(again[k], got[k], err_msg=k)
