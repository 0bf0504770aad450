"""Refusals of the sampling, page-table and store entry points: found on the host before anything touches a device, so they
are checked here with addresses that are never read (a call that were not refused would end in ORTHRUS_EHIP)."""
import ctypes

import pytest
import torch

import paper_2605_12825_amd as orthrus
from paper_2605_12825_amd import binding as B

A = 1 << 20      # an aligned address
_keep = ctypes.create_string_buffer(1 << 12)
CTX = ctypes.addressof(_keep)


class _Space:
    def __init__(self, nbytes, at=A):
        self.nbytes, self.at = nbytes, at

    def data_ptr(self):
        return self.at


def _params(**kw):
    full = dict(batch=3, num_q_heads=8, num_kv_heads=2, head_dim=128, block_k=4, page_size=16, max_pages_per_seq=9,
                max_seq_len=100, num_pages=50, vocab=1000)
    full.update(kw)
    return orthrus.make_params(**full)


def _sample(p=None, ctx=CTX, logits_type=0, stride=0, ws=None, **kw):
    a = dict(logits=A, temperature=A, top_k=A, top_p=A, min_p=A, u=A, tokens=A, logprobs=A)
    a.update(kw)
    return orthrus.orthrus_sample_tokens(ctx, p or _params(), logits_type, a["logits"], stride, a["temperature"], a["top_k"],
                                         a["top_p"], a["min_p"], a["u"], a["tokens"], a["logprobs"],
                                         ws or _Space(1 << 40), 0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(ctx=None), B.ORTHRUS_EINVAL), (dict(logits=None), B.ORTHRUS_EINVAL), (dict(temperature=None), B.ORTHRUS_EINVAL),
    (dict(u=None), B.ORTHRUS_EINVAL), (dict(tokens=None), B.ORTHRUS_EINVAL), (dict(logits_type=3), B.ORTHRUS_EINVAL),
    (dict(logits_type=-1), B.ORTHRUS_EINVAL), (dict(stride=999), B.ORTHRUS_EINVAL), (dict(stride=-1), B.ORTHRUS_EINVAL),
    (dict(logits=A + 2), B.ORTHRUS_EINVAL), (dict(logits=A + 1, logits_type=1), B.ORTHRUS_EINVAL),
    (dict(u=A + 2), B.ORTHRUS_EINVAL), (dict(logprobs=A + 1), B.ORTHRUS_EINVAL), (dict(top_k=A + 3), B.ORTHRUS_EINVAL),
    (dict(p=_params(vocab=0)), B.ORTHRUS_EINVAL), (dict(p=_params(vocab=(1 << 20) + 1)), B.ORTHRUS_EUNSUPPORTED),
    (dict(p=_params(batch=65535, block_k=32, vocab=1 << 20)), B.ORTHRUS_EUNSUPPORTED),   # more than a launch counts
    (dict(p=_params(block_k=33)), B.ORTHRUS_EUNSUPPORTED), (dict(p=_params(block_k=0)), B.ORTHRUS_EINVAL),
    (dict(p=_params(batch=-1)), B.ORTHRUS_EINVAL), (dict(p=_params(batch=70000)), B.ORTHRUS_EUNSUPPORTED),
    (dict(p=_params(batch=0)), B.ORTHRUS_OK),
])
def test_sample_tokens(kw, status):
    assert _sample(**kw) == status


def _filtered(p=None, ctx=CTX, logits_type=0, stride=0, ws=None, **kw):
    names = ("ar_logits", "diff_logits", "temperature", "top_k", "top_p", "min_p", "draft_tokens", "accept_u", "gumbel",
             "k_blk_ar", "v_blk_ar", "k_pool", "v_pool", "page_table", "seq_lens", "accept_len", "num_committed",
             "out_tokens", "next_anchor")
    a = dict.fromkeys(names, A)
    a.update(kw)
    v = [a[n] for n in names]
    return orthrus.orthrus_filtered_consensus_commit(ctx, p or _params(), logits_type, v[0], v[1], stride, *v[2:],
                                                     workspace=ws or _Space(1 << 40), stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(ctx=None), B.ORTHRUS_EINVAL), (dict(diff_logits=None), B.ORTHRUS_EINVAL), (dict(gumbel=None), B.ORTHRUS_EINVAL),
    (dict(accept_u=None), B.ORTHRUS_EINVAL), (dict(temperature=None), B.ORTHRUS_EINVAL), (dict(k_blk_ar=None), B.ORTHRUS_EINVAL),
    (dict(v_pool=None), B.ORTHRUS_EINVAL), (dict(seq_lens=None), B.ORTHRUS_EINVAL), (dict(next_anchor=None), B.ORTHRUS_EINVAL),
    (dict(stride=5), B.ORTHRUS_EINVAL), (dict(logits_type=9), B.ORTHRUS_EINVAL), (dict(k_pool=A + 8), B.ORTHRUS_EINVAL),
    (dict(diff_logits=A + 2), B.ORTHRUS_EINVAL), (dict(gumbel=A + 2), B.ORTHRUS_EINVAL),
    (dict(p=_params(vocab=1 << 22)), B.ORTHRUS_EUNSUPPORTED), (dict(p=_params(num_layers=0)), B.ORTHRUS_EINVAL),
    (dict(p=_params(num_layers=70000)), B.ORTHRUS_EUNSUPPORTED), (dict(p=_params(page_size=24)), B.ORTHRUS_EUNSUPPORTED),
    (dict(ws=_Space(16)), B.ORTHRUS_EWORKSPACE), (dict(ws=_Space(1 << 40, A + 128)), B.ORTHRUS_EWORKSPACE),
    (dict(p=_params(batch=0)), B.ORTHRUS_OK),
])
def test_filtered_consensus(kw, status):
    assert _filtered(**kw) == status


def _tables(p=None, ctx=CTX, max_tokens=10, ws=None, **kw):
    names = ("seq_lens", "new_lens", "page_table", "free_pages", "free_state", "granted", "token_starts", "slot_map")
    a = dict.fromkeys(names, A)
    a.update(kw)
    return orthrus.orthrus_page_tables_update(ctx, p or _params(), *[a[n] for n in names], max_tokens, ws or _Space(1 << 30), 0,
                                              check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(ctx=None), B.ORTHRUS_EINVAL), (dict(seq_lens=None), B.ORTHRUS_EINVAL), (dict(free_state=None), B.ORTHRUS_EINVAL),
    (dict(slot_map=None), B.ORTHRUS_EINVAL), (dict(token_starts=None), B.ORTHRUS_EINVAL), (dict(max_tokens=-1), B.ORTHRUS_EINVAL),
    (dict(max_tokens=1 << 31), B.ORTHRUS_EUNSUPPORTED), (dict(granted=A + 2), B.ORTHRUS_EINVAL),
    (dict(p=_params(max_seq_len=9 * 16 + 1)), B.ORTHRUS_EINVAL), (dict(p=_params(max_seq_len=-1)), B.ORTHRUS_EINVAL),
    (dict(p=_params(num_pages=1 << 27)), B.ORTHRUS_EUNSUPPORTED), (dict(p=_params(num_pages=0)), B.ORTHRUS_EINVAL),
    (dict(ws=_Space(8)), B.ORTHRUS_EWORKSPACE), (dict(ws=_Space(1 << 30, A + 4)), B.ORTHRUS_EWORKSPACE),
])
def test_page_tables(kw, status):
    assert _tables(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(ctx=None), B.ORTHRUS_EINVAL), (dict(k=None), B.ORTHRUS_EINVAL), (dict(slots=None), B.ORTHRUS_EINVAL),
    (dict(vp=None), B.ORTHRUS_EINVAL), (dict(n=-1), B.ORTHRUS_EINVAL), (dict(k=A + 8), B.ORTHRUS_EINVAL),
    (dict(slots=A + 2), B.ORTHRUS_EINVAL), (dict(count=A + 1), B.ORTHRUS_EINVAL), (dict(p=_params(num_layers=0)), B.ORTHRUS_EINVAL),
    (dict(p=_params(num_pages=1 << 27)), B.ORTHRUS_EUNSUPPORTED), (dict(p=_params(head_dim=96)), B.ORTHRUS_EUNSUPPORTED),
    (dict(p=_params(blk_stride_row=100)), B.ORTHRUS_EUNSUPPORTED), (dict(n=0), B.ORTHRUS_OK),
    (dict(n=0, k=None, v=None, slots=None), B.ORTHRUS_OK), (dict(n=0, kp=None), B.ORTHRUS_EINVAL),
])
def test_kv_store(kw, status):
    a = dict(ctx=CTX, p=_params(), n=5, k=A, v=A, slots=A, count=None, kp=A, vp=A)
    a.update(kw)
    assert orthrus.orthrus_kv_store(a["ctx"], a["p"], a["n"], a["k"], a["v"], a["slots"], a["count"], a["kp"], a["vp"], 0,
                                    check=False) == status


def test_kv_store_of_more_rows_than_a_launch_counts():
    """A workgroup of 256 threads to a row of 8192 elements and more, 32 bits for the threads of a launch."""
    def store(n, heads):
        return orthrus.orthrus_kv_store(CTX, _params(num_q_heads=heads, num_kv_heads=heads), n, A, A, A, None, A, A, 0, check=False)
    assert store(1 << 24, 64) == store(2 ** 31 - 1, 64) == store(2 ** 31 - 1, 1000) == store(2 ** 31 - 1, 8) == B.ORTHRUS_EUNSUPPORTED
    # (what is not refused gets as far as the launch, which finds no device here)


def test_logits_tensors():
    from paper_2605_12825_amd import runtime
    x = torch.zeros((2, 3, 8))
    assert runtime._logits_type(0, x) == B.ORTHRUS_F32 and runtime._logits_type(8, x[..., :5].bfloat16(), x.bfloat16()) == B.ORTHRUS_BF16
    for bad in ((0, x.double()), (0, x, x.half()), (0, x[..., :5]), (0, x, x.transpose(1, 2))):
        with pytest.raises(ValueError):
            runtime._logits_type(*bad)


def test_filter_tensors():
    from paper_2605_12825_amd import runtime
    for n in (1, 2):
        t, k = torch.zeros(n), torch.zeros(n, dtype=torch.int32)
        runtime._check_filters(n, t, k, t, t)
        runtime._check_filters(n, t, None, None, None)
        runtime._check_filters(n, A, A, A, A)
        runtime._check_filters(n, None, k, t, t)       # (refused by the library)
        bad = [(t, k.long(), t, t), (t.double(), k, t, t), (t, k, t.half(), t), (t, k, t, k), (k, k, t, t), (t, t, t, t)]
        if n == 2:
            bad += [(t[:1], k, t, t), (t, k[:1], t, t), (t, k, torch.zeros(2, 4)[:, 0], t), (t, k, t, t[:1].expand(2))]
        for f in bad:
            with pytest.raises(ValueError):
                runtime._check_filters(n, *f)


def test_tokens_and_random_numbers_of_another_type():
    from paper_2605_12825_amd import runtime
    step = object.__new__(runtime.DecodeStep)
    step.params, step.ctx, step.sample_ws, step.filtered_ws = _params(batch=1), CTX, _Space(8), _Space(8)   # (too small: nothing is launched)
    x, t, u, i = torch.zeros(1, 4, 1000), torch.zeros(1), torch.zeros(1, 4), torch.zeros(1, 4, dtype=torch.int32)
    n, gumbel = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1000)
    verify = [i, u, gumbel] + [None] * 6 + [n, n, i, n]
    step.params.vocab = 5000
    for f, args, names in ((step.sample_tokens, [u, i], (0, 1)), (step.filtered_consensus_commit, verify, (0, 1, 2, 11))):
        logits = [x] if f == step.sample_tokens else [x, x]
        with pytest.raises(orthrus.OrthrusError):
            f(*logits, t, None, None, None, *args, stream=0)
        for k in names:
            for bad in (args[k].double(), args[k].long()):
                with pytest.raises(ValueError):
                    f(*logits, t, None, None, None, *args[:k], bad, *args[k + 1:], stream=0)
    step.ctx = None


def test_page_table_tensors():
    from paper_2605_12825_amd import runtime
    step = object.__new__(runtime.DecodeStep)
    step.params, step.ctx, step.tables_ws = _params(), CTX, _Space(8)     # (a workspace that is too small: nothing is launched)
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    good = [i32(3), i32(3), i32(3, 9), i32(50), i32(2), i32(3), i32(4), i32(10)]
    with pytest.raises(orthrus.OrthrusError):
        step.update_page_tables(*good, stream=0)
    for i, x in ((1, good[1].long()), (1, good[1].float()), (3, good[3][1:])):
        with pytest.raises(ValueError):
            step.update_page_tables(*good[:i], x, *good[i + 1:], stream=0)
    step.ctx = None


@pytest.mark.parametrize("explicit", [False, True])
def test_rows_of_a_store(explicit):
    from paper_2605_12825_amd import runtime
    step = object.__new__(runtime.DecodeStep)
    step.ctx = None
    step.params = _params(num_layers=2, **(dict(blk_stride_row=20 * 128, blk_stride_head=128, blk_stride_layer=7 * 20 * 128) if explicit else {}))
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    x, k = z(2, 30, 20, 128), z(2, 30, 2, 128)
    p = step._params_for_rows(x[:, :, :2], x[:, :, 2:4], 30)
    assert (p.blk_stride_layer, p.blk_stride_row, p.blk_stride_head) == (30 * 20 * 128, 20 * 128, 128)
    p = step._params_for_rows(k, k, 30)
    assert (p.blk_stride_layer, p.blk_stride_row, p.blk_stride_head) == (30 * 256, 256, 128) and p.num_pages == 50
    p = step._params_for_rows(z(2, 1, 2, 128), x[:, :1, :2].contiguous(), 1)
    assert (p.blk_stride_layer, p.blk_stride_row, p.blk_stride_head) == (256, 0, 128)
    p = step._params_for_rows(z(2, 0, 2, 128), z(2, 0, 2, 128), 0)
    assert (p.blk_stride_layer, p.blk_stride_row, p.blk_stride_head) == (0, 0, 0)
    with pytest.raises(ValueError):
        step.store_kv(k, k, torch.zeros(30, dtype=torch.int64), A, A)
    wide = z(2, 30, 2, 256)[..., ::2]
    for a, b, n in ((k, k, 31), (k[:, :29], k, 30), (k, k[:1], 30), (k[0], k[0], 30), (k.float(), k.float(), 30), (k, k.float(), 30),
                    (k, x[:, :, :2], 30), (wide, wide, 30), (k[:1].expand(2, -1, -1, -1), k, 30), (k.transpose(1, 2), k.transpose(1, 2), 30),
                    (k[:, :1].expand(-1, 30, -1, -1),) * 2 + (30,)):
        with pytest.raises(ValueError):
            step._params_for_rows(a, b, n)


def test_workspace_queries():
    for f in (orthrus.orthrus_sample_workspace_bytes, orthrus.orthrus_filtered_workspace_bytes):
        assert f(_params()) >= 0 and f(_params(batch=0)) >= 0
        with pytest.raises(orthrus.OrthrusError):
            f(_params(vocab=1 << 22))
    # per row and view what its filters keep (24 bytes and more), two words per sequence
    assert orthrus.orthrus_filtered_workspace_bytes(_params()) >= 2 * 12 * 24 + 3 * 2 * 4
    assert orthrus.orthrus_page_tables_workspace_bytes(_params()) >= (3 * 3 + 2) * 4
    with pytest.raises(orthrus.OrthrusError):
        orthrus.orthrus_page_tables_workspace_bytes(_params(max_seq_len=9 * 16 + 1))
    with pytest.raises(orthrus.OrthrusError):
        orthrus.orthrus_page_tables_workspace_bytes(_params(num_pages=1 << 27))
