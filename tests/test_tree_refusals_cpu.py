"""Refusals of the tree and logit-rule entry points: found on the host before anything touches a device, so they are checked here with
addresses that are never read (a call that were not refused would end in ORTHRUS_EHIP)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2605_12825_amd as orthrus
from paper_2605_12825_amd import binding as B
from paper_2605_12825_amd import runtime as rt

A = 1 << 20      # an aligned address
_keep = ctypes.create_string_buffer(1 << 12)
CTX = ctypes.addressof(_keep)
EINVAL, EUNSUPPORTED, EWORKSPACE = B.ORTHRUS_EINVAL, B.ORTHRUS_EUNSUPPORTED, B.ORTHRUS_EWORKSPACE


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


def _attn(p=None, ctx=CTX, nodes=40, ws=None, **kw):
    names = ("parents", "q", "k_blk", "v_blk", "k_pool", "v_pool", "page_table", "seq_lens", "out", "lse")
    a = dict.fromkeys(names, A)
    a.update(kw)
    return orthrus.orthrus_tree_attn(ctx, p or _params(), nodes, *[a[n] for n in names], workspace=ws or _Space(1 << 40), stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(ctx=None), EINVAL), (dict(nodes=0), EINVAL), (dict(nodes=-1), EINVAL), (dict(nodes=65), EUNSUPPORTED),
    (dict(p=_params(num_q_heads=32), nodes=33), EUNSUPPORTED), (dict(p=_params(batch=0, num_q_heads=32), nodes=32), B.ORTHRUS_OK),
    (dict(p=_params(batch=0)), B.ORTHRUS_OK), (dict(p=_params(batch=0, block_k=40)), B.ORTHRUS_OK),   # block_k is not this call's
    (dict(p=_params(num_q_heads=7)), EINVAL), (dict(p=_params(head_dim=96)), EUNSUPPORTED), (dict(p=_params(page_size=8)), EUNSUPPORTED),
    (dict(p=_params(max_seq_len=200)), EINVAL), (dict(p=_params(num_splits=-2)), EINVAL), (dict(p=_params(sm_scale=0.0)), EINVAL),
    (dict(p=_params(pool_stride_tok=132)), EUNSUPPORTED), (dict(p=_params(batch=-1)), EINVAL),
    (dict(q=A + 8), EINVAL), (dict(v_pool=A + 2), EINVAL), (dict(parents=A + 2), EINVAL), (dict(lse=A + 1), EINVAL),
    (dict(p=_params(num_splits=3), ws=_Space(64)), EWORKSPACE), (dict(p=_params(num_splits=-1), ws=_Space(1 << 40, A + 128)), EWORKSPACE),
    (dict(p=_params(batch=65535, num_kv_heads=2, num_q_heads=16, max_pages_per_seq=1 << 20, max_seq_len=1 << 24, num_pages=1 << 26, num_splits=60000), nodes=64), EUNSUPPORTED),
] + [(dict([(n, None)]), EINVAL) for n in ("parents", "q", "k_blk", "v_blk", "k_pool", "v_pool", "page_table", "seq_lens", "out")])
def test_tree_attn(kw, status):
    assert _attn(**kw) == status


def test_tree_attn_workspaces():
    need = lambda p, n: orthrus.orthrus_tree_attn_workspace_bytes(None, p, n)  # noqa: E731
    assert need(_params(num_splits=1), 40) == 0
    units, rows = 3 * 2, 4 * 40
    n = need(_params(num_splits=3, max_seq_len=140), 40)
    assert n >= units * 3 * rows * (128 + 2) * 4
    # two row groups share a head's rows; in the balanced form a workgroup holds at most seven blocks of 32
    assert need(_params(num_splits=2, num_q_heads=16), 64) == need(_params(num_splits=2, num_kv_heads=4, num_q_heads=16), 64)
    assert need(_params(num_splits=-1), 64) == 2 * 256 * 128 * (128 + 2) * 4
    for p, nodes in ((_params(), 0), (_params(), 65), (_params(num_q_heads=7), 3), (_params(head_dim=32), 3)):
        with pytest.raises(orthrus.OrthrusError):
            need(p, nodes)


def _walk(p=None, ctx=CTX, logits_type=0, stride=0, nodes=40, max_path=9, ws=None, **kw):
    names = ("parents", "node_tokens", "k_blk_ar", "v_blk_ar", "k_pool", "v_pool", "page_table", "seq_lens", "accept_len", "num_committed",
             "path_nodes", "out_tokens", "next_anchor")
    a = {n: A + 64 * i for i, n in enumerate(names)}
    a.update(kw)
    return orthrus.orthrus_tree_consensus_commit(ctx, p or _params(), logits_type, a.pop("ar_logits", A), stride, nodes, max_path,
                                                 *[a[n] for n in names], workspace=ws or _Space(1 << 40), stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(ctx=None), EINVAL), (dict(nodes=0), EINVAL), (dict(nodes=65), EUNSUPPORTED), (dict(max_path=0), EINVAL), (dict(max_path=-1), EINVAL),
    (dict(logits_type=3), EINVAL), (dict(stride=999), EINVAL), (dict(stride=-1), EINVAL), (dict(ar_logits=A + 2), EINVAL),
    (dict(ar_logits=A + 1, logits_type=2), EINVAL), (dict(ar_logits=None), EINVAL), (dict(k_blk_ar=None), EINVAL),
    (dict(p=_params(vocab=0)), EINVAL), (dict(p=_params(vocab=(1 << 20) + 1)), EUNSUPPORTED), (dict(p=_params(num_layers=0)), EINVAL),
    (dict(p=_params(num_layers=70000)), EUNSUPPORTED), (dict(k_pool=A + 8), EINVAL), (dict(path_nodes=A + 2), EINVAL), (dict(seq_lens=A + 1), EINVAL),
    (dict(out_tokens=A, node_tokens=A), EINVAL), (dict(out_tokens=A, parents=A), EINVAL), (dict(path_nodes=A, node_tokens=A), EINVAL),
    (dict(path_nodes=A, parents=A), EINVAL), (dict(path_nodes=A, out_tokens=A), EINVAL),
    (dict(ws=_Space(16)), EWORKSPACE), (dict(ws=_Space(1 << 40, A + 64)), EWORKSPACE),
    (dict(p=_params(batch=0)), B.ORTHRUS_OK), (dict(p=_params(batch=0, block_k=33), max_path=1000), B.ORTHRUS_OK),
    (dict(p=_params(batch=0, head_dim=7), k_blk_ar=None, v_blk_ar=None), B.ORTHRUS_OK),   # consensus only: no cache
] + [(dict([(n, None)]), EINVAL) for n in ("parents", "node_tokens", "accept_len", "num_committed", "path_nodes", "out_tokens", "next_anchor",
                                           "k_pool", "page_table", "seq_lens")])
def test_tree_consensus(kw, status):
    assert _walk(**kw) == status


def _rules(**kw):
    full = dict(history=A, history_lens=A, prompt_lens=A, history_stride=10, repetition=A, presence=A, frequency=A, bias_starts=A, bias_tokens=A,
                bias_values=A, num_biases=5, masks=A, mask_rows=A, num_masks=2, mask_stride=0)
    full.update(kw)
    r = B.orthrus_logit_rules()
    for k, v in full.items():
        setattr(r, k, v)
    return r


def _process(p=None, ctx=CTX, logits_type=0, stride=0, out_stride=0, rows=3, logits=A, out=A, tokens=A, parents=A, rules=None, none=False, **kw):
    return orthrus.orthrus_logits_process(ctx, p or _params(batch=0), logits_type, logits, stride, rows, tokens, parents,
                                          None if none else rules or _rules(**kw), out, out_stride, 0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(), B.ORTHRUS_OK), (dict(ctx=None), EINVAL), (dict(logits=None), EINVAL), (dict(out=None), EINVAL), (dict(none=True), EINVAL),
    (dict(rows=0), EINVAL), (dict(rows=65), EUNSUPPORTED), (dict(rows=64), B.ORTHRUS_OK), (dict(logits_type=3), EINVAL),
    (dict(stride=999, out_stride=999), EINVAL), (dict(stride=1001), EINVAL), (dict(stride=1001, out_stride=1001), B.ORTHRUS_OK),   # in place: one stride
    (dict(stride=1001, out=2 * A), B.ORTHRUS_OK), (dict(out=2 * A + 2), EINVAL), (dict(out=2 * A + 2, logits_type=1), B.ORTHRUS_OK),
    (dict(logits=A + 1, logits_type=1), EINVAL), (dict(tokens=A + 2), EINVAL), (dict(parents=A + 1), EINVAL), (dict(tokens=None), B.ORTHRUS_OK),
    (dict(history=None), EINVAL), (dict(history_lens=None), EINVAL), (dict(history=None, history_lens=None), EINVAL),
    (dict(history=None, history_lens=None, prompt_lens=None), B.ORTHRUS_OK), (dict(history_stride=0), EINVAL), (dict(history=A + 2), EINVAL),
    (dict(presence=A + 2), EINVAL), (dict(bias_starts=None), EINVAL), (dict(bias_tokens=None), EINVAL), (dict(bias_values=None), EINVAL),
    (dict(num_biases=-1), EINVAL), (dict(num_biases=0, bias_tokens=None, bias_values=None), B.ORTHRUS_OK), (dict(mask_rows=None), EINVAL),
    (dict(masks=None), EINVAL), (dict(masks=None, mask_rows=None), B.ORTHRUS_OK), (dict(num_masks=-1), EINVAL), (dict(mask_stride=31), EINVAL),
    (dict(mask_stride=32), B.ORTHRUS_OK), (dict(mask_stride=-32), EINVAL), (dict(masks=A + 2), EINVAL), (dict(p=_params(vocab=0)), EINVAL),
    (dict(p=_params(vocab=(1 << 20) + 1)), EUNSUPPORTED), (dict(p=_params(batch=70000)), EUNSUPPORTED),
    (dict(p=_params(batch=65535, vocab=20000), rows=64), EUNSUPPORTED),
])
def test_logits_process(kw, status):
    assert _process(**kw) == status


def test_rules_struct_matches_the_header():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "orthrus.h")).read()
    end = text.index("} orthrus_logit_rules;")
    body = re.sub(r"/\*.*?\*/", "", text[text.rindex("typedef struct {", 0, end):end], flags=re.S)
    fields = re.findall(r"\b((?:const )?\w+) \*?([a-z_]+)\s*;", body)
    assert [f[1] for f in fields] == [f[0] for f in B.orthrus_logit_rules._fields_]
    for (kind, name), (_, ctype) in zip(fields, B.orthrus_logit_rules._fields_):
        assert ctype is (ctypes.c_void_p if kind.startswith("const") else ctypes.c_int64), name


def test_rules_of_the_wrong_kind_are_refused():
    i32, f32 = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    h = torch.zeros((4, 9), dtype=torch.int32)
    rt.LogitRules(history=h, history_lens=i32, repetition=f32)
    for kw in (dict(history=h), dict(history=h.long(), history_lens=i32), dict(history=i32, history_lens=i32), dict(history=h.t(), history_lens=i32),
               dict(prompt_lens=i32), dict(repetition=i32), dict(presence=f32.double()), dict(bias_starts=i32), dict(bias_tokens=i32, bias_values=f32),
               dict(bias_starts=i32, bias_tokens=i32, bias_values=f32[:3]), dict(masks=h), dict(mask_rows=i32), dict(masks=h.long(), mask_rows=i32)):
        with pytest.raises(ValueError):
            rt.LogitRules(**kw)
    for kw, call in ((dict(repetition=f32), (5, 1, 30)), (dict(history=h, history_lens=i32), (5, 1, 30)), (dict(history=h[:3], history_lens=i32), (4, 1, 30)),
                     (dict(masks=h, mask_rows=i32), (4, 2, 30)), (dict(masks=h, mask_rows=i32), (4, 1, 289)), (dict(masks=h, mask_rows=i32), (2, 1, 30)),
                     (dict(bias_starts=i32, bias_tokens=i32, bias_values=f32), (4, 1, 30))):
        with pytest.raises(ValueError):
            rt.LogitRules(**kw).check(*call)
    with pytest.raises(ValueError):   # on another device than the logits
        rt.LogitRules(repetition=f32).check(4, 1, 30, torch.device("cuda", 0))
    rt.LogitRules(repetition=f32).check(4, 1, 30, f32.device)
    rt.LogitRules(masks=h, mask_rows=i32.view(2, 2)).check(2, 2, 288)
    none = rt.LogitRules(history=h[:, :0].contiguous(), history_lens=i32, prompt_lens=i32, masks=h[:0], mask_rows=i32, bias_starts=i32,
                         bias_tokens=i32[:0], bias_values=f32[:0])   # nothing in them: the same as without
    assert not none.c.history and not none.c.history_lens and not none.c.prompt_lens and not none.c.masks and not none.c.mask_rows
    assert _process(rules=none.c, p=_params(batch=0)) == B.ORTHRUS_OK
    rt.LogitRules(bias_starts=i32, bias_tokens=i32, bias_values=f32).check(3, 7, 30)


class _Step(rt.DecodeStep):
    """The checks of a step without a device."""

    def __init__(self, **kw):
        self.params, self.ctx = _params(**kw), None
        self._tree_attn_key = self._tree_consensus_key = (None, None)

    def _stream(self, stream):
        raise AssertionError("not refused")

    _tree_attn_ws = _tree_consensus_ws = _stream


def test_operands_of_another_type_or_size_are_refused():
    s, N = _Step(), 5
    i = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    h = lambda *n: torch.zeros(n, dtype=torch.bfloat16)  # noqa: E731
    good = dict(parents=i(3, N), q=h(3, N, 8, 128), k_blk=h(3, N, 2, 128), v_blk=h(3, N, 2, 128), k_pool=A, v_pool=A, page_table=A, seq_lens=A,
                out=h(3, N, 8, 128), lse=torch.zeros((3, 8, N)))
    with pytest.raises(AssertionError):
        s.tree_attn(**good)
    for name, bad in (("parents", i(3, N).long()), ("parents", i(N, 3).t()), ("parents", i(2, N)), ("q", h(3, N, 8, 64)), ("q", h(3, N, 8, 128).float()),
                      ("q", h(3, N, 128, 8).transpose(2, 3)), ("k_blk", h(3, N, 4, 128)[:, :, :2]), ("v_blk", h(3, 4, 2, 128)), ("out", h(3, N, 8, 256)[..., :128]),
                      ("out", torch.zeros((3, N, 8, 128))), ("lse", torch.zeros((3, 8, N)).double()), ("lse", torch.zeros((3, 4, N)))):
        with pytest.raises(ValueError):
            s.tree_attn(**dict(good, **{name: bad}))
    good = dict(ar_logits=torch.zeros((3, N, 1000)), parents=i(3, N), node_tokens=i(3, N), k_blk_ar=h(1, 3, N, 2, 128), v_blk_ar=h(1, 3, N, 2, 128),
                k_pool=A, v_pool=A, page_table=A, seq_lens=A, accept_len=i(3), num_committed=i(3), path_nodes=i(3, N), out_tokens=i(3, N), next_anchor=i(3))
    with pytest.raises(AssertionError):
        s.tree_consensus_commit(**good)
    for name, bad in (("ar_logits", torch.zeros((3, N, 999))), ("ar_logits", torch.zeros((3, N, 1000)).double()), ("node_tokens", i(3, N).long()),
                      ("ar_logits", torch.zeros((3, N, 1001))[..., :1000]), ("path_nodes", i(3, 4)), ("out_tokens", i(N, 3).t()), ("accept_len", i(2)),
                      ("next_anchor", torch.zeros(3)), ("k_blk_ar", h(2, 3, N, 2, 128)), ("v_blk_ar", h(1, 3, N, 4, 128)[:, :, :, :2])):
        with pytest.raises(ValueError):
            s.tree_consensus_commit(**dict(good, **{name: bad}))
    with pytest.raises(AssertionError):   # rows of a padded head, with their stride
        s.tree_consensus_commit(**dict(good, ar_logits=torch.zeros((3, N, 1001))), logits_stride_row=1001)
    with pytest.raises(ValueError):       # the last row ends behind the memory
        s.tree_consensus_commit(**dict(good, ar_logits=torch.zeros((3, N, 1000))), logits_stride_row=1001)
    x, r = torch.zeros((3, N, 1000)), rt.LogitRules()
    for kw in (dict(logits=x[:2], rules=r), dict(logits=x[0, 0], rules=r), dict(logits=x, rules=r, tokens=i(3, N).long()), dict(logits=x, rules=r, tokens=i(3, 4)),
               dict(logits=x, rules=r, tokens=i(3, N), parents=i(3, 4)), dict(logits=x, rules=r, out=x.half()), dict(logits=x, rules=r, out=x[:, :4]),
               dict(logits=x.double(), rules=r), dict(logits=x[..., ::2], rules=r), dict(logits=x, rules=r, out=torch.zeros((3, N, 1000)), out_stride_row=1001)):
        with pytest.raises(ValueError):
            s.process_logits(**kw)
    for kw in (dict(logits=x, rules=r), dict(logits=x[:, 0].contiguous(), rules=r, tokens=i(3, 1)), dict(logits=x, rules=r, out=torch.zeros((3, N, 1003)), out_stride_row=1003)):
        with pytest.raises(AssertionError):
            s.process_logits(**kw)


def test_logits_do_not_go_from_one_device_to_another():
    with pytest.raises(ValueError):
        _Step().process_logits(torch.zeros((3, 5, 1000)), rt.LogitRules(), out=torch.zeros((3, 5, 1000), device="meta"))
