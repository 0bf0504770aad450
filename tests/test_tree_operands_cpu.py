"""What the tree and rule calls of a DecodeStep make of operands that do not lie as the call would read them: refused on the host, before
anything touches a device."""
import ctypes

import pytest
import torch

import paper_2605_12825_amd as orthrus
from paper_2605_12825_amd import runtime as rt

B, N, V = 3, 5, 1000


class _Accepted(Exception):
    pass


class _Step(rt.DecodeStep):
    """The checks of a step without a device."""

    def __init__(self, **kw):
        full = dict(batch=B, num_q_heads=8, num_kv_heads=2, head_dim=128, block_k=4, page_size=16, max_pages_per_seq=9, max_seq_len=100, num_pages=50,
                    vocab=V)
        full.update(kw)
        self.params, self.ctx = orthrus.make_params(**full), None
        self._tree_attn_key = self._tree_consensus_key = (None, None)

    def _stream(self, stream):
        raise _Accepted

    _tree_attn_ws = _tree_consensus_ws = _stream


def _i(*n):
    return torch.zeros(n, dtype=torch.int32)


def _h(*n):
    return torch.zeros(n, dtype=torch.bfloat16)


A = 1 << 20   # an address


def _walk_args(**kw):
    a = dict(ar_logits=torch.zeros((B, N, V)), parents=_i(B, N), node_tokens=_i(B, N), k_blk_ar=_h(1, B, N, 2, 128), v_blk_ar=_h(1, B, N, 2, 128),
             k_pool=A, v_pool=A, page_table=A, seq_lens=A, accept_len=_i(B), num_committed=_i(B), path_nodes=_i(B, N), out_tokens=_i(B, N),
             next_anchor=_i(B))
    return dict(a, **kw)


def _full(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


# (view, rows apart): row (b, r) would be read at (b * N + r) * stride, which is another sequence's
_WRONG_ROWS = [
    (_full(B, 8, V)[:, :N], V), (_full(2 * B, N, V)[::2], V), (_full(B, 2 * N, V)[:, ::2], V), (_full(B, 2 * N, V)[:, ::2], 3 * V),
    (_full(B, 8, V)[:, 3:], V), (_full(N, B, V).transpose(0, 1), V), (_full(B, N, 2 * V)[..., ::2], 2 * V), (_full(B, V, N).transpose(1, 2), N),
    (_full(B, N, V).expand(B, N, V)[:, :1].expand(B, N, V), V), (_full(B, 8, V + 3)[:, :N, :V], V + 3), (_full(B, N, V + 3)[..., :V], V + 2),
]
_RIGHT_ROWS = [
    (_full(B, N, V), 0), (_full(B, N, V), V), (_full(B, N, V + 3), V + 3), (_full(B, N, V + 3)[..., :V], V + 3), (_full(B, N, V + 3)[..., 2:V + 2], V + 3),
    (_full(B, 2 * N, V)[:, ::2], 2 * V), (_full(2, B, N, V)[1], 0),
]


@pytest.mark.parametrize("case", range(len(_WRONG_ROWS)))
def test_logits_whose_rows_lie_elsewhere_are_refused(case):
    x, stride = _WRONG_ROWS[case]
    s, r = _Step(), rt.LogitRules()
    with pytest.raises(ValueError):
        s.tree_consensus_commit(**_walk_args(ar_logits=x), logits_stride_row=stride)
    with pytest.raises(ValueError):
        s.process_logits(x, r, logits_stride_row=stride)
    with pytest.raises(ValueError):
        s.process_logits(_full(B, N, V), r, out=x, out_stride_row=stride)


@pytest.mark.parametrize("case", range(len(_RIGHT_ROWS)))
def test_logits_whose_rows_lie_there_are_taken(case):
    x, stride = _RIGHT_ROWS[case]
    s, r = _Step(), rt.LogitRules()
    for call in (lambda: s.tree_consensus_commit(**_walk_args(ar_logits=x), logits_stride_row=stride),
                 lambda: s.process_logits(x, r, logits_stride_row=stride), lambda: s.process_logits(_full(B, N, V), r, out=x, out_stride_row=stride)):
        with pytest.raises(_Accepted):
            call()


def test_dimensions_of_one_have_no_stride():
    one = _Step(batch=1)
    for x, stride in ((_full(4, 8, V)[:1, :N], V), (_full(1, 8, V)[:, :1], 0), (_full(7, 8, V)[6:, 7:], V), (_full(1, V)[:, :], 5 * V)):
        with pytest.raises(_Accepted):
            one.process_logits(x, rt.LogitRules(), logits_stride_row=stride)
    with pytest.raises(_Accepted):   # a row a request, of the last position's among eight
        _Step().process_logits(_full(B, 8, V)[:, 7], rt.LogitRules(), logits_stride_row=8 * V)
    with pytest.raises(ValueError):
        _Step().process_logits(_full(B, 8, V)[:, 7], rt.LogitRules(), logits_stride_row=V)


def _attn_args(**kw):
    a = dict(parents=_i(B, N), q=_h(B, N, 8, 128), k_blk=_h(B, N, 2, 128), v_blk=_h(B, N, 2, 128), k_pool=_h(50, 2, 16, 128), v_pool=_h(50, 2, 16, 128),
             page_table=_i(B, 9), seq_lens=_i(B), out=_h(B, N, 8, 128))
    return dict(a, **kw)


def _committed(**kw):
    return _walk_args(**dict(dict(k_pool=_h(1, 50, 2, 16, 128), v_pool=_h(1, 50, 2, 16, 128), page_table=_i(B, 9), seq_lens=_i(B)), **kw))


_ODD_CACHES = [("seq_lens", _i(B).long()), ("seq_lens", _i(B - 1)), ("seq_lens", _i(B, 2)[:, 0]), ("seq_lens", torch.zeros(B)),
               ("page_table", _i(B, 9).long()), ("page_table", _i(B, 8)), ("page_table", _i(9, B).t()), ("page_table", _i(B, 18)[:, :9])]


@pytest.mark.parametrize("mixed", [False, True])
def test_caches_of_another_type_or_size_are_refused(mixed):
    """Lengths and pages of 64 bits would be read in halves; `mixed`: with addresses among the other operands."""
    s = _Step()
    attn, walk = (dict(k_pool=A), dict(k_pool=A)) if mixed else ({}, {})
    for call in (lambda: s.tree_attn(**_attn_args(**attn)), lambda: s.tree_consensus_commit(**_committed(**walk))):
        with pytest.raises(_Accepted):
            call()
    for name, bad in _ODD_CACHES:
        with pytest.raises(ValueError, match=name):
            s.tree_attn(**_attn_args(**attn, **{name: bad}))
        with pytest.raises(ValueError, match=name):
            s.tree_consensus_commit(**_committed(**walk, **{name: bad}))


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32, torch.int32, torch.uint8])
def test_rows_that_are_not_bf16_are_refused(dtype):
    """As many bytes of another type too."""
    s, size = _Step(), torch.empty(0, dtype=dtype).element_size()
    for name in ("q", "k_blk", "v_blk", "out", "k_pool", "v_pool"):
        good = _attn_args()[name]
        for bad in (good.to(dtype), torch.zeros(good.numel() * 2 // size, dtype=dtype)):
            with pytest.raises(ValueError, match=name):
                s.tree_attn(**_attn_args(**{name: bad}))
    for name in ("k_blk_ar", "v_blk_ar", "k_pool", "v_pool"):
        good = _committed()[name]
        for bad in (good.to(dtype), torch.zeros(good.numel() * 2 // size, dtype=dtype)):
            with pytest.raises(ValueError, match=name):
                s.tree_consensus_commit(**_committed(**{name: bad}))


def test_bits_of_bf16_are_taken_in_any_mix():
    s = _Step()
    for name in ("q", "k_blk", "out", "v_pool"):
        for dtype in (torch.int16, torch.uint16):
            with pytest.raises(_Accepted):
                s.tree_attn(**_attn_args(**{name: _attn_args()[name].view(dtype)}))
    with pytest.raises(_Accepted):
        s.tree_consensus_commit(**_committed(k_pool=_committed()["k_pool"].view(torch.int16)))


class _OnGpu(_Step):
    """Of a device of its own: the workspaces are there, the call into the library is the only thing left."""

    def __init__(self):
        super().__init__()
        self.device = torch.device("cuda", 0)

    def _tree_attn_ws(self, nodes):
        return torch.zeros(256, dtype=torch.uint8, device="meta")

    _tree_consensus_ws = _tree_attn_ws


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("elsewhere", ["cpu", "meta"])
def test_operands_on_another_device_than_the_step_are_refused(mixed, elsewhere):
    """All of them in host memory, or one call's parts of them; nothing reaches a stream or the library."""
    s = _OnGpu()
    move = lambda a: {k: v.to(elsewhere) if torch.is_tensor(v) else v for k, v in a.items()}  # noqa: E731
    attn, walk = _attn_args(lse=torch.zeros((B, 8, N))), _committed()
    if mixed:
        attn["k_pool"] = walk["k_pool"] = A
    with pytest.raises(ValueError, match="must be on cuda:0"):
        s.tree_attn(**move(attn))
    with pytest.raises(ValueError, match="must be on cuda:0"):
        s.tree_consensus_commit(**move(walk))
    with pytest.raises(ValueError, match="must be on cuda:0"):
        s.tree_consensus_commit(**move(dict(walk, k_blk_ar=None, v_blk_ar=None, k_pool=None, v_pool=None, page_table=None, seq_lens=None)))


def test_logits_and_rules_on_another_device_than_the_step_are_refused():
    class Step(_OnGpu):
        def _stream(self, stream):
            return 0
    s, x = Step(), torch.zeros((B, N, V))
    for kw in (dict(), dict(tokens=_i(B, N)), dict(out=torch.zeros((B, N, V))), dict(tokens=_i(B, N), parents=_i(B, N))):
        with pytest.raises(ValueError, match="logits must be on cuda:0"):
            s.process_logits(x, rt.LogitRules(repetition=torch.ones(B)), **kw)
    s.device = torch.device("cpu")      # the logits are where the step is, what is fed is not
    for kw in (dict(tokens=_i(B, N).to("meta")), dict(parents=_i(B, N).to("meta"))):
        with pytest.raises(ValueError, match="must be on cpu, not on meta"):
            s.process_logits(x, rt.LogitRules(), **kw)


class _Streams:
    """Torch's streams without a device: which one is current, and which are being recorded."""

    def __init__(self, monkeypatch, recorded):
        self.current, self.recorded, self.waits = 0, recorded, 0
        monkeypatch.setattr(torch.cuda, "device", lambda d: self)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: type("S", (), dict(cuda_stream=handle)))
        monkeypatch.setattr(torch.cuda, "stream", lambda s: type("On", (), dict(__enter__=lambda _: setattr(self, "current", s.cuda_stream),
                                                                                 __exit__=lambda *_: setattr(self, "current", 0)))())
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: self.current in self.recorded)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *_: self)

    def __enter__(self):
        return self

    def __exit__(self, *_):
        return None

    def synchronize(self):
        self.waits += 1


class _Workspaces(rt.DecodeStep):
    def __init__(self):
        self.ctx, self._outgrown, self.device = None, [], torch.device("cpu")
        self.params = orthrus.make_params(batch=2, num_q_heads=4, num_kv_heads=2, head_dim=128, block_k=4, page_size=16, max_pages_per_seq=70000,
                                          max_seq_len=4000, num_pages=200, vocab=V, num_splits=4)
        self._tree_attn_key = self._tree_consensus_key = (None, None)


def test_no_workspace_is_made_while_the_calls_stream_is_recorded(monkeypatch):
    """The stream that a call names, while torch's current one is another."""
    streams, s = _Streams(monkeypatch, {77}), _Workspaces()
    stream = type("S", (), dict(cuda_stream=77))
    for kind in (s._tree_attn_ws, s._tree_consensus_ws):
        for handle in (77, stream):
            with pytest.raises(RuntimeError, match="reserve"):
                kind(9, handle)
        assert not hasattr(s, "tree_attn_ws" if kind == s._tree_attn_ws else "tree_consensus_ws") and streams.waits == 0 and streams.current == 0
        assert kind(9, 78).numel() > 0 and kind(5, stream).numel() > 0   # on another stream, and no larger one while it is recorded
        streams.waits = 0
    streams.recorded = {0}    # torch's own, whatever the call names
    with pytest.raises(RuntimeError, match="reserve"):
        s._tree_attn_ws(40, 78)


def test_workspaces_that_grow_stay_few(monkeypatch):
    """Bounds that a loop raises step by step: what all outgrown buffers hold stays below what the last one does, and none is given up."""
    _Streams(monkeypatch, set())
    s, seen = _Workspaces(), []
    s.params.num_splits = 0
    s.params.num_pages = 100000
    for bound in range(16, 60000, 16):
        s.params.max_seq_len = bound
        need = orthrus.orthrus_tree_attn_workspace_bytes(None, s.params, 33)
        ws = s._tree_attn_ws(33)
        assert ws.numel() >= need
        seen += [] if any(ws is x for x in seen) else [ws]
    assert len(seen) > 2 and all(any(x is y for y in s._outgrown) for x in seen[:-1])
    assert sum(x.numel() for x in s._outgrown) < seen[-1].numel()


@pytest.mark.parametrize("mixed", [False, True])
def test_rows_that_do_not_lie_as_the_steps_strides_say_are_refused(mixed):
    """Dense rows, or those of a narrower projection, in a step whose rows are the parts of a fused one: the last rows would be read behind
    the tensors' memory."""
    row = (8 + 2 + 2) * 128
    s = _Step(q_stride_row=row, q_stride_head=128, blk_stride_row=row, blk_stride_head=128)
    other = dict(k_pool=A) if mixed else {}
    fused, wide = _h(B, N, 12, 128), _h(B, N, 16, 128)
    parts = lambda f: dict(q=f[:, :, :8], k_blk=f[:, :, 8:10], v_blk=f[:, :, 10:12])  # noqa: E731
    flat = lambda f: {k: v.flatten(0, 1) for k, v in parts(f).items()}  # noqa: E731
    for good in (parts(fused), flat(fused)):
        with pytest.raises(_Accepted):
            s.tree_attn(**_attn_args(**good, **other))
    for name in ("q", "k_blk", "v_blk"):
        good = parts(fused)
        heads = good[name].shape[2]
        for bad in (good[name].contiguous(), parts(wide)[name], _h(B, N, 128, heads).transpose(2, 3), _h(B, 2 * N, 12, 128)[:, ::2, :heads],
                    _h(B, N + 1, 12, 128)[:, :N, :heads], _h(B, N, heads, 1).expand(B, N, heads, 128)):
            with pytest.raises(ValueError, match=name):
                s.tree_attn(**_attn_args(**dict(good, **{name: bad}), **other))
    with pytest.raises(_Accepted):   # a single row has none
        _Step(batch=1, blk_stride_row=row, blk_stride_head=128).tree_attn(
            **dict(_attn_args(**other), parents=_i(1, 1), q=_h(1, 1, 8, 128), k_blk=_h(1, 1, 2, 128), v_blk=_h(1, 1, 2, 128), out=_h(1, 1, 8, 128)))


@pytest.mark.parametrize("layer", [0, 9000 * 128])
def test_committed_rows_that_do_not_lie_as_the_steps_strides_say_are_refused(layer):
    row, L = 12 * 128, 2
    s = _Step(num_layers=L, blk_stride_row=row, blk_stride_head=128, blk_stride_layer=layer)
    fused = _h(L, 9000 * 128)[:, :B * N * row].unflatten(1, (B, N, 12, 128)) if layer else _h(L, B, N, 12, 128)
    pools = dict(k_pool=_h(L, 50, 2, 16, 128), v_pool=_h(L, 50, 2, 16, 128))
    good = dict(k_blk_ar=fused[:, :, :, 8:10], v_blk_ar=fused[:, :, :, 10:], **pools)
    with pytest.raises(_Accepted):
        s.tree_consensus_commit(**_committed(**good))
    for name in ("k_blk_ar", "v_blk_ar"):
        for bad in (good[name].contiguous(), _h(L, B, N, 16, 128)[..., 8:10, :], _h(L + 1, B, N, 12, 128)[::2, :, :, :2], _h(L, B + 1, N, 12, 128)[:, :B, :, :2],
                    _h(L, B, N, 2, 128)):
            with pytest.raises(ValueError, match=name):
                s.tree_consensus_commit(**_committed(**dict(good, **{name: bad})))
            with pytest.raises(ValueError, match=name):
                s.tree_consensus_commit(**_committed(**dict(good, k_pool=A, **{name: bad})))


class _Host:
    """Stands for the device that the tensors of these tests are on."""
    index = -1

    def __eq__(self, other):
        return getattr(other, "type", None) == "cpu"

    def __ne__(self, other):
        return not self == other

    def __str__(self):
        return "the host"


class _Calling(_Step):
    """A step whose calls reach a stand-in for the library."""

    def __init__(self, monkeypatch, **kw):
        super().__init__(**kw)
        self.device, self.calls = _Host(), []
        self._tree_attn_known = self._tree_consensus_known = (None, None)
        for name in ("orthrus_tree_attn", "orthrus_tree_consensus_commit"):
            monkeypatch.setattr(rt.B._lib, name, lambda *a: self.calls.append(a) or 0)

    def _stream(self, stream):
        return 0

    def _tree_attn_ws(self, nodes):
        self.ws = torch.zeros(256, dtype=torch.uint8)
        return self.ws

    _tree_consensus_ws = _tree_attn_ws


@pytest.mark.parametrize("pools", [torch.bfloat16, torch.int16])
@pytest.mark.parametrize("fused", [False, True])
def test_a_call_like_the_one_before_is_looked_at_as_closely(monkeypatch, fused, pools):
    """The second call of the same sizes goes another way through the host: with the same arguments for the library, and the same refusals."""
    monkeypatch.setattr(rt, "_raw_stream", lambda index: 0)
    row = 12 * 128 if fused else 0
    s = _Calling(monkeypatch, q_stride_row=row, q_stride_head=row and 128, blk_stride_row=row, blk_stride_head=row and 128)
    f, g = _h(B, N, 12, 128), _h(1, B, N, 12, 128)
    attn = _attn_args(lse=torch.zeros((B, 8, N)), **(dict(q=f[:, :, :8], k_blk=f[:, :, 8:10], v_blk=f[:, :, 10:]) if fused else {}))
    walk = _committed(**(dict(k_blk_ar=g[..., 8:10, :], v_blk_ar=g[..., 10:, :]) if fused else {}))
    for a in (attn, walk):     # caches of bits next to rows of bf16 as well
        a.update(k_pool=a["k_pool"].view(pools), v_pool=a["v_pool"].view(pools))
    odd_rows = [("k_blk", _h(B, N, 16, 128)[:, :, :2]), ("q", _h(B, N, 16, 128)[:, :, :8]), ("v_blk", _h(B, N, 4, 128)[:, :, :2])]
    bad_attn = _ODD_CACHES + odd_rows + [
        ("parents", _i(B, N).long()), ("parents", _i(N, B).t()), ("parents", _i(B - 1, N)), ("q", attn["q"].half()), ("q", attn["q"].float()),
        ("k_blk", _h(B, N, 4, 128)), ("v_blk", attn["v_blk"].half()), ("out", _h(B, N, 8, 256)[..., :128]), ("out", _h(B, N, 8, 128).half()),
        ("lse", torch.zeros((B, 8, N)).double()), ("lse", torch.zeros((B, N, 8)).transpose(1, 2)), ("lse", torch.zeros((B, 4, N))),
        ("k_pool", attn["k_pool"].half()), ("v_pool", attn["v_pool"].float())]
    bad_walk = _ODD_CACHES + [(a + "_ar", t[None]) for a, t in odd_rows if a != "q"] + [
        ("ar_logits", torch.zeros((B, N, V - 1))), ("ar_logits", torch.zeros((B, 8, V))[:, :N]), ("ar_logits", torch.zeros((B, N, V)).double()),
        ("parents", _i(N, B).t()), ("node_tokens", _i(B, N).long()), ("path_nodes", _i(B, 4)), ("out_tokens", _i(N, B).t()), ("accept_len", _i(B - 1)),
        ("next_anchor", torch.zeros(B)), ("num_committed", _i(B, 2)[:, 0]), ("k_blk_ar", walk["k_blk_ar"].half()), ("v_pool", walk["v_pool"].half()),
        ("k_pool", walk["k_pool"].float())]
    for call, good, bad in ((s.tree_attn, attn, bad_attn), (s.tree_consensus_commit, walk, bad_walk)):
        assert not s.calls
        call(**good)
        ws = s.ws
        for _ in range(2):
            call(**good)
            assert s.ws is ws, "the second call looks at everything anew"
        first, *others = [[x if not hasattr(x, "_obj") else bytes(x._obj) for x in c] for c in s.calls]
        assert len(others) == 2 and all(c == first for c in others)
        for name, t in bad:
            with pytest.raises(ValueError):
                call(**dict(good, **{name: t}))
        assert len(s.calls) == 3
        call(**dict(good, k_pool=A))          # an address among them
        assert len(s.calls) == 4
        s.params.max_seq_len = 90             # parameters that changed: looked at anew
        call(**good)
        assert s.ws is not ws
        s.calls.clear()
    s.tree_consensus_commit(**dict(walk, k_blk_ar=None, v_blk_ar=None, k_pool=None, v_pool=None, page_table=None, seq_lens=None))
    s.tree_consensus_commit(**dict(walk, ar_logits=torch.zeros((B, N, V + 3))), logits_stride_row=V + 3)
    assert len(s.calls) == 2
    with pytest.raises(ValueError):
        s.tree_consensus_commit(**walk, logits_stride_row=V + 3)


@pytest.mark.parametrize("ends", [True, False])
def test_a_cycle_that_is_refused_while_it_is_recorded_leaves_no_graph(monkeypatch, ends):
    """Part of a cycle would be replayed as a whole one; the same stack can be captured again."""
    live, n = set(), iter(range(1, 9))

    def end(ctx, stream):
        if not ends:
            raise orthrus.OrthrusError(B_EHIP, "orthrus_graph_end")
        live.add(next(n))
        return max(live)
    B_EHIP = rt.B.ORTHRUS_EHIP
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *_: None)
    monkeypatch.setattr(torch.cuda, "Stream", lambda device=None: object())
    monkeypatch.setattr(rt.B, "orthrus_graph_begin", lambda ctx, stream: None)
    monkeypatch.setattr(rt.B, "orthrus_graph_end", end)
    monkeypatch.setattr(rt.B, "orthrus_graph_destroy", live.discard)
    stack = rt.DecodeStack.__new__(rt.DecodeStack)
    stack.graph, stack.step = None, type("Step", (), dict(device="cuda:0", ctx=None, close=lambda self: None))()

    def refused(stream):
        raise RuntimeError("reserve() comes before a call is recorded")
    stack.cycle = refused
    with pytest.raises(RuntimeError, match="reserve"):
        stack.capture()
    assert stack.graph is None and not live
    with pytest.raises(RuntimeError, match="capture"):
        stack.replay()
    if ends:
        stack.cycle = lambda stream: None
        stack.capture()
        assert stack.graph in live
    stack.close()
    assert not live


def test_an_attention_workspace_that_is_replaced_stays_for_its_graphs(monkeypatch):
    s = _Workspaces()
    monkeypatch.setattr(rt.B, "orthrus_attn_num_splits_on", lambda ctx, p: 4)
    monkeypatch.setattr(rt.B, "orthrus_attn_workspace_bytes_on", lambda ctx, p: 10 * p.max_seq_len)
    s.attn_ws = first = torch.empty(2560, dtype=torch.uint8)
    s.set_max_seq_len(200)
    assert s.attn_ws is first and not s._outgrown
    s.set_max_seq_len(4000)
    assert s.attn_ws.numel() >= 40000 and any(x is first for x in s._outgrown)


@pytest.mark.parametrize("kind,size", [(0, 4), (1, 2)])
def test_logits_and_out_that_share_memory_are_refused(kind, size):
    """Rows are read by some workgroups while others write them.  (A call that is not refused ends in ORTHRUS_EHIP here: no device.)"""
    keep = ctypes.create_string_buffer(1 << 12)
    p, r = orthrus.make_params(batch=B, num_q_heads=1, num_kv_heads=1, head_dim=64, block_k=1, page_size=16, max_pages_per_seq=1, max_seq_len=0,
                               num_pages=1, vocab=V), rt.B.orthrus_logit_rules()
    end, big = (B * N - 1) * V + V, 2 * V + 10

    def call(out_at, stride=0, out_stride=0, base=1 << 30):
        return orthrus.orthrus_logits_process(ctypes.addressof(keep), p, kind, base, stride, N, None, None, r, base + out_at * size, out_stride, 0, check=False)
    for at, stride, out_stride in ((1, 0, 0), (-1, 0, 0), (end - 1, 0, 0), (1 - end, 0, 0), (V, 0, 0), (V - 1, big, big), (1 - V, big, big), (big - V + 1, big, big),
                                   (V + 11, big, big), (3 * big + V - 1, big, big), (V, 2 * V, 3 * V), (5 * V, 2 * V, V), (0, V, V + 1), (-V + 1, 0, big)):
        assert call(at, stride, out_stride) == rt.B.ORTHRUS_EINVAL, (at, stride, out_stride)
    if torch.cuda.is_available():
        return    # what is not refused would be launched
    for at, stride, out_stride in ((0, 0, 0), (0, V, V), (end, 0, 0), (-end, 0, 0), (V, big, big), (V + 10, big, big), (-V, big, big), (3 * big + V, big, big),
                                   (V, 2 * V, 4 * V), (V * 2 * B * N, 2 * V, 3 * V), (-3 * V * B * N, 2 * V, 3 * V)):
        assert call(at, stride, out_stride) == rt.B.ORTHRUS_EHIP, (at, stride, out_stride)


@pytest.mark.parametrize("layers,row", [(1, 0), (2, 0), (2, 12 * 128)])
def test_a_batch_of_nobody_is_taken(layers, row):
    s = _Step(batch=0, num_layers=layers, blk_stride_row=row, blk_stride_head=row and 128)
    walk = dict(ar_logits=torch.zeros((0, N, V)), parents=_i(0, N), node_tokens=_i(0, N), k_blk_ar=_h(layers, 0, N, 2, 128), v_blk_ar=_h(layers, 0, N, 2, 128),
                k_pool=_h(layers, 50, 2, 16, 128), v_pool=_h(layers, 50, 2, 16, 128), page_table=_i(0, 9), seq_lens=_i(0), accept_len=_i(0),
                num_committed=_i(0), path_nodes=_i(0, N), out_tokens=_i(0, N), next_anchor=_i(0))
    for call in (lambda: s.tree_consensus_commit(**walk), lambda: s.process_logits(torch.zeros((0, N, V)), rt.LogitRules()),
                 lambda: s.tree_attn(**_attn_args(parents=_i(0, N), q=_h(0, N, 8, 128), k_blk=_h(0, N, 2, 128), v_blk=_h(0, N, 2, 128), out=_h(0, N, 8, 128),
                                                  page_table=_i(0, 9), seq_lens=_i(0)))):
        with pytest.raises(_Accepted):
            call()
