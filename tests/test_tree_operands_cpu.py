"""What the tree and rule calls of a DecodeStep make of operands that do not lie as the call would read them: refused on the host, before
anything touches a device."""
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
