"""CPU-only checks of the C-ABI library: it loads, exports every declared symbol, and its host-side
argument validation answers without touching a GPU (no compute call is made here)."""
import ctypes
import os
import re

import pytest

import paper_2605_12825_amd as orthrus
from paper_2605_12825_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _declared_functions():
    text = open(os.path.join(ROOT, "include", "orthrus.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(orthrus_[a-z_]+)\s*\(", text)))


def test_library_exports_every_declared_symbol():
    lib = ctypes.CDLL(orthrus.library_path())
    names = _declared_functions()
    assert len(names) >= 9
    for n in names:
        assert hasattr(lib, n), n
    assert sorted(B.EXPORTED) == names


def test_binding_struct_matches_header_field_order():
    text = open(os.path.join(ROOT, "include", "orthrus.h")).read()
    body = text[text.index("typedef struct {"):text.index("} orthrus_params;")]
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = re.findall(r"\b(?:int32_t|int64_t|float)\s+([a-z_]+)\s*;", body)
    assert fields == [f[0] for f in B.orthrus_params._fields_]


def _good():
    return orthrus.make_params(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, block_k=16, page_size=16,
                               max_pages_per_seq=70, max_seq_len=1000, num_pages=200, vocab=1000)


def test_status_strings():
    for code in (0, -1, -2, -3, -4, -5, 7):
        assert isinstance(orthrus.orthrus_status_string(code), str) and orthrus.orthrus_status_string(code)


def test_workspace_queries_and_split_planning():
    p = _good()
    assert orthrus.orthrus_attn_num_splits(p) >= 1
    assert orthrus.orthrus_attn_workspace_bytes(p) >= 0
    assert orthrus.orthrus_consensus_workspace_bytes(p) > 0
    p.num_splits = 1
    assert orthrus.orthrus_attn_num_splits(p) == 1 and orthrus.orthrus_attn_workspace_bytes(p) == 0
    p.num_splits = 4
    n = orthrus.orthrus_attn_num_splits(p)
    assert 1 <= n <= 4
    # partials: units * splits * padded rows * (d + 2) floats, padded to 256 bytes
    assert orthrus.orthrus_attn_workspace_bytes(p) >= 2 * 2 * n * 64 * (128 + 2) * 4


def _params_for(w, max_seq_len):
    pages = (max_seq_len + w.page_size - 1) // w.page_size + 1
    return B.make_params(batch=w.batch, num_q_heads=w.num_q_heads, num_kv_heads=w.num_kv_heads, head_dim=w.head_dim,
                         block_k=w.block_k, page_size=w.page_size, max_pages_per_seq=pages, max_seq_len=max_seq_len,
                         num_pages=pages * max(w.batch, 1), vocab=max(w.vocab, 1))


def test_split_planning_aims_at_one_workgroup_per_cu():
    """Host logic only: the cost model's choices for the workloads of the build contract (256 CUs)."""
    from orthrus_inputs import WORKLOADS
    got = {}
    for name, L in (("long", 32768), ("stress", 2048 + 512), ("layer8b", 4096), ("mixed", 8192), ("tiny", 128)):
        got[name] = orthrus.orthrus_attn_num_splits(_params_for(WORKLOADS[name], L))
    assert got["long"] == 8            # 4 x 8 (sequence, head) units x 8 splits = 256 workgroups
    assert got["stress"] == 1          # 512 units already: no split, no combine
    assert got["mixed"] == 4           # 64 units x 4
    # 8 units, chip far from full: a workgroup's time is its chain of tiles (~0.56 us each), a split costs
    # ~0.25 us in partials, dispatch and merge; 16 splits of 8 tiles measured fastest (13.2 us per call
    # against 14.2 at 26 and 15.9 at 8)
    assert 12 <= got["layer8b"] <= 22
    assert got["tiny"] == 1
    # the same sequence alone at other lengths: more tiles, more splits, never more than one workgroup per CU
    w = WORKLOADS["layer8b"]
    by_len = [orthrus.orthrus_attn_num_splits(_params_for(w, L)) for L in (256, 1024, 4096, 16384, 32768)]
    assert by_len == sorted(by_len) and by_len[0] == 1 and by_len[-1] * w.num_kv_heads <= 256
    # a half-full chip takes the split count that fills it
    import dataclasses
    w4 = dataclasses.replace(w, batch=4)
    assert orthrus.orthrus_attn_num_splits(_params_for(w4, 4096)) == 8
    # the 64 splits the long configuration names are honoured when asked for
    p = _params_for(WORKLOADS["long"], 32768)
    p.num_splits = 64
    assert orthrus.orthrus_attn_num_splits(p) == 64
    rows, d = 64, 128
    assert orthrus.orthrus_attn_workspace_bytes(p) >= 4 * 8 * 64 * rows * (d + 2) * 4


def test_balanced_partition_plan_on_the_host():
    """num_splits = -1: no fixed split count, workspace = two partials per resident workgroup, whatever the lengths."""
    from orthrus_inputs import WORKLOADS
    p = _params_for(WORKLOADS["mixed"], 8192)
    p.num_splits = -1
    assert orthrus.orthrus_attn_num_splits(p) == 0
    rows, d, wgs = 7 * 32, 128, 256              # R = 224 rows in 7 blocks: 8 waves, one workgroup per CU
    want = 2 * wgs * rows * (d + 2) * 4
    assert want <= orthrus.orthrus_attn_workspace_bytes(p) <= want + 512
    p.max_seq_len = 512
    assert want <= orthrus.orthrus_attn_workspace_bytes(p) <= want + 512
    p.num_splits = -2
    with pytest.raises(orthrus.OrthrusError):
        orthrus.orthrus_attn_num_splits(p)


@pytest.mark.parametrize("batch,K,vocab,greedy,sampling", [(1, 16, 128256, 2304, 4608), (8, 32, 151936, 39168, 80640),
                                                          (3, 5, 2049, 768, 768), (2, 4, 1, 768, 768)])
def test_consensus_workspaces_do_not_grow(batch, K, vocab, greedy, sampling):
    """Programs keep these buffers: one entry per (row, 8192-element chunk), one per (sequence, chunk) for the draw and two
    words per sequence, each padded to 256 bytes."""
    p = _good()
    p.batch, p.block_k, p.vocab = batch, K, vocab
    assert orthrus.orthrus_consensus_workspace_bytes(p) == greedy
    assert orthrus.orthrus_sampling_workspace_bytes(p) == sampling


@pytest.mark.parametrize("batch,K,vocab,sample,filtered", [
    (1, 1, 1, 0, 768), (3, 4, 1792, 0, 1280), (3, 4, 1793, 13056, 26880), (1, 16, 128256, 1056768, 2114816),
    (64, 16, 151936, 80490752, 161076480), (2, 3, 1 << 20, 3226112, 6458880), (0, 1, 5000, 256, 256)])
def test_filter_workspaces_do_not_grow(batch, K, vocab, sample, filtered):
    """As many bytes as these: per row (consensus: and view) and 2048 logits 24 bytes and a list of 128 pairs, a number per row; nothing
    of these up to 1792 logits.  The consensus adds 32 bytes per row and view, two words per sequence, 24 bytes per sequence
    and 8192 logits.  Each part padded to 256 bytes."""
    p = _good()
    p.batch, p.block_k, p.vocab = batch, K, vocab
    up = lambda n: (n + 255) // 256 * 256  # noqa: E731
    rows, chunks = batch * K, (vocab + 7 + 2047) // 2048

    def plan(n):
        return up(n * chunks * 24) + up(n * chunks * 1024) + up((n + 1) * 4) if vocab > 1792 else 0
    assert orthrus.orthrus_sample_workspace_bytes(p) == plan(rows) == sample
    whole = up(2 * rows * 32) + up(batch * 8) + up(batch * ((vocab + 8191) // 8192) * 24) + plan(2 * rows)
    assert orthrus.orthrus_filtered_workspace_bytes(p) == whole == filtered


@pytest.mark.parametrize("batch,want", [(0, 256), (1, 256), (20, 256), (21, 512), (4096, 49408)])
def test_page_table_workspace_does_not_grow(batch, want):
    """Three words per sequence, two for the ring."""
    p = _good()
    p.batch = batch
    assert orthrus.orthrus_page_tables_workspace_bytes(p) == ((3 * batch + 2) * 4 + 255) // 256 * 256 == want


@pytest.mark.parametrize("batch,q_heads,kv_heads,d,K,max_seq_len,splits,workspace", [
    (1, 32, 8, 128, 16, 4112, 13, 3461120), (1, 32, 8, 128, 16, 8000, 21, 5591040), (1, 32, 8, 128, 1, 2000, 11, 1464320),
    (1, 32, 8, 128, 32, 40000, 30, 15974400), (4, 32, 8, 128, 16, 32768, 8, 8519680), (4, 32, 8, 128, 8, 1000, 4, 2129920),
    (1, 28, 4, 128, 8, 12000, 27, 3594240), (1, 8, 8, 128, 4, 6000, 19, 2529280), (1, 4, 2, 64, 16, 400, 1, 0),
    (4, 4, 2, 64, 16, 32768, 47, 3176448), (8, 16, 2, 64, 32, 2000, 9, 9732096), (64, 32, 8, 128, 16, 3071, 1, 0),
])
def test_attention_split_plan_stays(batch, q_heads, kv_heads, d, K, max_seq_len, splits, workspace):
    """Programs keep these buffers too, and another split count gives other bits."""
    pages = (max_seq_len + 15) // 16
    p = orthrus.make_params(batch=batch, num_q_heads=q_heads, num_kv_heads=kv_heads, head_dim=d, block_k=K, page_size=16,
                            max_pages_per_seq=pages, max_seq_len=max_seq_len, num_pages=batch * pages)
    assert (orthrus.orthrus_attn_num_splits(p), orthrus.orthrus_attn_workspace_bytes(p)) == (splits, workspace)


def test_prefill_workspace_and_argument_checks_on_the_host():
    p = _good()
    assert orthrus.orthrus_prefill_workspace_bytes(p, 4096) >= 2 * 4 * p.batch
    with pytest.raises(B.OrthrusError):
        orthrus.orthrus_prefill_workspace_bytes(p, -1)
    lib = ctypes.CDLL(orthrus.library_path())
    lib.orthrus_prefill_attn.restype = ctypes.c_int
    # null context is refused before anything else is looked at
    assert lib.orthrus_prefill_attn(None, ctypes.byref(p), 16, None, None, None, None, None, None, None, None, None,
                                    None, ctypes.c_size_t(0), None) == B.ORTHRUS_EINVAL
    assert lib.orthrus_graph_begin(None, None) == B.ORTHRUS_EINVAL
    assert lib.orthrus_graph_launch(None, None) == B.ORTHRUS_EINVAL
    assert lib.orthrus_graph_destroy(None) == B.ORTHRUS_EINVAL
    assert lib.orthrus_attn_timing(None, 1) == B.ORTHRUS_EINVAL


@pytest.mark.parametrize("field,value,status", [
    ("batch", -1, B.ORTHRUS_EINVAL),
    ("num_q_heads", 7, B.ORTHRUS_EINVAL),          # not a multiple of num_kv_heads
    ("head_dim", 96, B.ORTHRUS_EUNSUPPORTED),
    ("page_size", 8, B.ORTHRUS_EUNSUPPORTED),
    ("page_size", 24, B.ORTHRUS_EUNSUPPORTED),
    ("block_k", 33, B.ORTHRUS_EUNSUPPORTED),
    ("block_k", 0, B.ORTHRUS_EINVAL),
    ("max_seq_len", 70 * 16 + 1, B.ORTHRUS_EINVAL),  # longer than the page table can map
    ("sm_scale", 0.0, B.ORTHRUS_EINVAL),
    ("pool_stride_tok", 100, B.ORTHRUS_EUNSUPPORTED),
    ("num_pages", 0, B.ORTHRUS_EINVAL),
])
def test_bad_params_are_rejected_on_the_host(field, value, status):
    p = _good()
    setattr(p, field, value)
    with pytest.raises(orthrus.OrthrusError) as e:
        orthrus.orthrus_attn_workspace_bytes(p)
    assert e.value.status == status


def test_group_times_block_limit():
    p = orthrus.make_params(batch=1, num_q_heads=64, num_kv_heads=2, head_dim=128, block_k=16, page_size=16,
                            max_pages_per_seq=8, max_seq_len=100, num_pages=8)
    with pytest.raises(orthrus.OrthrusError) as e:
        orthrus.orthrus_attn_num_splits(p)          # 32 * 16 = 512 rows > 256
    assert e.value.status == B.ORTHRUS_EUNSUPPORTED


def test_compute_entry_points_reject_null_context_before_any_launch():
    p = _good()
    lib = B._lib
    st = lib.orthrus_dual_view_attn(None, ctypes.byref(p), 0, None, None, None, None, None, None, None, None, None,
                                    None, 0, None)
    assert st == B.ORTHRUS_EINVAL
    st = lib.orthrus_consensus_commit(None, ctypes.byref(p), None, None, None, None, None, None, None, None, None,
                                      None, None, None, None, 0, None)
    assert st == B.ORTHRUS_EINVAL
    code = ctypes.c_int32(0)
    assert lib.orthrus_last_device_error(None, None, ctypes.byref(code)) == B.ORTHRUS_EINVAL
    assert lib.orthrus_destroy(None) == B.ORTHRUS_EINVAL


class _Device:
    """Stands for a tensor: counts how often its address is asked for."""
    nbytes = 64

    def __init__(self):
        self.asked = 0

    def data_ptr(self):
        self.asked += 1
        return 4096


@pytest.mark.parametrize("call,operands,before", [
    (orthrus.orthrus_dual_view_attn, 8, (0,)), (orthrus.orthrus_consensus_commit, 12, ()),
    (orthrus.orthrus_sampling_consensus_commit, 15, (1.0,)),
])
@pytest.mark.parametrize("plain", [4096, None])
def test_a_call_takes_each_operand_once_whatever_mix_of_tensors_and_addresses(call, operands, before, plain):
    for at in range(operands):
        args = [_Device() for _ in range(operands)]
        args[at] = plain
        ws = _Device()
        assert call(None, _good(), *before, *args, workspace=ws, stream=0, check=False) == B.ORTHRUS_EINVAL   # no context
        assert [x.asked for x in args if x is not plain] == [1] * (operands - 1) and ws.asked == 1
    args, ws = [_Device() for _ in range(operands)], object()   # an operand that is neither: its error, raised once
    with pytest.raises(AttributeError):
        call(None, _good(), *before, *args, workspace=ws, stream=0, check=False)
    assert [x.asked for x in args] == [1] * operands
