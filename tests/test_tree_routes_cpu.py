"""Which form of a kernel a tree call goes to (host logic only, for 256 CUs): the GPU tests of a form assert by the same functions that they
reach it."""
import ctypes

import pytest

import paper_2605_12825_amd as orthrus

_lib = ctypes.CDLL(orthrus.library_path())
_walks = getattr(_lib, "_ZN7orthrus10tree_walksEiiiii")
_walks.restype, _walks.argtypes = ctypes.c_int, [ctypes.c_int] * 5
_chunk = getattr(_lib, "_ZN7orthrus10tree_chunkEiiiii")
_chunk.restype, _chunk.argtypes = ctypes.c_int, [ctypes.c_int] * 5
_plan = getattr(_lib, "_ZN7orthrus14plan_tree_attnEiiiiiiiiidPNS_8AttnPlanEPi")
_TYPE = {"f32": 0, "bf16": 1, "f16": 2}


class AttnPlan(ctypes.Structure):
    """Mirror of orthrus_internal.h's."""
    _fields_ = [("rows", ctypes.c_int), ("wide", ctypes.c_bool)] + [(n, ctypes.c_int) for n in ("waves", "rows_padded", "chunk_tokens", "num_splits",
                "bal_wgs", "merge_waves", "by_size", "kv_nt")] + [(n, ctypes.c_size_t) for n in ("lds_bytes", "part_o_bytes", "part_ml_bytes")]


_plan.restype, _plan.argtypes = ctypes.c_int, [ctypes.c_int] * 9 + [ctypes.c_double, ctypes.POINTER(AttnPlan), ctypes.POINTER(ctypes.c_int)]


def consensus_form(B, N, V, max_path=None, kind="f32"):
    """("walk" or "scan", logits of a workgroup)."""
    walk = _walks(B, N, max_path or N, V, _TYPE[kind])
    return "walk" if walk else "scan", _chunk(walk, B, N, V, _TYPE[kind])


def attn_form(Hq, H, d, N, B, max_seq_len, splits=0, layers=1, pool_tokens=1 << 40):
    """(64-row kernel, compute waves, order: "balanced", "by size" or "plain", non-temporal loads, row groups, pieces)."""
    p, groups = AttnPlan(), ctypes.c_int()
    assert _plan(d, Hq // H, N, B, H, max_seq_len, splits, 256, layers, float(pool_tokens), ctypes.byref(p), ctypes.byref(groups)) == 0
    return p.wide, p.waves, "balanced" if p.bal_wgs else "by size" if p.by_size else "plain", p.kv_nt, groups.value, p.num_splits


@pytest.mark.parametrize("form,B,N,V,max_path,kind", [
    (("scan", 2048), 1, 32, 151936, 8, "f32"), (("scan", 2048), 4, 16, 151936, 8, "f32"), (("scan", 2048), 4, 64, 100000, None, "bf16"),
    (("scan", 8192), 16, 16, 151936, 8, "f32"), (("scan", 4096), 8, 48, 151669, 6, "bf16"), (("walk", 2048), 8, 64, 151936, 8, "f32"),
    (("walk", 2048), 16, 32, 151936, 5, "f32"), (("walk", 8192), 64, 64, 151936, 8, "f32"), (("walk", 8192), 64, 64, 151936, 8, "f16"),
    (("scan", 8192), 64, 64, 151936, None, "f32"), (("scan", 8192), 64, 64, 151936, 64, "f32"), (("scan", 4096), 64, 64, 151936, 1000, "f16"),
    (("scan", 2048), 1, 1, 1, 1, "f32"),
])
def test_consensus_form(form, B, N, V, max_path, kind):
    assert consensus_form(B, N, V, max_path, kind) == form


@pytest.mark.parametrize("form,args", [
    # 32/8 and 28/4 heads, trees of few and of many nodes
    ((False, 1, "plain", 0, 1, 16), (32, 8, 128, 8, 1, 4096)), ((True, 4, "by size", 1, 1, 1), (32, 8, 128, 64, 64, 2500)),
    ((False, 7, "balanced", 0, 1, 1), (28, 4, 128, 32, 16, 8192, -1)), ((False, 4, "balanced", 0, 2, 1), (32, 8, 128, 64, 16, 8192, -1)),
    ((False, 6, "balanced", 0, 3, 1), (64, 8, 128, 64, 16, 8192, -1)), ((False, 8, "plain", 0, 2, 1), (64, 8, 128, 64, 1, 200)),
])
def test_attention_form(form, args):
    assert attn_form(*args) == form
