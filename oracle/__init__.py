"""ctypes front end of the CPU oracle (test infrastructure only).

Only tests, the smoke check and the benchmark's CPU-baseline leg import this package.  It
compiles ``orthrus_oracle.c`` with gcc on first use (plain -O2, no fast-math, OpenMP over
independent outputs) and exposes the two oracle entry points on numpy arrays.  It imports
nothing from the GPU package.
"""
from __future__ import annotations

import ctypes
import os
import subprocess
from typing import Dict, Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_SRC = os.path.join(_HERE, "orthrus_oracle.c")
_LIB = os.path.join(_HERE, "liborthrus_oracle.so")
# sanitizer builds (CPU test suite): the same source under AddressSanitizer + UndefinedBehaviorSanitizer as a
# library (selected with ORTHRUS_ORACLE_SANITIZE=1; load it with ASAN_OPTIONS=verify_asan_link_order=0) and
# as a self-contained driver executable (sanitize_selftest.c)
_LIB_SAN = os.path.join(_HERE, "liborthrus_oracle_asan.so")
_SELFTEST_SRC = os.path.join(_HERE, "sanitize_selftest.c")
_SELFTEST = os.path.join(_HERE, "sanitize_selftest")
_SAN_FLAGS = ["-O1", "-g", "-std=c11", "-fopenmp", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
              "-fno-omit-frame-pointer", "-Wall", "-Wextra"]

VIEW_DIFFUSION = 0
VIEW_AR_VERIFY = 1

_lib = None


def build(force: bool = False) -> str:
    """Compile the oracle's C source into a shared library next to it."""
    if force or not os.path.exists(_LIB) or os.path.getmtime(_LIB) < os.path.getmtime(_SRC):
        tmp = _LIB + ".tmp.%d" % os.getpid()
        cmd = ["gcc", "-O2", "-std=c11", "-fPIC", "-shared", "-fopenmp", "-Wall", "-Wextra",
               "-o", tmp, _SRC, "-lm"]
        subprocess.run(cmd, check=True)
        os.replace(tmp, _LIB)
    return _LIB


def build_sanitized() -> str:
    """The oracle as a shared library under ASan + UBSan (gcc's shared sanitizer runtimes)."""
    tmp = _LIB_SAN + ".tmp.%d" % os.getpid()
    subprocess.run(["gcc"] + _SAN_FLAGS + ["-fPIC", "-shared", "-o", tmp, _SRC, "-lm"], check=True)
    os.replace(tmp, _LIB_SAN)
    return _LIB_SAN


def build_selftest() -> str:
    """The sanitizer driver executable: oracle + sanitize_selftest.c under ASan + UBSan."""
    tmp = _SELFTEST + ".tmp.%d" % os.getpid()
    subprocess.run(["gcc"] + _SAN_FLAGS + ["-o", tmp, _SRC, _SELFTEST_SRC, "-lm"], check=True)
    os.replace(tmp, _SELFTEST)
    return _SELFTEST


def _load():
    global _lib
    if _lib is None:
        lib = ctypes.CDLL(build_sanitized() if os.environ.get("ORTHRUS_ORACLE_SANITIZE") == "1" else build())
        i32, i64, f64 = ctypes.c_int, ctypes.c_int64, ctypes.c_double
        p = ctypes.c_void_p
        lib.orthrus_oracle_num_threads.restype = ctypes.c_int
        lib.orthrus_oracle_dual_view_attn.restype = ctypes.c_int
        lib.orthrus_oracle_dual_view_attn.argtypes = [
            i32, i32, i32, i32, i32, i32, i32, i64, i32, f64,
            p, p, p, p, p, i64, i64, i64, p, p, p, p]
        lib.orthrus_oracle_consensus_commit.restype = ctypes.c_int
        lib.orthrus_oracle_consensus_commit.argtypes = [
            i32, i32, i32, i32, i32, i32, i32, i32, i64,
            p, p, p, p, p, p, i64, i64, i64, i64, p, p, p, p, p, p]
        lib.orthrus_oracle_sampling_consensus_commit.restype = ctypes.c_int
        lib.orthrus_oracle_sampling_consensus_commit.argtypes = [
            i32, i32, i32, f64, i32, i32, i32, i32, i32, i64,
            p, p, p, p, p, p, p, p, p, i64, i64, i64, i64, p, p, p, p, p, p, p, p]
        lib.orthrus_oracle_prefill_attn.restype = ctypes.c_int
        lib.orthrus_oracle_prefill_attn.argtypes = [
            i32, i32, i32, i32, i32, i32, i32, i64, f64,
            p, p, p, p, p, p, i64, i64, i64, p, p, p]
        _lib = lib
    return _lib


def num_threads() -> int:
    return int(_load().orthrus_oracle_num_threads())


def _ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


def _check(a: np.ndarray, dtype, name: str) -> np.ndarray:
    if a.dtype != dtype or not a.flags["C_CONTIGUOUS"]:
        raise TypeError("%s must be a C-contiguous %s array" % (name, np.dtype(dtype).name))
    return a


def _pool_strides(pool: np.ndarray):
    """Element strides (page, head, token) of a [pages, H_kv, P, d] pool."""
    if pool.ndim != 4:
        raise ValueError("pool must be [pages, H_kv, P, d]")
    es = pool.itemsize
    return pool.strides[0] // es, pool.strides[1] // es, pool.strides[2] // es


def dual_view_attn(view: int, sm_scale: float, q: np.ndarray, k_blk: np.ndarray, v_blk: np.ndarray,
                   k_pool: np.ndarray, v_pool: np.ndarray, page_table: np.ndarray,
                   seq_lens: np.ndarray, want_lse: bool = False):
    """Eq. 4 of the paper on bf16-bit inputs; returns fp64 ``out[B,K,H_q,d]`` (and ``lse[B,H_q,K]``)."""
    lib = _load()
    B, K, Hq, d = q.shape
    Hkv = k_blk.shape[2]
    _check(q, np.uint16, "q"); _check(k_blk, np.uint16, "k_blk"); _check(v_blk, np.uint16, "v_blk")
    _check(k_pool, np.uint16, "k_pool"); _check(v_pool, np.uint16, "v_pool")
    _check(page_table, np.int32, "page_table"); _check(seq_lens, np.int32, "seq_lens")
    if k_blk.shape != (B, K, Hkv, d) or v_blk.shape != k_blk.shape:
        raise ValueError("block K/V shape mismatch")
    if k_pool.shape != v_pool.shape or k_pool.shape[1] != Hkv or k_pool.shape[3] != d:
        raise ValueError("pool shape mismatch")
    sp, sh, st = _pool_strides(k_pool)
    out = np.empty((B, K, Hq, d), dtype=np.float64)
    lse = np.empty((B, Hq, K), dtype=np.float64) if want_lse else None
    rc = lib.orthrus_oracle_dual_view_attn(
        B, Hq, Hkv, d, K, k_pool.shape[2], page_table.shape[1], k_pool.shape[0], int(view),
        float(sm_scale), _ptr(q), _ptr(k_blk), _ptr(v_blk), _ptr(k_pool), _ptr(v_pool),
        sp, sh, st, _ptr(page_table), _ptr(seq_lens), _ptr(out), _ptr(lse))
    if rc != 0:
        raise RuntimeError("orthrus_oracle_dual_view_attn failed with status %d" % rc)
    return (out, lse) if want_lse else out


def prefill_attn(sm_scale: float, q: np.ndarray, k_new: np.ndarray, v_new: np.ndarray, new_lens: np.ndarray,
                 k_pool: np.ndarray, v_pool: np.ndarray, page_table: np.ndarray, seq_lens: np.ndarray,
                 allow_capacity_error: bool = False):
    """AR prefill of one layer: appends the new tokens' K/V, causal attention of each over the cache.

    ``q`` is ``[B,T,H_q,d]``, ``k_new``/``v_new`` ``[B,T,H_kv,d]`` (bf16 bits), ``new_lens[b] <= T``;
    pools and ``seq_lens`` are updated in place.  Returns fp64 ``out[B,T,H_q,d]`` (rows past
    ``new_lens[b]`` are NaN) and the status (0, or -4 when allowed).
    """
    lib = _load()
    B, T, Hq, d = q.shape
    Hkv = k_new.shape[2]
    for a, n in ((q, "q"), (k_new, "k_new"), (v_new, "v_new"), (k_pool, "k_pool"), (v_pool, "v_pool")):
        _check(a, np.uint16, n)
    _check(page_table, np.int32, "page_table"); _check(seq_lens, np.int32, "seq_lens")
    _check(new_lens, np.int32, "new_lens")
    if k_new.shape != (B, T, Hkv, d) or v_new.shape != k_new.shape:
        raise ValueError("new K/V shape mismatch")
    if k_pool.shape != v_pool.shape or k_pool.shape[1] != Hkv or k_pool.shape[3] != d:
        raise ValueError("pool shape mismatch")
    sp, sh, st = _pool_strides(k_pool)
    out = np.full((B, T, Hq, d), np.nan, dtype=np.float64)
    rc = lib.orthrus_oracle_prefill_attn(
        B, T, Hq, Hkv, d, k_pool.shape[2], page_table.shape[1], k_pool.shape[0], float(sm_scale),
        _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(new_lens), _ptr(k_pool), _ptr(v_pool), sp, sh, st,
        _ptr(page_table), _ptr(seq_lens), _ptr(out))
    if rc != 0 and not (rc == -4 and allow_capacity_error):
        raise RuntimeError("orthrus_oracle_prefill_attn failed with status %d" % rc)
    return out, rc


def consensus_commit(ar_logits: np.ndarray, draft_tokens: np.ndarray,
                     k_blk_ar: Optional[np.ndarray] = None, v_blk_ar: Optional[np.ndarray] = None,
                     k_pool: Optional[np.ndarray] = None, v_pool: Optional[np.ndarray] = None,
                     page_table: Optional[np.ndarray] = None, seq_lens: Optional[np.ndarray] = None,
                     allow_capacity_error: bool = False) -> Dict[str, np.ndarray]:
    """Eq. 8 consensus plus in-place commit.

    ``k_blk_ar``/``v_blk_ar`` are ``[layers,B,K,H_kv,d]`` (or ``[B,K,H_kv,d]`` for one layer);
    pools are ``[layers,pages,H_kv,P,d]`` or ``[pages,H_kv,P,d]``; both pools and ``seq_lens``
    are updated in place.  With the K/V arguments omitted only the consensus outputs are made.
    """
    lib = _load()
    B, K, V = ar_logits.shape
    _check(ar_logits, np.float32, "ar_logits"); _check(draft_tokens, np.int32, "draft_tokens")
    accept_len = np.empty(B, np.int32); num_committed = np.empty(B, np.int32)
    out_tokens = np.empty((B, K), np.int32); next_anchor = np.empty(B, np.int32)
    if k_blk_ar is None:
        rc = lib.orthrus_oracle_consensus_commit(
            B, K, V, 0, 0, 0, 0, 0, 0, _ptr(ar_logits), _ptr(draft_tokens), None, None, None, None,
            0, 0, 0, 0, None, None, _ptr(accept_len), _ptr(num_committed), _ptr(out_tokens),
            _ptr(next_anchor))
    else:
        kb = k_blk_ar if k_blk_ar.ndim == 5 else k_blk_ar[None]
        vb = v_blk_ar if v_blk_ar.ndim == 5 else v_blk_ar[None]
        kp = k_pool if k_pool.ndim == 5 else k_pool[None]
        vp = v_pool if v_pool.ndim == 5 else v_pool[None]
        for a, n in ((kb, "k_blk_ar"), (vb, "v_blk_ar"), (kp, "k_pool"), (vp, "v_pool")):
            _check(a, np.uint16, n)
        _check(page_table, np.int32, "page_table"); _check(seq_lens, np.int32, "seq_lens")
        layers, _, _, Hkv, d = kb.shape
        if kb.shape != (layers, B, K, Hkv, d) or vb.shape != kb.shape:
            raise ValueError("block K/V shape mismatch")
        if kp.shape != vp.shape or kp.shape[0] != layers or kp.shape[2] != Hkv or kp.shape[4] != d:
            raise ValueError("pool shape mismatch")
        es = kp.itemsize
        sl, sp, sh, st = (kp.strides[0] // es, kp.strides[1] // es, kp.strides[2] // es,
                          kp.strides[3] // es)
        rc = lib.orthrus_oracle_consensus_commit(
            B, K, V, layers, Hkv, d, kp.shape[3], page_table.shape[1], kp.shape[1],
            _ptr(ar_logits), _ptr(draft_tokens), _ptr(kb), _ptr(vb), _ptr(kp), _ptr(vp),
            sl, sp, sh, st, _ptr(page_table), _ptr(seq_lens), _ptr(accept_len),
            _ptr(num_committed), _ptr(out_tokens), _ptr(next_anchor))
    if rc != 0 and not (rc == -4 and allow_capacity_error):
        raise RuntimeError("orthrus_oracle_consensus_commit failed with status %d" % rc)
    return dict(accept_len=accept_len, num_committed=num_committed, out_tokens=out_tokens,
                next_anchor=next_anchor, status=rc)


def sampling_consensus_commit(ar_logits: np.ndarray, diff_logits: np.ndarray, draft_tokens: np.ndarray,
                              accept_u: np.ndarray, gumbel: np.ndarray, temperature: float,
                              k_blk_ar: Optional[np.ndarray] = None, v_blk_ar: Optional[np.ndarray] = None,
                              k_pool: Optional[np.ndarray] = None, v_pool: Optional[np.ndarray] = None,
                              page_table: Optional[np.ndarray] = None, seq_lens: Optional[np.ndarray] = None,
                              allow_capacity_error: bool = False) -> Dict[str, np.ndarray]:
    """Temperature > 0 consensus (speculative-sampling accept/replace rule) plus in-place commit.

    Shapes as in ``consensus_commit``; ``diff_logits`` like ``ar_logits``; ``accept_u`` is ``[B,K]``
    fp32 in [0,1), ``gumbel`` is ``[B,V]`` fp32 standard Gumbel noise.  Also returns the decision
    margins the oracle reports (``margin_accept [B,K]``, ``margin_draw [B]``).
    """
    lib = _load()
    B, K, V = ar_logits.shape
    for a, n in ((ar_logits, "ar_logits"), (diff_logits, "diff_logits"), (accept_u, "accept_u"), (gumbel, "gumbel")):
        _check(a, np.float32, n)
    _check(draft_tokens, np.int32, "draft_tokens")
    if diff_logits.shape != (B, K, V) or accept_u.shape != (B, K) or gumbel.shape != (B, V):
        raise ValueError("sampling input shape mismatch")
    accept_len = np.empty(B, np.int32); num_committed = np.empty(B, np.int32)
    out_tokens = np.empty((B, K), np.int32); next_anchor = np.empty(B, np.int32)
    m_acc = np.empty((B, K), np.float64); m_draw = np.empty(B, np.float64)
    if k_blk_ar is None:
        rc = lib.orthrus_oracle_sampling_consensus_commit(
            B, K, V, float(temperature), 0, 0, 0, 0, 0, 0, _ptr(ar_logits), _ptr(diff_logits),
            _ptr(draft_tokens), _ptr(accept_u), _ptr(gumbel), None, None, None, None, 0, 0, 0, 0, None, None,
            _ptr(accept_len), _ptr(num_committed), _ptr(out_tokens), _ptr(next_anchor), _ptr(m_acc), _ptr(m_draw))
    else:
        kb = k_blk_ar if k_blk_ar.ndim == 5 else k_blk_ar[None]
        vb = v_blk_ar if v_blk_ar.ndim == 5 else v_blk_ar[None]
        kp = k_pool if k_pool.ndim == 5 else k_pool[None]
        vp = v_pool if v_pool.ndim == 5 else v_pool[None]
        for a, n in ((kb, "k_blk_ar"), (vb, "v_blk_ar"), (kp, "k_pool"), (vp, "v_pool")):
            _check(a, np.uint16, n)
        _check(page_table, np.int32, "page_table"); _check(seq_lens, np.int32, "seq_lens")
        layers, _, _, Hkv, d = kb.shape
        es = kp.itemsize
        sl, sp, sh, st = (kp.strides[0] // es, kp.strides[1] // es, kp.strides[2] // es, kp.strides[3] // es)
        rc = lib.orthrus_oracle_sampling_consensus_commit(
            B, K, V, float(temperature), layers, Hkv, d, kp.shape[3], page_table.shape[1], kp.shape[1],
            _ptr(ar_logits), _ptr(diff_logits), _ptr(draft_tokens), _ptr(accept_u), _ptr(gumbel),
            _ptr(kb), _ptr(vb), _ptr(kp), _ptr(vp), sl, sp, sh, st, _ptr(page_table), _ptr(seq_lens),
            _ptr(accept_len), _ptr(num_committed), _ptr(out_tokens), _ptr(next_anchor), _ptr(m_acc), _ptr(m_draw))
    if rc != 0 and not (rc == -4 and allow_capacity_error):
        raise RuntimeError("orthrus_oracle_sampling_consensus_commit failed with status %d" % rc)
    return dict(accept_len=accept_len, num_committed=num_committed, out_tokens=out_tokens,
                next_anchor=next_anchor, status=rc, margin_accept=m_acc, margin_draw=m_draw)


def block_mask_attn(sm_scale: float, block_k: int, anchors: np.ndarray, q_diff: np.ndarray,
                    k_ar: np.ndarray, v_ar: np.ndarray, k_diff: np.ndarray, v_diff: np.ndarray) -> np.ndarray:
    """Diffusion-view attention under the training block mask M_diff (Section 3.2, Eq. 6), evaluated literally.

    The key axis is the L clean AR keys followed by the NB*K diffusion keys of all blocks.  For the diffusion
    query at index qi (block nb = qi // K, anchor a = anchors[nb]) and key index k:
        allowed  <=>  (k < L and k <= a - 1)  or  (k >= L and qi // K == (k - L) // K)
    Dense scores over the whole key axis, the mask, a softmax and the weighted sum, in fp64 with numpy
    (one query head at a time).  ``q_diff`` [NB*K,H_q,d], ``k_ar``/``v_ar`` [L,H_kv,d],
    ``k_diff``/``v_diff`` [NB*K,H_kv,d] as bf16 bit patterns; returns fp64 [NB*K,H_q,d].
    """
    from orthrus_inputs import bf16_bits_to_f32
    f = lambda a: bf16_bits_to_f32(a).astype(np.float64)
    Q, KA, VA, KD, VD = f(q_diff), f(k_ar), f(v_ar), f(k_diff), f(v_diff)
    NQ, Hq, d = Q.shape
    L, Hkv, _ = KA.shape
    K = int(block_k)
    if NQ % K or KD.shape[0] != NQ or len(anchors) != NQ // K:
        raise ValueError("shape mismatch")
    G = Hq // Hkv
    qi = np.arange(NQ)[:, None]
    kk = np.arange(L + NQ)[None, :]
    a_of_q = np.asarray(anchors, dtype=np.int64)[qi // K]
    allowed = ((kk < L) & (kk <= a_of_q - 1)) | ((kk >= L) & (qi // K == (kk - L) // K))
    out = np.empty((NQ, Hq, d), dtype=np.float64)
    for h in range(Hq):
        g = h // G
        keys = np.concatenate([KA[:, g], KD[:, g]])
        vals = np.concatenate([VA[:, g], VD[:, g]])
        s = (Q[:, h] @ keys.T) * float(sm_scale)
        s = np.where(allowed, s, -np.inf)
        s = s - s.max(axis=1, keepdims=True)
        p = np.exp(s)
        p /= p.sum(axis=1, keepdims=True)
        out[:, h] = p @ vals
    return out


# ---- the operators around the decode step: plain numpy, fp64, one row or request after another

def filter_row(x: np.ndarray, temperature: float, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0):
    """What temperature, top-k, top-p and min-p leave of one logits row: (kept tokens in rising order, their
    probabilities), both empty for a row of nothing but -inf."""
    idx, w = _filter_weights(x, temperature, top_k, top_p, min_p)
    return idx, w / w.sum()


def _filter_weights(x, temperature, top_k, top_p, min_p):
    """The same with the weights before they are normalised (whole numbers stay whole: equal logits weigh 1 each).

    Literal: sort by (logit falling, index rising), weights exp((x - max) / T); the first top_k; of those the shortest
    prefix holding top_p of their weight; of those the ones with a weight of at least min_p; renormalise.
    """
    x = np.asarray(x, dtype=np.float64).copy()
    x[np.isnan(x)] = -np.inf
    x = np.minimum(x, np.float64(np.finfo(np.float32).max))
    order = np.lexsort((np.arange(x.size), -x))
    order = order[x[order] > -np.inf]
    if order.size == 0:
        return order, np.empty(0)
    if not temperature > 0:
        return order[:1], np.ones(1)
    w = np.exp((x[order] - x[order[0]]) / np.float64(min(temperature, np.finfo(np.float32).max)))
    if 0 < top_k < x.size:
        order, w = order[:top_k], w[:top_k]
    if top_p < 1:
        sums = np.cumsum(w)
        n = int(np.count_nonzero(sums < np.float64(top_p) * sums[-1])) + 1
        order, w = order[:max(n, 1)], w[:max(n, 1)]
    if min_p > 0:
        keep = w >= min(np.float64(min_p), 1.0)
        order, w = order[keep], w[keep]
    by_index = np.argsort(order)
    return order[by_index], w[by_index]


def sample_tokens(logits: np.ndarray, temperature, top_k, top_p, min_p, u: np.ndarray):
    """Tokens [B,K] and log-probabilities: the first kept token whose running probability exceeds u.

    ``logits`` [B,K,V] (any float type numpy can widen); the filters are arrays [B] or None.  Also returns, per row, how
    far u is from the nearest value at which the token would change.
    """
    B, K, V = logits.shape
    tokens, lp, margin = np.full((B, K), -1, np.int32), np.full((B, K), -np.inf), np.full((B, K), np.inf)
    for b in range(B):
        f = (float(temperature[b]), 0 if top_k is None else int(top_k[b]), 1.0 if top_p is None else float(top_p[b]),
             0.0 if min_p is None else float(min_p[b]))
        for k in range(K):
            idx, w = _filter_weights(logits[b, k], *f)
            if not idx.size:
                continue
            v = float(u[b, k])
            v = 0.0 if np.isnan(v) else min(max(v, 0.0), 1.0 - 2.0 ** -24)
            sums = np.cumsum(w)
            i = min(int(np.count_nonzero(sums <= v * sums[-1])), idx.size - 1)
            tokens[b, k] = idx[i]
            lp[b, k] = np.log(w[i] / sums[-1]) if w[i] > 0 else -np.inf
            if idx.size > 1:
                margin[b, k] = np.min(np.abs(sums[:-1] / sums[-1] - v))
    return tokens, lp, margin


def filtered_consensus_commit(ar_logits, diff_logits, temperature, top_k, top_p, min_p, draft_tokens, accept_u, gumbel,
                              k_blk_ar=None, v_blk_ar=None, k_pool=None, v_pool=None, page_table=None, seq_lens=None):
    """The keep/replace rule of ``sampling_consensus_commit`` on the filtered distributions, and the commit
    (pools [layers,pages,H_kv,P,d] and ``seq_lens`` updated in place; an unmapped position leaves the sequence alone)."""
    B, K, V = ar_logits.shape
    accept_len, num_committed, next_anchor = (np.zeros(B, np.int32) for _ in range(3))
    out_tokens = np.full((B, K), -1, np.int32)
    status = 0
    margin = np.inf
    for b in range(B):
        f = (float(temperature[b]), 0 if top_k is None else int(top_k[b]), 1.0 if top_p is None else float(top_p[b]),
             0.0 if min_p is None else float(min_p[b]))
        j = 0
        while j < K:
            p, q = np.zeros(V), np.zeros(V)
            for x, into in ((ar_logits[b, j], p), (diff_logits[b, j], q)):
                idx, prob = filter_row(x, *f)
                into[idx] = prob
            x = int(draft_tokens[b, j])
            if 0 <= x < V:
                a, c = float(accept_u[b, j]) * q[x], p[x]
                margin = min(margin, abs(a - c) / max(a, c) if max(a, c) > 0 else np.inf)
                if a < c:
                    out_tokens[b, j] = next_anchor[b] = x
                    j += 1
                    continue
            r = p - q
            if not (r > 0).any():
                r = p
            score = np.full(V, -np.inf)
            pos = r > 0
            score[pos] = np.log(r[pos]) + gumbel[b].astype(np.float64)[pos]
            out_tokens[b, j] = next_anchor[b] = int(np.argmax(score)) if pos.any() else -1
            break
        accept_len[b] = j
        m = num_committed[b] = min(j + 1, K)
        if k_blk_ar is None:
            continue
        P, L = k_pool.shape[3], int(seq_lens[b])
        slots = [(L + i) // P for i in range(m)]
        pages = [int(page_table[b, s]) if s < page_table.shape[1] else -1 for s in slots]
        if any(not 0 <= g < k_pool.shape[1] for g in pages):
            num_committed[b], status = 0, -4
            continue
        for i, g in enumerate(pages):
            k_pool[:, g, :, (L + i) % P] = k_blk_ar[:, b, i]
            v_pool[:, g, :, (L + i) % P] = v_blk_ar[:, b, i]
        seq_lens[b] = L + m
    return dict(accept_len=accept_len, num_committed=num_committed, out_tokens=out_tokens, next_anchor=next_anchor,
                status=status, margin=margin)


def page_tables_update(seq_lens, new_lens, page_table, free_pages, free_state, page_size: int, max_seq_len: int, max_tokens: int,
                       slot_map: np.ndarray):
    """Pages and slots for requests that grow, pages back from those that ended; tables, ring and ``slot_map`` in place.
    Returns granted, token_starts and the status (0 or -4)."""
    B, width = page_table.shape
    N, P = free_pages.size, page_size
    mapped = lambda page: 0 <= page < N  # noqa: E731
    head, count = int(free_state[0]) % N, min(max(int(free_state[1]), 0), N)
    granted, starts = np.zeros(B, np.int32), np.zeros(B + 1, np.int32)
    wanted, taken, back, status, tokens = 0, 0, [], 0, 0
    for b in range(B):
        L, n, row = int(seq_lens[b]), int(new_lens[b]), page_table[b]
        starts[b] = min(tokens, 2 ** 31 - 1)
        if n < 0:
            for e in range(width):
                if mapped(row[e]):
                    back.append(int(row[e]))
                    row[e] = -1
            continue
        if L < 0 or L + n > max_seq_len or (n > 0 and L % P and not mapped(row[L // P])):
            status = -4
            continue
        lacks = [e for e in range(L // P, (L + n - 1) // P + 1) if not mapped(row[e])] if n else []
        wanted += len(lacks)
        if lacks and wanted > count:
            status = -4
            continue
        for e in lacks:
            row[e] = free_pages[(head + taken) % N]
            taken += 1
        granted[b] = n
        for i in range(n):
            page = int(row[(L + i) // P])
            status = status if mapped(page) else -4
            if tokens + i < max_tokens:
                slot_map[tokens + i] = page * P + (L + i) % P if mapped(page) else -1
        tokens += n
    starts[B] = min(tokens, 2 ** 31 - 1)
    if len(back) > N - count or tokens > max_tokens:
        status = -4
    for i, page in enumerate(back[:N - count]):
        free_pages[(head + count + i) % N] = page
    free_state[0], free_state[1] = (head + taken) % N, count - taken + min(len(back), N - count)
    return granted, starts, status


def kv_store(k_new, v_new, slot_map, k_pool, v_pool, num_valid=None):
    """Rows [layers,N,H_kv,d] to their slots of the pools [layers,pages,H_kv,P,d], in place; the status (0 or -4)."""
    P, slots, status = k_pool.shape[3], k_pool.shape[1] * k_pool.shape[3], 0
    n = len(slot_map) if num_valid is None else min(max(int(num_valid), 0), len(slot_map))
    for t in range(n):
        s = int(slot_map[t])
        if s >= slots:
            status = -4
        elif s >= 0:
            k_pool[:, s // P, :, s % P] = k_new[:, t]
            v_pool[:, s // P, :, s % P] = v_new[:, t]
    return status
