"""Convenience holder for one decode-step configuration: context, params and workspaces.

Pure plumbing around the C ABI (torch provides device memory and the current stream); every
computation happens inside liborthrus.so.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import numpy as np
import torch

from . import binding as B


def to_device_bits(a: np.ndarray, device="cuda:0") -> torch.Tensor:
    """Uploads a numpy array; uint16 bf16 bit patterns travel as int16 (same bits)."""
    if a.dtype == np.uint16:
        a = a.view(np.int16)
    return torch.from_numpy(np.ascontiguousarray(a)).to(device)


def bits_to_numpy(t: torch.Tensor) -> np.ndarray:
    a = t.detach().cpu().numpy()
    return a.view(np.uint16) if a.dtype == np.int16 else a


_LOGITS_TYPES = {torch.float32: B.ORTHRUS_F32, torch.bfloat16: B.ORTHRUS_BF16, torch.float16: B.ORTHRUS_F16}


def _logits_type(stride_row, *logits) -> int:
    """The ABI's name of the logits' type; every tensor of a call has the same.  A view of padded rows comes with its stride."""
    dtype = logits[0].dtype
    t = _LOGITS_TYPES.get(dtype)
    for x in logits:
        if t is None or x.dtype is not dtype:
            raise ValueError("logits must be float32, bfloat16 or float16, all of one type")
        if stride_row == 0 and not x.is_contiguous():
            raise ValueError("logits whose rows are not dense need logits_stride_row")
    return t


_F32, _I32 = torch.float32, torch.int32
_ROWS_16 = frozenset((torch.bfloat16, torch.int16, torch.uint16))   # bf16, or its bits
_DENSE = (0, 0, 0)   # strides of layer, row and head
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _recording(stream, device) -> bool:
    """Whether what is called on that stream (a torch Stream or a handle) goes into a graph; None: not asked."""
    handle = 0 if stream is None else stream if stream.__class__ is int else int(stream.cuda_stream)
    if handle == 0:   # (the null stream cannot be recorded)
        return False
    with torch.cuda.stream(torch.cuda.ExternalStream(handle, device=device)):
        return torch.cuda.is_current_stream_capturing()


def _check_operands(*operands) -> None:
    """(name, tensor, type, elements): what is of another type (torch makes whole numbers 64 bits wide), too short, or a column of
    something larger would be read as what it is not.  None and addresses stand for themselves."""
    for name, t, dtype, count in operands:
        if t is not None and t.__class__ is not int and (t.dtype is not dtype or t.numel() < count or not t.is_contiguous()):
            raise ValueError("%s must hold %d dense elements of %s, not %s of %s with strides %s"
                             % (name, count, dtype, tuple(t.shape), t.dtype, t.stride()))


def _check_type(name, t, dtype) -> None:
    if t is not None and t.__class__ is not int and t.dtype is not dtype:
        raise ValueError("%s must be of %s, not %s" % (name, dtype, t.dtype))


def _check_filters(batch, temperature, top_k, top_p, min_p) -> None:
    # (The smallest calls take as long as the host needs for them, and the types say all there is to say of one element: 0.5 us, the
    # whole check 1.5.)
    if batch == 1 and (temperature is None or temperature.__class__ is int or temperature.dtype is _F32) and \
            (top_k is None or top_k.__class__ is int or top_k.dtype is _I32) and \
            (top_p is None or top_p.__class__ is int or top_p.dtype is _F32) and \
            (min_p is None or min_p.__class__ is int or min_p.dtype is _F32):
        return
    _check_operands(("temperature", temperature, _F32, batch), ("top_k", top_k, _I32, batch), ("top_p", top_p, _F32, batch),
                    ("min_p", min_p, _F32, batch))


def _rows_lie(t, shape, strides) -> bool:
    """Whether a tensor's elements lie where a call looks for rows [layers, rows, heads, d] with these strides of a layer, row and head
    (0: dense), in whatever dimensions."""
    layers, rows, heads, d = shape
    layer, row, head = strides
    head = head or d
    row = row or heads * d
    try:
        at = t.view(shape).stride()
    except RuntimeError:   # (its rows are not evenly apart)
        return False
    return rows == 0 or all(n == 1 or x == y for n, x, y in zip(shape, at, (layer or rows * row, row, head, 1)))


def _lie(*tensors):
    return tuple((t.shape, t.stride()) for t in tensors)


def _check_rows(name, t, shape, strides) -> None:
    if t.__class__ is not int and (t.dtype not in _ROWS_16 or t.numel() != math.prod(shape) or not _rows_lie(t, shape, strides)):
        raise ValueError("%s must hold [%s] elements of bf16 with strides %s of layer, row and head (0: dense), not %s of %s with strides %s"
                         % (name, ", ".join(map(str, shape)), strides, tuple(t.shape), t.dtype, t.stride()))


def _check_cache(p, k_pool, v_pool, page_table, seq_lens) -> None:
    """A call's cache: bf16 pools, pages and lengths of 32 bits (of 64, every other one would be the upper half of its neighbour)."""
    for name, t in (("k_pool", k_pool), ("v_pool", v_pool)):
        if t is not None and t.__class__ is not int and t.dtype not in _ROWS_16:
            raise ValueError("%s must be of bf16, not %s" % (name, t.dtype))
    _check_operands(("page_table", page_table, _I32, p.batch * p.max_pages_per_seq), ("seq_lens", seq_lens, _I32, p.batch))


def _check_device(device, **operands) -> None:
    """Everything lies on the step's device: a kernel given another address space's would fault.  None and addresses stand for
    themselves."""
    for name, t in operands.items():
        if t is not None and t.__class__ is not int and t.device != device:
            raise ValueError("%s must be on %s, not on %s" % (name, device, t.device))


def _check_logits_rows(name, t, rows, vocab, stride_row) -> None:
    """A tensor of logits, or a view of one, has its rows where the call reads them: row i at i * stride_row from its start."""
    pitch = stride_row or vocab
    if t.is_contiguous() and (t.numel() == rows * pitch or t.dim() == 1 and t.numel() >= (rows - 1) * pitch + vocab):
        return
    fits = t.dim() > 0 and t.shape[-1] >= vocab and (t.shape[-1] == 1 or t.stride(-1) == 1)
    n = 1   # rows of the dimensions so far
    for size, stride in zip(t.shape[-2::-1], t.stride()[-2::-1]):
        fits = fits and (size == 1 or stride == n * pitch)
        n *= size
    if not fits or n != rows:
        raise ValueError("%s must hold %d rows of %d logits, %d apart, not %s with strides %s" % (name, rows, vocab, pitch, tuple(t.shape), t.stride()))


class LogitRules:
    """What requests ask of their tokens, for DecodeStep.process_logits: tensors on the device, one entry a request.  What is None
    is off.  The tensors' contents may change from call to call.

    history [batch, most tokens] and history_lens: the tokens before the anchor, the prompt's (prompt_lens of them) first;
    repetition, presence, frequency: penalties for tokens that are in it or on the row's path; bias_starts [batch + 1], bias_tokens
    and bias_values: entries bias_starts[b] .. bias_starts[b + 1] - 1 are request b's, the last of a token counts; masks
    [number, words of 32 tokens] with a bit set for every token allowed and mask_rows [batch, rows] that names each row's, -1 for none.
    """

    def __init__(self, *, history=None, history_lens=None, prompt_lens=None, repetition=None, presence=None, frequency=None,
                 bias_starts=None, bias_tokens=None, bias_values=None, masks=None, mask_rows=None):
        for name, t, dims, dtype in (("history", history, 2, _I32), ("history_lens", history_lens, 1, _I32), ("prompt_lens", prompt_lens, 1, _I32),
                                     ("repetition", repetition, 1, _F32), ("presence", presence, 1, _F32), ("frequency", frequency, 1, _F32),
                                     ("bias_starts", bias_starts, 1, _I32), ("bias_tokens", bias_tokens, 1, _I32),
                                     ("bias_values", bias_values, 1, _F32), ("masks", masks, 2, _I32), ("mask_rows", mask_rows, None, _I32)):
            if t is not None and (t.dtype is not dtype or dims is not None and t.dim() != dims or not t.is_contiguous()):
                raise ValueError("%s must be dense, of %s%s, not %s of %s" % (name, dtype, "" if dims is None else " and %d dimensions" % dims,
                                                                              tuple(t.shape), t.dtype))
        for a, b, both in ((history, history_lens, "history and history_lens"), (masks, mask_rows, "masks and mask_rows"),
                           (bias_starts, bias_tokens, "bias_starts and bias_tokens"), (bias_tokens, bias_values, "bias_tokens and bias_values")):
            if (a is None) != (b is None):
                raise ValueError("%s come together" % both)
        if prompt_lens is not None and history is None:
            raise ValueError("prompt_lens comes with history")
        if bias_tokens is not None and bias_tokens.numel() != bias_values.numel():
            raise ValueError("bias_tokens and bias_values have as many entries")
        self.history, self.history_lens, self.prompt_lens = history, history_lens, prompt_lens
        self.repetition, self.presence, self.frequency = repetition, presence, frequency
        self.bias_starts, self.bias_tokens, self.bias_values = bias_starts, bias_tokens, bias_values
        self.masks, self.mask_rows = masks, mask_rows
        r = self.c = B.orthrus_logit_rules()
        for name in ("history", "history_lens", "prompt_lens", "repetition", "presence", "frequency", "bias_starts", "bias_tokens",
                     "bias_values", "masks", "mask_rows"):
            setattr(r, name, B._ptr(getattr(self, name)))
        if history is not None and history.numel() == 0:   # nothing can stand in it
            r.history = r.history_lens = r.prompt_lens = None
        if masks is not None and (masks.numel() == 0 or mask_rows.numel() == 0):   # no row has one
            r.masks = r.mask_rows = None
        r.history_stride = 0 if history is None else history.shape[1]
        r.num_biases = 0 if bias_tokens is None else bias_tokens.numel()
        r.num_masks, r.mask_stride = masks.shape if r.masks else (0, 0)
        self.checked = None   # the batch, rows, vocabulary and device that they are known to fit

    def check(self, batch, rows, vocab, device=None) -> None:
        """Refuses rules of another batch, block or vocabulary, or on another device."""
        for name in ("history", "history_lens", "prompt_lens", "repetition", "presence", "frequency", "bias_starts", "bias_tokens",
                     "bias_values", "masks", "mask_rows"):
            t = getattr(self, name)
            if t is not None and device is not None and t.device != device:
                raise ValueError("%s must be on %s, not on %s" % (name, device, t.device))
        _check_operands(*((name, getattr(self, name), dtype, batch) for name, dtype in
                          (("history_lens", _I32), ("prompt_lens", _I32), ("repetition", _F32), ("presence", _F32), ("frequency", _F32))),
                        ("bias_starts", self.bias_starts, _I32, batch + 1), ("mask_rows", self.mask_rows, _I32, batch * rows))
        if self.history is not None and self.history.shape[0] != batch:
            raise ValueError("history must have a row for each of %d requests, not %s" % (batch, tuple(self.history.shape)))
        if self.mask_rows is not None and self.mask_rows.numel() != batch * rows:
            raise ValueError("mask_rows must name a mask for each of %d x %d rows, not %s" % (batch, rows, tuple(self.mask_rows.shape)))
        if self.masks is not None and self.masks.shape[1] < (vocab + 31) // 32:
            raise ValueError("masks must have %d words for %d tokens, not %d" % ((vocab + 31) // 32, vocab, self.masks.shape[1]))
        self.checked = (batch, rows, vocab, device)


class DecodeStep:
    """Owns an orthrus context plus the attention / consensus workspaces for fixed shapes."""

    def __init__(self, *, batch, num_q_heads, num_kv_heads, head_dim, block_k, page_size, max_pages_per_seq,
                 max_seq_len, num_pages, vocab=0, num_layers=1, num_splits=0, sm_scale=None, device=0,
                 pool_strides=None, min_seq_len_bound=None, block_strides=None):
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2605_12825_amd needs a HIP device; there is no CPU path")
        self.device = torch.device("cuda", device)
        kw = {}
        if pool_strides is not None:
            kw = dict(pool_stride_layer=pool_strides[0], pool_stride_page=pool_strides[1],
                      pool_stride_head=pool_strides[2], pool_stride_tok=pool_strides[3])
        if block_strides is not None:   # (q_stride_row, q_stride_head, blk_stride_row, blk_stride_head, blk_stride_layer)
            kw.update(q_stride_row=block_strides[0], q_stride_head=block_strides[1], blk_stride_row=block_strides[2],
                      blk_stride_head=block_strides[3], blk_stride_layer=block_strides[4])
        self.params = B.make_params(batch=batch, num_q_heads=num_q_heads, num_kv_heads=num_kv_heads,
                                    head_dim=head_dim, block_k=block_k, page_size=page_size,
                                    max_pages_per_seq=max_pages_per_seq, max_seq_len=max_seq_len,
                                    num_pages=num_pages, num_splits=num_splits, num_layers=num_layers,
                                    vocab=vocab, sm_scale=sm_scale, **kw)
        # store_kv: how rows lie that the parameters describe; for the last number of them, their strides and bytes
        p = self.params
        self._row_strides = (p.blk_stride_row or num_kv_heads * head_dim, p.blk_stride_head or head_dim, 1)
        self._row_elements = num_layers * num_kv_heads * head_dim
        self._layout = (-1, None, 0)
        self.ctx = B.orthrus_create(device)
        # plans and sizes for the device the context lives on
        self.num_splits = B.orthrus_attn_num_splits_on(self.ctx, self.params)
        # workspace for every host bound on the lengths the caller may set later (see set_max_seq_len)
        n = B.orthrus_attn_workspace_bytes_on(self.ctx, self.params)
        lo = max_seq_len if min_seq_len_bound is None else min_seq_len_bound
        for bound in range(lo, max_seq_len, max(block_k, 1)):
            self.params.max_seq_len = bound
            n = max(n, B.orthrus_attn_workspace_bytes_on(self.ctx, self.params))
        self.params.max_seq_len = max_seq_len
        self._outgrown = []
        self._tree_attn_key = self._tree_consensus_key = (None, None)   # what their workspaces are made for, and these
        # the parameters of the last call whose operands were looked at in full, and what a call of the same ones compares: sizes in
        # bytes, how rows lie, its workspace
        self._tree_attn_known = self._tree_consensus_known = (None, None)
        self.attn_ws = torch.empty(max(n, 256), dtype=torch.uint8, device=self.device)
        self.cons_ws = None
        if vocab > 0:
            n = max(B.orthrus_consensus_workspace_bytes(self.params), B.orthrus_sampling_workspace_bytes(self.params))
            self.cons_ws = torch.empty(max(n, 256), dtype=torch.uint8, device=self.device)

    def set_max_seq_len(self, bound: int) -> None:
        """Tightens the host upper bound on the sequence lengths (it sizes the attention grid).

        `bound` must lie between the `min_seq_len_bound` and the `max_seq_len` given at construction,
        and must not be below any current sequence length.
        """
        self.params.max_seq_len = int(bound)
        self.num_splits = B.orthrus_attn_num_splits_on(self.ctx, self.params)
        # the constructor sized the workspace for the bounds min_seq_len_bound + i * block_k; any other bound
        # whose plan needs more gets a larger one here (rare, and never inside a captured sequence); graphs may have the smaller one
        n = B.orthrus_attn_workspace_bytes_on(self.ctx, self.params)
        if n > self.attn_ws.numel():
            self._outgrown.append(self.attn_ws)
            self.attn_ws = torch.empty(n, dtype=torch.uint8, device=self.device)

    def close(self):
        if self.ctx:
            torch.cuda.synchronize(self.device)
            B.orthrus_destroy(self.ctx)
            self.ctx = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    def attn(self, view, q, k_blk, v_blk, k_pool, v_pool, page_table, seq_lens, out, lse=None, stream=None):
        return B.orthrus_dual_view_attn(self.ctx, self.params, view, q, k_blk, v_blk, k_pool, v_pool, page_table,
                                        seq_lens, out, lse, self.attn_ws, stream)

    def consensus_commit(self, ar_logits, draft_tokens, k_blk_ar, v_blk_ar, k_pool, v_pool, page_table, seq_lens,
                         accept_len, num_committed, out_tokens, next_anchor, stream=None):
        return B.orthrus_consensus_commit(self.ctx, self.params, ar_logits, draft_tokens, k_blk_ar, v_blk_ar,
                                          k_pool, v_pool, page_table, seq_lens, accept_len, num_committed,
                                          out_tokens, next_anchor, self.cons_ws, stream)

    def sampling_consensus_commit(self, temperature, ar_logits, diff_logits, draft_tokens, accept_u, gumbel,
                                  k_blk_ar, v_blk_ar, k_pool, v_pool, page_table, seq_lens, accept_len,
                                  num_committed, out_tokens, next_anchor, stream=None):
        return B.orthrus_sampling_consensus_commit(self.ctx, self.params, temperature, ar_logits, diff_logits,
                                                   draft_tokens, accept_u, gumbel, k_blk_ar, v_blk_ar, k_pool, v_pool,
                                                   page_table, seq_lens, accept_len, num_committed, out_tokens,
                                                   next_anchor, self.cons_ws, stream)

    def prefill(self, max_new_tokens, q, k_new, v_new, new_lens, k_pool, v_pool, page_table, seq_lens, out,
                stream=None):
        """AR-view prefill attention of one layer (appends the new K/V rows, causal attention over the cache)."""
        need = B.orthrus_prefill_workspace_bytes(self.params, max_new_tokens)
        if getattr(self, "prefill_ws", None) is None or self.prefill_ws.numel() < need:
            self.prefill_ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        return B.orthrus_prefill_attn(self.ctx, self.params, max_new_tokens, q, k_new, v_new, new_lens, k_pool,
                                      v_pool, page_table, seq_lens, out, self.prefill_ws, stream)

    def _workspace(self, name, query):
        """The buffer kept for one kind of call (made on its first use; ahead of a captured sequence by reserve)."""
        ws = getattr(self, name, None)
        if ws is None:
            ws = torch.empty(max(query(self.params), 256), dtype=torch.uint8, device=self.device)
            with torch.cuda.device(self.device):
                if not torch.cuda.is_current_stream_capturing():   # the call may be on another stream than what used this memory before
                    torch.cuda.current_stream().synchronize()
            setattr(self, name, ws)
        return ws

    def reserve(self, sampling=False, tables=False, tree_nodes=0) -> None:
        """Makes the workspaces of sample_tokens and filtered_consensus_commit, of update_page_tables, or of tree_attn and
        tree_consensus_commit for trees of so many nodes (under the present max_seq_len), ahead of their first call: a program that
        records calls into a graph does this before.  Calls that overlap in time, in replays of two graphs as on two streams, need a
        step each."""
        if sampling:
            self._workspace("sample_ws", B.orthrus_sample_workspace_bytes)
            self._workspace("filtered_ws", B.orthrus_filtered_workspace_bytes)
        if tables:
            self._workspace("tables_ws", B.orthrus_page_tables_workspace_bytes)
        if tree_nodes:
            self._tree_attn_ws(tree_nodes)
            if self.params.vocab > 0:
                self._tree_consensus_ws(tree_nodes)

    def sample_tokens(self, logits, temperature, top_k, top_p, min_p, u, tokens, logprobs=None, stream=None,
                      logits_stride_row=0):
        """One token per logits row [batch, block_k, vocab] (float32, bfloat16 or float16; rows dense or logits_stride_row
        elements apart) by each sequence's temperature, top-k, top-p and min-p (each of the last three a [batch] tensor or None)
        from the uniform numbers u [batch, block_k]."""
        _check_filters(self.params.batch, temperature, top_k, top_p, min_p)
        _check_type("u", u, _F32)
        _check_type("tokens", tokens, _I32)
        ws = self._workspace("sample_ws", B.orthrus_sample_workspace_bytes)
        return B.orthrus_sample_tokens(self.ctx, self.params, _logits_type(logits_stride_row, logits), logits,
                                       logits_stride_row, temperature, top_k, top_p, min_p, u, tokens, logprobs, ws, stream)

    def filtered_consensus_commit(self, ar_logits, diff_logits, temperature, top_k, top_p, min_p, draft_tokens, accept_u,
                                  gumbel, k_blk_ar, v_blk_ar, k_pool, v_pool, page_table, seq_lens, accept_len,
                                  num_committed, out_tokens, next_anchor, stream=None, logits_stride_row=0):
        """sampling_consensus_commit where both views' distributions are filtered as in sample_tokens."""
        _check_filters(self.params.batch, temperature, top_k, top_p, min_p)
        _check_type("draft_tokens", draft_tokens, _I32)
        _check_type("accept_u", accept_u, _F32)
        _check_type("gumbel", gumbel, _F32)
        _check_type("out_tokens", out_tokens, _I32)
        ws = self._workspace("filtered_ws", B.orthrus_filtered_workspace_bytes)
        return B.orthrus_filtered_consensus_commit(self.ctx, self.params, _logits_type(logits_stride_row, ar_logits, diff_logits),
                                                   ar_logits, diff_logits, logits_stride_row, temperature, top_k, top_p, min_p,
                                                   draft_tokens, accept_u, gumbel, k_blk_ar, v_blk_ar, k_pool, v_pool,
                                                   page_table, seq_lens, accept_len, num_committed, out_tokens,
                                                   next_anchor, ws, stream)

    def update_page_tables(self, seq_lens, new_lens, page_table, free_pages, free_state, granted, token_starts, slot_map,
                           stream=None):
        """Pages for the sequences that grow by new_lens tokens, pages back from those with new_lens < 0, and the slots of
        the new tokens (packed; slot_map's length is the bound on their number)."""
        # (what a program makes anew for every step, and the ring, whose length it does not pass)
        if new_lens is not None and new_lens.__class__ is not int and new_lens.dtype is not _I32 or \
                free_pages is not None and free_pages.__class__ is not int and free_pages.numel() < self.params.num_pages:
            _check_operands(("new_lens", new_lens, _I32, self.params.batch), ("free_pages", free_pages, _I32, self.params.num_pages))
        ws = self._workspace("tables_ws", B.orthrus_page_tables_workspace_bytes)
        return B.orthrus_page_tables_update(self.ctx, self.params, seq_lens, new_lens, page_table, free_pages, free_state,
                                            granted, token_starts, slot_map, 0 if slot_map is None else slot_map.numel(),
                                            ws, stream)

    def store_kv(self, k_new, v_new, slot_map, k_pool, v_pool, num_valid=None, stream=None):
        """Copies packed K/V rows [num_layers, N, H_kv, d] (N = slot_map's length) to their slots in every layer's cache.  The rows
        are read where k_new and v_new have them (views of a fused projection's output, say), laid out alike; given as
        addresses, by the step's block strides."""
        rows = slot_map.numel()
        if slot_map.dtype is not _I32:   # (64-bit slots would be read as twice as many, every other one slot 0)
            _check_type("slot_map", slot_map, _I32)
        p = self.params
        if k_new.__class__ is not int and v_new.__class__ is not int:
            known, strides, size = self._layout
            if known != rows:
                strides, size = (p.blk_stride_layer or rows * self._row_strides[0],) + self._row_strides, 2 * rows * self._row_elements
                self._layout = (rows, strides, size)
            if k_new.stride() != strides or v_new.stride() != strides or k_new.nbytes != size or v_new.nbytes != size:
                p = self._params_for_rows(k_new, v_new, rows)
        try:   # straight to the library: a call of few rows takes as long as the host needs for it
            st = B._lib.orthrus_kv_store(self.ctx, ctypes.byref(p), rows, k_new.data_ptr(), v_new.data_ptr(), slot_map.data_ptr(),
                                         None if num_valid is None else num_valid.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(),
                                         B._stream_handle(stream))
        except AttributeError:   # (addresses among the operands)
            return B.orthrus_kv_store(self.ctx, p, rows, k_new, v_new, slot_map, num_valid, k_pool, v_pool, stream)
        if st != B.ORTHRUS_OK:
            raise B.OrthrusError(st, "orthrus_kv_store")
        return st

    def _params_for_rows(self, k_new, v_new, rows):
        """The step's parameters with the strides of these rows."""
        p, shape = self.params, (self.params.num_layers, rows, self.params.num_kv_heads, self.params.head_dim)
        if k_new.shape != shape or v_new.shape != shape or k_new.element_size() != 2 or v_new.element_size() != 2:
            raise ValueError("k_new and v_new must be [num_layers, slots, H_kv, d] = %s of 16 bits, not %s and %s of %s"
                             % (shape, tuple(k_new.shape), tuple(v_new.shape), k_new.dtype))
        strides = [0, 0, 0, 0]   # (0 is the library's word for dense; the stride of an axis of one element means nothing)
        if rows > 0:
            for i, (n, s, t) in enumerate(zip(shape, k_new.stride(), v_new.stride())):
                if n > 1 and (s != t or s == 0 or i == 3 and s != 1):
                    raise ValueError("k_new and v_new must be laid out alike, rows of dense elements, none of them twice: strides %s and %s"
                                     % (k_new.stride(), v_new.stride()))
                strides[i] = s if n > 1 else 0
        q = B.orthrus_params.from_buffer_copy(p)
        q.blk_stride_layer, q.blk_stride_row, q.blk_stride_head = strides[:3]
        return q

    def _stream(self, stream):
        """The caller's stream, or the current one of the step's device (a torch Stream object for it would take 2.9 us)."""
        if stream is not None:
            return stream
        return torch.cuda.current_stream(self.device) if _raw_stream is None else _raw_stream(self.device.index)

    def _sized_workspace(self, name, need, stream):
        """The buffer of a kind of call whose size goes by its arguments; a larger one takes its place (never inside a captured
        sequence: reserve comes before).  The smaller one stays: graphs and other streams may have it.  Each is at least twice
        as large as the one before, so that all of them together stay below twice the last."""
        ws = getattr(self, name, None)
        if ws is None or ws.numel() < need:
            with torch.cuda.device(self.device):
                if _recording(stream, self.device) or torch.cuda.is_current_stream_capturing():
                    raise RuntimeError("reserve() comes before a call is recorded")
                size = max(need, 256 if ws is None else 2 * ws.numel())
                new = torch.empty(size, dtype=torch.uint8, device=self.device)
                torch.cuda.current_stream().synchronize()   # the call may be on another stream than what used this memory before
            if ws is not None:
                self._outgrown.append(ws)
            ws = new
            setattr(self, name, ws)
        return ws

    def _tree_attn_ws(self, nodes, stream=None):
        key, ws = self._tree_attn_key
        if key != (nodes, self.params.max_seq_len):   # (a query is a call into the library)
            ws = self._sized_workspace("tree_attn_ws", B.orthrus_tree_attn_workspace_bytes(self.ctx, self.params, nodes), stream)
            self._tree_attn_key = (nodes, self.params.max_seq_len), ws
        return ws

    def _tree_consensus_ws(self, nodes, stream=None):
        key, ws = self._tree_consensus_key
        if key != nodes:
            ws = self._sized_workspace("tree_consensus_ws", B.orthrus_tree_consensus_workspace_bytes(self.params, nodes), stream)
            self._tree_consensus_key = nodes, ws
        return ws

    def tree_attn(self, parents, q, k_blk, v_blk, k_pool, v_pool, page_table, seq_lens, out, lse=None, stream=None):
        """Attention of a tree of drafts per sequence: parents [batch, nodes] (at most 64) names the node that each follows, -1 for
        node 0 and for unused ones; every node sees the cache, the nodes above it and itself.  Block tensors are [batch, nodes, ...]."""
        p, nodes = self.params, parents.shape[1]
        try:   # (the smallest calls take as long as the host needs for them: straight to the library where everything is as it was)
            key, known = self._tree_attn_known
            if key == (nodes, bytes(p)):
                types, parents_bytes, q_bytes, kv_bytes, table_bytes, lens_bytes, lse_bytes, lie, ws, ws_bytes, _ = known
                index = self.device.index
                if index == parents.get_device() == q.get_device() == k_blk.get_device() == v_blk.get_device() == k_pool.get_device() == \
                        v_pool.get_device() == page_table.get_device() == seq_lens.get_device() == out.get_device() and \
                        _I32 is parents.dtype is page_table.dtype is seq_lens.dtype and \
                        types == (q.dtype, k_blk.dtype, v_blk.dtype, k_pool.dtype, v_pool.dtype, out.dtype) and \
                        parents.nbytes == parents_bytes and q.nbytes == out.nbytes == q_bytes and k_blk.nbytes == v_blk.nbytes == kv_bytes and \
                        page_table.nbytes >= table_bytes and seq_lens.nbytes >= lens_bytes and \
                        parents.is_contiguous() and out.is_contiguous() and page_table.is_contiguous() and seq_lens.is_contiguous() and \
                        (q.is_contiguous() and k_blk.is_contiguous() and v_blk.is_contiguous() if lie is None else lie == _lie(q, k_blk, v_blk)) and \
                        (lse is None or lse.dtype is _F32 and lse.nbytes == lse_bytes and lse.is_contiguous() and lse.get_device() == index):
                    handle = _raw_stream(index) if stream is None and _raw_stream is not None else B._stream_handle(self._stream(stream))
                    st = B._lib.orthrus_tree_attn(self.ctx, ctypes.byref(p), nodes, parents.data_ptr(), q.data_ptr(), k_blk.data_ptr(),
                                                  v_blk.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), page_table.data_ptr(),
                                                  seq_lens.data_ptr(), out.data_ptr(), None if lse is None else lse.data_ptr(), ws, ws_bytes, handle)
                    if st != B.ORTHRUS_OK:
                        raise B.OrthrusError(st, "orthrus_tree_attn")
                    return st
        except AttributeError:   # (addresses among the operands)
            pass
        batch, hq, h, d = p.batch, p.num_q_heads, p.num_kv_heads, p.head_dim
        rows, at_q, at_kv = batch * nodes, (0, p.q_stride_row, p.q_stride_head), (0, p.blk_stride_row, p.blk_stride_head)
        _check_operands(("parents", parents, _I32, rows))
        _check_rows("q", q, (1, rows, hq, d), at_q)
        _check_rows("k_blk", k_blk, (1, rows, h, d), at_kv)
        _check_rows("v_blk", v_blk, (1, rows, h, d), at_kv)
        _check_rows("out", out, (1, rows, hq, d), _DENSE)
        _check_operands(("lse", lse, _F32, rows * hq))
        _check_cache(p, k_pool, v_pool, page_table, seq_lens)
        ws = self._tree_attn_ws(nodes) if stream is None else self._tree_attn_ws(nodes, stream)
        _check_device(self.device, parents=parents, q=q, k_blk=k_blk, v_blk=v_blk, k_pool=k_pool, v_pool=v_pool, page_table=page_table,
                      seq_lens=seq_lens, out=out, lse=lse)
        st = B.orthrus_tree_attn(self.ctx, p, nodes, parents, q, k_blk, v_blk, k_pool, v_pool, page_table, seq_lens, out, lse, ws,
                                 self._stream(stream))
        rows_16 = (q, k_blk, v_blk, k_pool, v_pool, out)
        if not any(t.__class__ is int for t in rows_16):
            self._tree_attn_known = (nodes, bytes(p)), (
                tuple(t.dtype for t in rows_16), 4 * rows, 2 * rows * hq * d, 2 * rows * h * d, 4 * batch * p.max_pages_per_seq, 4 * batch, 4 * rows * hq,
                None if at_q == at_kv == _DENSE else _lie(q, k_blk, v_blk), ws.data_ptr(), ws.nbytes, ws)
        return st

    def tree_consensus_commit(self, ar_logits, parents, node_tokens, k_blk_ar, v_blk_ar, k_pool, v_pool, page_table, seq_lens,
                              accept_len, num_committed, path_nodes, out_tokens, next_anchor, max_path=None, stream=None,
                              logits_stride_row=0):
        """Greedy consensus of a tree of drafts: from node 0 on to the child that holds the node's greedy token, for as long as there
        is one (and at most max_path nodes, where the trees are no deeper a bound on the launches); the path's K/V rows are committed.
        A row of nothing but -inf (no token is allowed) ends the path: next_anchor is -1."""
        p, nodes = self.params, parents.shape[1]
        longest = nodes if max_path is None else max_path
        try:
            key, known = self._tree_consensus_known
            if key == (nodes, logits_stride_row, bytes(p)):
                types, logits, kind, node_bytes, batch_bytes, table_bytes, kv_bytes, lie, ws, ws_bytes, _ = known
                index = self.device.index
                if index == ar_logits.get_device() == parents.get_device() == node_tokens.get_device() == path_nodes.get_device() == \
                        out_tokens.get_device() == accept_len.get_device() == num_committed.get_device() == next_anchor.get_device() == \
                        k_blk_ar.get_device() == v_blk_ar.get_device() == k_pool.get_device() == v_pool.get_device() == \
                        page_table.get_device() == seq_lens.get_device() and \
                        _I32 is parents.dtype is node_tokens.dtype is path_nodes.dtype is out_tokens.dtype is accept_len.dtype is num_committed.dtype \
                        is next_anchor.dtype is page_table.dtype is seq_lens.dtype and \
                        types == (k_blk_ar.dtype, v_blk_ar.dtype, k_pool.dtype, v_pool.dtype) and logits == (ar_logits.dtype, ar_logits.shape, ar_logits.stride()) and \
                        parents.nbytes == node_tokens.nbytes == path_nodes.nbytes == out_tokens.nbytes == node_bytes and \
                        accept_len.nbytes == num_committed.nbytes == next_anchor.nbytes == batch_bytes and seq_lens.nbytes >= batch_bytes and \
                        page_table.nbytes >= table_bytes and k_blk_ar.nbytes == v_blk_ar.nbytes == kv_bytes and \
                        parents.is_contiguous() and node_tokens.is_contiguous() and path_nodes.is_contiguous() and out_tokens.is_contiguous() and \
                        accept_len.is_contiguous() and num_committed.is_contiguous() and next_anchor.is_contiguous() and \
                        page_table.is_contiguous() and seq_lens.is_contiguous() and \
                        (k_blk_ar.is_contiguous() and v_blk_ar.is_contiguous() if lie is None else lie == _lie(k_blk_ar, v_blk_ar)):
                    handle = _raw_stream(index) if stream is None and _raw_stream is not None else B._stream_handle(self._stream(stream))
                    st = B._lib.orthrus_tree_consensus_commit(
                        self.ctx, ctypes.byref(p), kind, ar_logits.data_ptr(), logits_stride_row, nodes, longest, parents.data_ptr(),
                        node_tokens.data_ptr(), k_blk_ar.data_ptr(), v_blk_ar.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), page_table.data_ptr(),
                        seq_lens.data_ptr(), accept_len.data_ptr(), num_committed.data_ptr(), path_nodes.data_ptr(), out_tokens.data_ptr(),
                        next_anchor.data_ptr(), ws, ws_bytes, handle)
                    if st != B.ORTHRUS_OK:
                        raise B.OrthrusError(st, "orthrus_tree_consensus_commit")
                    return st
        except AttributeError:   # (addresses among the operands, or no rows to commit)
            pass
        batch = p.batch
        rows = batch * nodes
        kind = _logits_type(logits_stride_row, ar_logits)
        _check_logits_rows("ar_logits", ar_logits, rows, p.vocab, logits_stride_row)
        kv, at_kv = (p.num_layers, rows, p.num_kv_heads, p.head_dim), (p.blk_stride_layer, p.blk_stride_row, p.blk_stride_head)
        _check_operands(("parents", parents, _I32, rows), ("node_tokens", node_tokens, _I32, rows), ("path_nodes", path_nodes, _I32, rows),
                        ("out_tokens", out_tokens, _I32, rows), ("accept_len", accept_len, _I32, batch),
                        ("num_committed", num_committed, _I32, batch), ("next_anchor", next_anchor, _I32, batch))
        if k_blk_ar is not None and v_blk_ar is not None:
            _check_rows("k_blk_ar", k_blk_ar, kv, at_kv)
            _check_rows("v_blk_ar", v_blk_ar, kv, at_kv)
            _check_cache(p, k_pool, v_pool, page_table, seq_lens)
        ws = self._tree_consensus_ws(nodes) if stream is None else self._tree_consensus_ws(nodes, stream)
        _check_device(self.device, ar_logits=ar_logits, parents=parents, node_tokens=node_tokens, k_blk_ar=k_blk_ar, v_blk_ar=v_blk_ar, k_pool=k_pool,
                      v_pool=v_pool, page_table=page_table, seq_lens=seq_lens, accept_len=accept_len, num_committed=num_committed,
                      path_nodes=path_nodes, out_tokens=out_tokens, next_anchor=next_anchor)
        st = B.orthrus_tree_consensus_commit(self.ctx, p, kind, ar_logits, logits_stride_row, nodes, longest, parents, node_tokens, k_blk_ar,
                                             v_blk_ar, k_pool, v_pool, page_table, seq_lens, accept_len, num_committed, path_nodes, out_tokens,
                                             next_anchor, ws, self._stream(stream))
        rows_16 = (k_blk_ar, v_blk_ar, k_pool, v_pool)
        if all(torch.is_tensor(t) for t in rows_16):
            self._tree_consensus_known = (nodes, logits_stride_row, bytes(p)), (
                tuple(t.dtype for t in rows_16), (ar_logits.dtype, ar_logits.shape, ar_logits.stride()), kind, 4 * rows, 4 * batch, 4 * batch * p.max_pages_per_seq, 2 * math.prod(kv),
                None if at_kv == _DENSE else _lie(k_blk_ar, v_blk_ar), ws.data_ptr(), ws.nbytes, ws)
        return st

    def process_logits(self, logits, rules, tokens=None, parents=None, out=None, stream=None, logits_stride_row=0, out_stride_row=0):
        """Puts logits [batch, rows, vocab] (or [batch, vocab]) through their requests' LogitRules: in place, or into `out`.  tokens
        [batch, rows] are those fed at the rows and parents [batch, rows] the row that each follows (None: the one before it); they
        count as written on the way to a row.  Rows are dense or the given numbers of elements apart."""
        p, shape = self.params, logits.shape
        if len(shape) not in (2, 3) or shape[0] != p.batch:
            raise ValueError("logits must be [batch, rows, vocab] or [batch, vocab], not %s" % (tuple(shape),))
        batch, rows = p.batch, 1 if len(shape) == 2 else shape[1]
        kind = _logits_type(logits_stride_row, logits)
        _check_logits_rows("logits", logits, batch * rows, p.vocab, logits_stride_row)
        if out is None or out is logits:
            out, out_stride_row = logits, out_stride_row if out is logits else logits_stride_row
        else:
            if _logits_type(out_stride_row, out) != kind or out.device != logits.device:
                raise ValueError("out must be of the logits' type, on their device")
            _check_logits_rows("out", out, batch * rows, p.vocab, out_stride_row)
        if not (tokens is None or tokens.__class__ is not int and tokens.dtype is _I32 and tokens.nbytes == 4 * batch * rows and tokens.is_contiguous()) \
                or parents is not None:
            _check_operands(("tokens", tokens, _I32, batch * rows), ("parents", parents, _I32, batch * rows))
        if rules.checked != (batch, rows, p.vocab, logits.device):
            rules.check(batch, rows, p.vocab, logits.device)
        handle = self._stream(stream)
        index = self.device.index   # (out and the rules are on the logits' device)
        if logits.get_device() != index or tokens is not None and (tokens.__class__ is int or tokens.get_device() != index) or parents is not None:
            _check_device(self.device, logits=logits, tokens=tokens, parents=parents)
        return B.orthrus_logits_process(self.ctx, p, kind, logits, logits_stride_row, rows, tokens, parents, rules.c, out, out_stride_row, handle)

    def attn_timing(self, enable: bool) -> None:
        """Attach HIP events to the attention kernels of the following attn() calls (or stop doing so)."""
        B.orthrus_attn_timing(self.ctx, enable)

    def attn_timing_read(self):
        """(split us, launches, combine us, launches) summed over the timed launches since the last read."""
        return B.orthrus_attn_timing_read(self.ctx)

    def attn_timing_samples(self, capacity: int = 4096):
        """[(split kernel us, combine kernel us)] per timed call since the last read, in launch order."""
        return B.orthrus_attn_timing_samples(self.ctx, capacity)

    def kv_stream_probe(self, k_pool, v_pool, page_table, seq_lens, stream=None) -> None:
        """The attention call's K/V stream over this cache with idle compute waves (measurement)."""
        B.orthrus_kv_stream_probe(self.ctx, self.params, k_pool, v_pool, page_table, seq_lens, stream)

    def device_error(self, stream=None) -> int:
        return B.orthrus_last_device_error(self.ctx, stream)


class DecodeStack:
    """One decode cycle over a stack of layers, eagerly or as a replayed HIP graph.

    The cycle is the paper's: the diffusion view's pass through every layer, the AR view's
    verification pass through every layer, then the consensus and the commit of the accepted
    tokens' K/V into every layer's cache (Section 3.2-3.3, Fig. 2(b)).  Only the attention of each
    layer is computed here; whatever produces a layer's queries and block K/V writes them into
    this object's static buffers (`q_diff[l]`, `k_blk_diff[l]`, ... `ar_logits`, `draft_tokens`).
    Argument marshalling only: the loop below calls the C ABI once per layer and view.
    """

    def __init__(self, *, num_layers, batch, num_q_heads, num_kv_heads, head_dim, block_k, page_size,
                 k_pool, v_pool, page_table, seq_lens, max_seq_len, vocab, num_splits=0, temperature=0.0,
                 diffusion_passes=1, device=0, filters=False, free_pages=None, free_state=None, tree_nodes=0, tree_depth=0,
                 rules=None):
        if k_pool.dim() != 5 or k_pool.shape[0] != num_layers or not k_pool.is_contiguous():
            raise ValueError("pools must be contiguous [layers, pages, H_kv, P, d]")
        L, pages, H, P, d = k_pool.shape
        self.num_layers, self.temperature = num_layers, float(temperature)
        # forward passes of the diffusion view per cycle: 1 is the paper's single-step projection, 2 the
        # multi-step denoising variant of its ablation (Section 5, Table 3); the passes run back to back
        # over the same buffers (whatever refines the block between them writes q_diff / k_blk_diff / v_blk_diff)
        self.diffusion_passes = int(diffusion_passes)
        if self.diffusion_passes < 1:
            raise ValueError("diffusion_passes must be >= 1")
        self.k_pool, self.v_pool, self.page_table, self.seq_lens = k_pool, v_pool, page_table, seq_lens
        self.step = DecodeStep(batch=batch, num_q_heads=num_q_heads, num_kv_heads=num_kv_heads, head_dim=head_dim,
                               block_k=block_k, page_size=page_size, max_pages_per_seq=page_table.shape[1],
                               max_seq_len=max_seq_len, num_pages=pages, vocab=vocab, num_layers=num_layers,
                               num_splits=num_splits, device=device,
                               pool_strides=(pages * H * P * d, H * P * d, P * d, d))
        dev = self.step.device
        # tree_nodes: the AR view verifies a tree of so many drafts per sequence (node 0 is the anchor) of at most tree_depth levels,
        # greedily: the program writes `parents` and `node_tokens` and the tree's rows into `q_ar`, `k_blk_ar`, `v_blk_ar` and
        # `ar_logits`; the cycle leaves the path in `path_nodes`.  `rules` (LogitRules): `ar_logits` go through them, in place, each
        # node by its own path.  Their history is the program's to extend between two cycles, by the path's node_tokens.  Where a
        # path comes to a node whose mask allows no token, it ends there and `next_anchor` is -1.
        self.tree_nodes, self.rules = int(tree_nodes), rules
        self.tree_depth = int(tree_depth) if tree_depth else self.tree_nodes
        if self.tree_nodes and (self.temperature > 0 or filters):
            raise ValueError("trees are verified greedily: no temperature, no filters")
        if (tree_depth or rules is not None) and not self.tree_nodes or self.tree_depth < 0 or self.tree_nodes < 0:
            raise ValueError("tree_depth and rules are for stacks with tree_nodes")
        verified = self.tree_nodes or block_k
        i16 = dict(dtype=torch.int16, device=dev)

        def block(rows, heads):
            return torch.zeros((num_layers, batch, rows, heads, head_dim), **i16)
        self.q_diff, self.q_ar = block(block_k, num_q_heads), block(verified, num_q_heads)
        self.k_blk_diff, self.v_blk_diff = block(block_k, num_kv_heads), block(block_k, num_kv_heads)
        self.k_blk_ar, self.v_blk_ar = block(verified, num_kv_heads), block(verified, num_kv_heads)
        self.out_diff, self.out_ar = block(block_k, num_q_heads), block(verified, num_q_heads)
        self.ar_logits = torch.zeros((batch, verified, vocab), dtype=torch.float32, device=dev)
        self.draft_tokens = torch.zeros((batch, block_k), dtype=torch.int32, device=dev)
        self.filters = bool(filters)
        if self.temperature > 0 and not self.filters:
            self.diff_logits = torch.zeros_like(self.ar_logits)
            self.accept_u = torch.zeros((batch, block_k), dtype=torch.float32, device=dev)
            self.gumbel = torch.zeros((batch, vocab), dtype=torch.float32, device=dev)
        i32 = dict(dtype=torch.int32, device=dev)
        # filters: every request samples by its own `temperatures`, `top_k`, `top_p` and `min_p`; the cycle draws the drafts
        # itself, from `diff_logits` by `draft_u`, and verifies them under the same filters.  `temperatures` start at
        # `temperature`, at 1 where none is given.
        if self.filters:
            f32 = dict(dtype=torch.float32, device=dev)
            self.temperatures = torch.full((batch,), self.temperature if self.temperature > 0 else 1.0, **f32)
            self.top_p = torch.ones((batch,), **f32)
            self.top_k, self.min_p = torch.zeros((batch,), **i32), torch.zeros((batch,), **f32)
            self.diff_logits = torch.zeros_like(self.ar_logits)
            self.draft_u, self.accept_u = torch.zeros((batch, block_k), **f32), torch.zeros((batch, block_k), **f32)
            self.draft_logprobs = torch.zeros((batch, block_k), **f32)
            self.gumbel = torch.zeros((batch, vocab), **f32)
            self.step.reserve(sampling=True)
        # a ring of free pages: the cycle first maps pages for `grow` tokens more per request, block_k each (tree_depth for trees).  A request that
        # is not granted them (`granted` is 0) sets the error word (ORTHRUS_ECAPACITY) as every page that is missing does; it is
        # decoded all the same, and where its kept rows do not fit into the pages that it has, none is committed (`num_committed`
        # is 0) and it goes on in a later cycle.  end() takes the pages of requests that are over between two cycles, without an
        # error.  -1 in `grow` takes them within one: put the length to 0 before it (the cycle decodes all slots, and tokens
        # behind cleared entries are read from page 0), and note that the commit finds no page for that slot and reports it.
        self.free_pages, self.free_state = free_pages, free_state
        if free_pages is not None:
            if free_pages.numel() != pages or free_state is None:
                raise ValueError("free_pages holds num_pages entries and comes with free_state")
            most = min(self.tree_depth, self.tree_nodes) if self.tree_nodes else block_k   # tokens that a cycle may commit
            self.grow = torch.full((batch,), most, **i32)
            self.granted, self.token_starts = torch.zeros((batch,), **i32), torch.zeros((batch + 1,), **i32)
            self.slot_map = torch.zeros((batch * most,), **i32)
            self.step.reserve(tables=True)
        self.accept_len, self.num_committed, self.next_anchor = (torch.zeros((batch,), **i32) for _ in range(3))
        self.out_tokens = torch.zeros((batch, verified), **i32)
        if self.tree_nodes:
            self.parents = torch.arange(-1, verified - 1, **i32).repeat(batch, 1)   # a chain
            self.node_tokens, self.path_nodes = torch.zeros_like(self.out_tokens), torch.zeros_like(self.out_tokens)
            self.step.reserve(tree_nodes=verified)
            if rules is not None:
                rules.check(batch, verified, vocab, self.ar_logits.device)
        self.graph = None
        self.graph_stream = None

    def cycle(self, stream=None) -> None:
        """Issues the whole cycle on `stream` (default: the current stream)."""
        s = self.step
        diff = (0, self.q_diff, self.k_blk_diff, self.v_blk_diff, self.out_diff)
        ar = (1, self.q_ar, self.k_blk_ar, self.v_blk_ar, self.out_ar)
        if self.free_pages is not None:
            s.update_page_tables(self.seq_lens, self.grow, self.page_table, self.free_pages, self.free_state, self.granted,
                                 self.token_starts, self.slot_map, stream)
        for view, q, kb, vb, out in (diff,) * self.diffusion_passes + (ar,):
            if view == 1 and self.filters:
                s.sample_tokens(self.diff_logits, self.temperatures, self.top_k, self.top_p, self.min_p, self.draft_u,
                                self.draft_tokens, self.draft_logprobs, stream)
            for l in range(self.num_layers):
                if view == 1 and self.tree_nodes:
                    s.tree_attn(self.parents, q[l], kb[l], vb[l], self.k_pool[l], self.v_pool[l], self.page_table, self.seq_lens,
                                out[l], None, stream)
                    continue
                s.attn(view, q[l], kb[l], vb[l], self.k_pool[l], self.v_pool[l], self.page_table, self.seq_lens,
                       out[l], None, stream)
        if self.tree_nodes:
            if self.rules is not None:
                s.process_logits(self.ar_logits, self.rules, self.node_tokens, self.parents, stream=stream)
            s.tree_consensus_commit(self.ar_logits, self.parents, self.node_tokens, self.k_blk_ar, self.v_blk_ar, self.k_pool,
                                    self.v_pool, self.page_table, self.seq_lens, self.accept_len, self.num_committed,
                                    self.path_nodes, self.out_tokens, self.next_anchor, self.tree_depth, stream)
        elif self.filters:
            s.filtered_consensus_commit(self.ar_logits, self.diff_logits, self.temperatures, self.top_k, self.top_p,
                                        self.min_p, self.draft_tokens, self.accept_u, self.gumbel, self.k_blk_ar,
                                        self.v_blk_ar, self.k_pool, self.v_pool, self.page_table, self.seq_lens,
                                        self.accept_len, self.num_committed, self.out_tokens, self.next_anchor, stream)
        elif self.temperature > 0:
            s.sampling_consensus_commit(self.temperature, self.ar_logits, self.diff_logits, self.draft_tokens,
                                        self.accept_u, self.gumbel, self.k_blk_ar, self.v_blk_ar, self.k_pool,
                                        self.v_pool, self.page_table, self.seq_lens, self.accept_len,
                                        self.num_committed, self.out_tokens, self.next_anchor, stream)
        else:
            s.consensus_commit(self.ar_logits, self.draft_tokens, self.k_blk_ar, self.v_blk_ar, self.k_pool,
                               self.v_pool, self.page_table, self.seq_lens, self.accept_len, self.num_committed,
                               self.out_tokens, self.next_anchor, stream)

    def end(self, ended) -> None:
        """Requests that are over, between two cycles: the pages of those that `ended` ([batch], bool) marks go back to the ring,
        their lengths to 0.  Runs on the current stream; `granted` and `token_starts` are afterwards those of this call.

        With `grow` left as it is made the slots stay in the cycles, each with a block's pages, until the next requests take them;
        put their lengths to 0 before every cycle, or what they commit lets them grow.
        """
        if self.free_pages is None:
            raise ValueError("end() is for stacks with free_pages")
        if ended.dtype is not torch.bool or ended.shape != self.seq_lens.shape:
            raise ValueError("ended must be [batch] of torch.bool, not %s of %s" % (tuple(ended.shape), ended.dtype))
        new_lens = ended.to(torch.int32).neg_()
        self.step.update_page_tables(self.seq_lens, new_lens, self.page_table, self.free_pages, self.free_state, self.granted,
                                     self.token_starts, self.slot_map)
        self.seq_lens.masked_fill_(ended, 0)

    def capture(self) -> None:
        """Records one cycle into a HIP graph (on a stream of its own, default priority)."""
        if self.graph is not None:
            raise RuntimeError("already captured")
        torch.cuda.synchronize(self.step.device)
        self.graph_stream = torch.cuda.Stream(device=self.step.device)
        B.orthrus_graph_begin(self.step.ctx, self.graph_stream)
        try:
            self.cycle(self.graph_stream)
        except BaseException:   # a call was refused: what has been recorded is part of a cycle
            try:
                B.orthrus_graph_destroy(B.orthrus_graph_end(self.step.ctx, self.graph_stream))
            except B.OrthrusError:
                pass
            raise
        self.graph = B.orthrus_graph_end(self.step.ctx, self.graph_stream)

    def replay(self, stream=None) -> None:
        if self.graph is None:
            raise RuntimeError("capture() first")
        B.orthrus_graph_launch(self.graph, self.graph_stream if stream is None else stream)

    def close(self) -> None:
        if self.graph is not None:
            torch.cuda.synchronize(self.step.device)
            B.orthrus_graph_destroy(self.graph)
            self.graph = None
        self.step.close()
