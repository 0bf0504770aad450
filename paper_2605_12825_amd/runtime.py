"""Convenience holder for one decode-step configuration: context, params and workspaces.

Pure plumbing around the C ABI (torch provides device memory and the current stream); every
computation happens inside liborthrus.so.
"""
from __future__ import annotations

import ctypes
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
        # whose plan needs more gets a larger one here (rare, and never inside a captured sequence)
        n = B.orthrus_attn_workspace_bytes_on(self.ctx, self.params)
        if n > self.attn_ws.numel():
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

    def reserve(self, sampling=False, tables=False) -> None:
        """Makes the workspaces of sample_tokens and filtered_consensus_commit, or of update_page_tables, ahead of their first
        call: a program that records calls into a graph does this before.  Calls that overlap in time, in replays of two graphs as on
        two streams, need a step each."""
        if sampling:
            self._workspace("sample_ws", B.orthrus_sample_workspace_bytes)
            self._workspace("filtered_ws", B.orthrus_filtered_workspace_bytes)
        if tables:
            self._workspace("tables_ws", B.orthrus_page_tables_workspace_bytes)

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
                 diffusion_passes=1, device=0, filters=False, free_pages=None, free_state=None):
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
        blk = (num_layers, batch, block_k, num_kv_heads, head_dim)
        qs = (num_layers, batch, block_k, num_q_heads, head_dim)
        i16 = dict(dtype=torch.int16, device=dev)
        self.q_diff, self.q_ar = torch.zeros(qs, **i16), torch.zeros(qs, **i16)
        self.k_blk_diff, self.v_blk_diff = torch.zeros(blk, **i16), torch.zeros(blk, **i16)
        self.k_blk_ar, self.v_blk_ar = torch.zeros(blk, **i16), torch.zeros(blk, **i16)
        self.out_diff, self.out_ar = torch.zeros(qs, **i16), torch.zeros(qs, **i16)
        self.ar_logits = torch.zeros((batch, block_k, vocab), dtype=torch.float32, device=dev)
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
        # a ring of free pages: the cycle first maps pages for `grow` tokens more per request, block_k each.  A request that
        # is not granted them (`granted` is 0) sets the error word (ORTHRUS_ECAPACITY) as every page that is missing does; it is
        # decoded all the same, and where its kept rows do not fit into the pages that it has, none is committed (`num_committed`
        # is 0) and it goes on in a later cycle.  end() takes the pages of requests that are over between two cycles, without an
        # error.  -1 in `grow` takes them within one: put the length to 0 before it (the cycle decodes all slots, and tokens
        # behind cleared entries are read from page 0), and note that the commit finds no page for that slot and reports it.
        self.free_pages, self.free_state = free_pages, free_state
        if free_pages is not None:
            if free_pages.numel() != pages or free_state is None:
                raise ValueError("free_pages holds num_pages entries and comes with free_state")
            self.grow = torch.full((batch,), block_k, **i32)
            self.granted, self.token_starts = torch.zeros((batch,), **i32), torch.zeros((batch + 1,), **i32)
            self.slot_map = torch.zeros((batch * block_k,), **i32)
            self.step.reserve(tables=True)
        self.accept_len, self.num_committed, self.next_anchor = (torch.zeros((batch,), **i32) for _ in range(3))
        self.out_tokens = torch.zeros((batch, block_k), **i32)
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
                s.attn(view, q[l], kb[l], vb[l], self.k_pool[l], self.v_pool[l], self.page_table, self.seq_lens,
                       out[l], None, stream)
        if self.filters:
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

        With `grow` left at block_k the slots stay in the cycles, each with a block's pages, until the next requests take them;
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
        finally:
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
