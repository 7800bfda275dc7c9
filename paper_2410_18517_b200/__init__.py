"""Decode attention over a layer-shared KV cache (KVSharer's inference path) for B200.

``binding`` exposes the C ABI one to one.  ``SharedKVCache`` is a small holder
that lets PyTorch own the device memory (pool and workspace tensors) and the
stream, and forwards every operation to the compiled library.
"""
from __future__ import annotations

from . import binding
from .binding import (  # noqa: F401
    KVS_BF16, KVS_CACHE_4BIT, KVS_CACHE_PLAIN, KVS_F32, KVS_OK, KVS_OPT_EARLY_START, KVS_OPT_FINISH_IN_KERNEL, KVS_OPT_HOST_CHUNKS, KVS_OPT_KERNEL, KVS_OPT_MAX_CTAS, KVS_OPT_REPLAY, KVS_OPT_WAIT_LIMIT_US, KvsError,
)

__all__ = ["binding", "SharedKVCache", "Rotary", "KvsError"]


_unfinished = []        # caches closed while a graph was being recorded: (context, device, memory)


def _finish():
    """Ends the caches in ``_unfinished``, unless a graph is still being recorded."""
    if not _unfinished:
        return
    import torch

    while not torch.cuda.is_current_stream_capturing():
        try:
            ctx, device, _ = _unfinished.pop()
        except IndexError:              # the last one, or another thread had it
            return
        torch.cuda.synchronize(device)
        binding.kvs_destroy(ctx)


class Rotary:
    """Rotary positions for ``append_rotary``: radians per position of every pair (``rotary_dim / 2`` numbers).

    ``Rotary.from_theta(dim, theta)`` gives the usual ``theta ** (-2 i / dim)``.  ``interleaved``: pair i is elements
    (2i, 2i + 1) of the head instead of (i, i + dim / 2).
    """

    def __init__(self, inv_freq, interleaved=False):
        import ctypes

        values = [float(x) for x in inv_freq]
        self._array = (ctypes.c_double * max(len(values), 1))(*values)
        self.rotary_dim, self.interleaved = 2 * len(values), int(bool(interleaved))
        self._structs = {}

    def _struct(self, eps):
        s = self._structs.get(eps)
        if s is None:
            s = self._structs[eps] = binding.kvs_rotary(self.rotary_dim, self.interleaved, eps, self._array)
        return s

    @classmethod
    def from_theta(cls, rotary_dim, theta=10000.0, interleaved=False):
        return cls([theta ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)], interleaved)


class SharedKVCache:
    """One context + the torch tensors backing it.

    ``share_map[l] == l``: layer l computes its own K/V; ``share_map[l] == s < l``:
    layer l reads layer s's cache and appends nothing.  ``cache_format``: ``"plain"`` (rows in the storage type) or
    ``"4bit"`` (``kvs_set_cache_format`` says what a row holds and which calls take it).
    """

    def __init__(self, n_layers, n_q_heads, n_kv_heads, head_dim, max_batch, max_seq, dtype="bf16",
                 share_map=None, softmax_scale=0.0, device=0, cache_format="plain"):
        import torch

        _finish()
        self._torch = torch
        self.device = torch.device("cuda", device)
        self._index = device
        # the current stream's handle without a Stream object around it, where this torch has it
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        self.shape = (n_layers, n_q_heads, n_kv_heads, head_dim)
        self.max_batch = max_batch
        self._planes = None         # the pool, and the planes seen in it so far (see plane())
        self.ctx = binding.kvs_create(n_layers, n_q_heads, n_kv_heads, head_dim, max_batch, max_seq,
                                      KVS_BF16 if dtype == "bf16" else KVS_F32, softmax_scale, device)
        try:
            if share_map is not None:
                binding.kvs_set_share_map(self.ctx, share_map)
            self.cache_format = {"plain": KVS_CACHE_PLAIN, "4bit": KVS_CACHE_4BIT}[cache_format]
            binding.kvs_set_cache_format(self.ctx, self.cache_format)
            self.pool_bytes, self.workspace_bytes = binding.kvs_required_bytes(self.ctx)
            self.pool = self._allocate(self.pool_bytes)
            self.workspace = self._allocate(self.workspace_bytes)
            binding.kvs_bind_memory(self.ctx, self.pool, self.pool_bytes, self.workspace, self.workspace_bytes)
        except Exception:
            binding.kvs_destroy(self.ctx)
            self.ctx = None
            raise

    def _allocate(self, nbytes):
        """Device memory for the pool or the workspace (256-byte aligned uint8 tensor of ``nbytes``)."""
        return self._torch.empty(nbytes, dtype=self._torch.uint8, device=self.device)

    def close(self):
        _finish()
        if getattr(self, "ctx", None):
            if self._torch.cuda.is_current_stream_capturing():
                # Python may collect a cache at any time, so also while a graph is being recorded, which waiting for the
                # device would end: its memory is kept until the next cache is made or closed
                _unfinished.append((self.ctx, self.device, (self.pool, self.workspace)))
            else:
                self._torch.cuda.synchronize(self.device)
                binding.kvs_destroy(self.ctx)
            self.ctx = None
            self.pool = self.workspace = self._planes = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self) -> int:
        if self._raw_stream is not None:
            return self._raw_stream(self._index)
        return self._torch.cuda.current_stream(self.device).cuda_stream

    def append(self, layer, k=None, v=None, batch=None, n_new=None):
        """k, v: ``[batch][n_new][n_kv_heads][head_dim]`` contiguous device tensors (None on a sharing layer)."""
        if k is not None:
            assert k.is_contiguous() and v.is_contiguous() and k.dtype == self.dtype and v.dtype == self.dtype
            assert k.shape == v.shape and k.shape[2:] == (self.shape[2], self.shape[3])
            batch, n_new = k.shape[0], k.shape[1]
        binding.kvs_append(self.ctx, layer, k, v, batch, n_new, self._stream())

    def decode_attention(self, layer, q, out=None):
        """q: ``[batch][n_q_heads][head_dim]``; returns float32 ``[batch][n_q_heads][head_dim]``."""
        torch = self._torch
        assert q.is_contiguous() and q.dtype == self.dtype and q.shape[1:] == (self.shape[1], self.shape[3])
        if out is None:
            out = torch.empty(q.shape, dtype=torch.float32, device=self.device)
        binding.kvs_decode_attention(self.ctx, layer, q, out, q.shape[0], self._stream())
        return out

    def decode_step(self, layer, q, k=None, v=None, out=None):
        """Append one token's k, v (``[batch][1][n_kv_heads][head_dim]``; None on a sharing layer) and attend
        with q: ``append`` then ``decode_attention`` in one call, the append riding in the attention kernel."""
        torch = self._torch
        assert q.is_contiguous() and q.dtype == self.dtype and q.shape[1:] == (self.shape[1], self.shape[3])
        if k is not None:
            assert k.is_contiguous() and v.is_contiguous() and k.dtype == self.dtype and v.dtype == self.dtype
            assert k.shape == v.shape == (q.shape[0], 1, self.shape[2], self.shape[3])
        if out is None:
            out = torch.empty(q.shape, dtype=torch.float32, device=self.device)
        binding.kvs_decode_step(self.ctx, layer, q, k, v, out, q.shape[0], self._stream())
        return out

    def prefill_attention(self, layer, q, out=None):
        """q: ``[batch][n_q][n_q_heads][head_dim]`` (the newest n_q positions, causal); returns float32 of that shape."""
        torch = self._torch
        assert q.is_contiguous() and q.dtype == self.dtype and q.ndim == 4
        assert q.shape[2:] == (self.shape[1], self.shape[3])
        if out is None:
            out = torch.empty(q.shape, dtype=torch.float32, device=self.device)
        binding.kvs_prefill_attention(self.ctx, layer, q, out, q.shape[0], q.shape[1], self._stream())
        return out

    def evict(self, layer, keep, n_keep):
        """keep: device int32 ``[batch][Hkv][stride]`` ascending row lists; n_keep: ``[batch][Hkv]`` counts (host)."""
        assert keep.is_contiguous() and keep.dtype == self._torch.int32 and keep.ndim == 3
        counts = [int(x) for x in self._torch.as_tensor(n_keep).reshape(-1).tolist()]
        binding.kvs_evict(self.ctx, layer, keep, counts, keep.shape[2], keep.shape[0], self._stream())

    def _here(self, *tensors):
        """Whether the tensors (None: left out) live on the cache's device."""
        index = self._index
        for x in tensors:
            if x is not None and x.get_device() != index:
                return False
        return True

    def _token_stride(self, x, heads, batch, n_new):
        """Elements between consecutive tokens of ``[batch][n_new][heads][head_dim]`` (heads contiguous)."""
        D = self.shape[3]
        assert x.shape == (batch, n_new, heads, D) and x.dtype is self.dtype and x.get_device() == self._index
        sb, st, sh, sd = x.stride()
        assert sd == 1 and (sh == D or heads == 1), "a token's heads must be contiguous"
        if n_new == 1:
            return sb if batch > 1 else heads * D
        assert batch == 1 or sb == n_new * st, "tokens of all sequences must be evenly spaced"
        return st

    def append_rotary(self, layer, q, k, v, positions, rotary, q_weight=None, k_weight=None, eps=1e-6, out=None):
        """New tokens: per-head RMS norm (where a weight is given) and rotary positions of q and k, k and v appended
        to the layer's slot, the finished queries returned.  q, k, v: ``[batch][n_new][heads][head_dim]``, slices of
        one projection's output allowed (k, v: None on a sharing layer); positions: int32 ``[batch][n_new]``."""
        torch = self._torch
        batch, n_new = q.shape[0], q.shape[1]
        _, Hq, Hkv, D = self.shape
        qs = self._token_stride(q, Hq, batch, n_new)
        ks = vs = 0
        if k is not None:
            ks, vs = self._token_stride(k, Hkv, batch, n_new), self._token_stride(v, Hkv, batch, n_new)
        assert positions is None or (positions.dtype is torch.int32 and positions.is_contiguous() and
                                     positions.shape == q.shape[:2])
        for w in (q_weight, k_weight):
            assert w is None or (w.dtype is self.dtype and w.is_contiguous() and w.numel() == D)
        assert self._here(positions, q_weight, k_weight, out)
        if out is None:
            out = torch.empty((batch, n_new, Hq, D), dtype=self.dtype, device=self.device)
        else:
            assert out.is_contiguous() and out.dtype is self.dtype and out.shape == q.shape
        binding.kvs_append_rotary(self.ctx, layer, rotary._struct(eps), q, qs, k, ks, v, vs, positions, q_weight, k_weight, out,
                                  batch, n_new, self._stream())
        return out

    def tree_attention(self, layer, q, mask=None, out=None):
        """Attention of drafted tokens, the newest n_t rows of the cache.  q: ``[batch][n_t][n_q_heads][head_dim]``;
        mask: int64 ``[batch][n_t]``, bit j of a word: the token sees draft j (None: a chain).  Returns q's type."""
        torch = self._torch
        assert q.is_contiguous() and q.dtype == self.dtype and q.ndim == 4 and q.shape[2:] == (self.shape[1], self.shape[3])
        assert mask is None or (mask.dtype in (torch.int64, torch.uint64) and mask.is_contiguous() and mask.shape == q.shape[:2])
        assert self._here(q, mask, out)
        if out is None:
            out = torch.empty_like(q)
        else:
            assert out.is_contiguous() and out.dtype == self.dtype and out.shape == q.shape
        binding.kvs_tree_attention(self.ctx, layer, q, out, mask, q.shape[0], q.shape[1], self._stream())
        return out

    def accept_draft(self, path, n_accept, n_draft):
        """Keep the accepted drafts in every slot.  path: int32 ``[batch][stride]`` draft numbers, ascending; n_accept:
        how many of them each sequence keeps (host)."""
        assert path.dtype == self._torch.int32 and path.is_contiguous() and path.ndim == 2 and len(n_accept) == path.shape[0]
        assert self._here(path)
        binding.kvs_accept_draft(self.ctx, path, path.shape[1], [int(x) for x in n_accept], n_draft, path.shape[0], self._stream())

    def decode_attention_weights(self, layer, q, total_in, total_out=None, out=None):
        """``decode_attention`` that also returns, in ``total_out``, ``total_in`` (None: zeros) plus every row's softmax
        weight summed over its group of q-heads: float32 ``[batch][n_kv_heads][stride]``; without ``total_out`` the
        totals are updated in place."""
        torch = self._torch
        assert q.is_contiguous() and q.dtype == self.dtype and q.shape[1:] == (self.shape[1], self.shape[3])
        if total_out is None:
            total_out = total_in
        for x in (total_in, total_out):
            assert x is None or (x.dtype == torch.float32 and x.is_contiguous() and x.ndim == 3 and x.shape == total_out.shape)
        assert total_out.shape[:2] == (q.shape[0], self.shape[2]) and self._here(q, total_in, total_out, out)
        if out is None:
            out = torch.empty(q.shape, dtype=torch.float32, device=self.device)
        else:
            assert out.is_contiguous() and out.dtype == torch.float32 and out.shape == q.shape
        binding.kvs_decode_attention_weights(self.ctx, layer, q, out, total_in, total_out, total_out.shape[2], q.shape[0],
                                             self._stream())
        return out

    def select_rows(self, layer, total, n_keep, n_recent, keep=None, kept_total=None):
        """The rows a budget keeps: the newest n_recent and those with the largest totals.  total: float32
        ``[batch][n_kv_heads][stride]``; n_keep: ``[batch][n_kv_heads]`` counts (host).  Returns the keep list ``evict``
        takes, int32 ``[batch][n_kv_heads][max n_keep]``, and the rows' totals in the same layout."""
        torch = self._torch
        assert total.dtype == torch.float32 and total.is_contiguous() and total.ndim == 3 and total.shape[1] == self.shape[2]
        counts = torch.as_tensor(n_keep, dtype=torch.int32, device="cpu").contiguous()
        assert counts.numel() == total.shape[0] * total.shape[1]
        if keep is None:
            keep = torch.zeros(*total.shape[:2], int(counts.max()), dtype=torch.int32, device=self.device)
        if kept_total is None:
            kept_total = torch.zeros(keep.shape, dtype=torch.float32, device=self.device)
        assert keep.is_contiguous() and keep.dtype == torch.int32 and keep.shape[:2] == total.shape[:2]
        assert kept_total.is_contiguous() and kept_total.dtype == torch.float32 and kept_total.shape == keep.shape
        assert self._here(total, keep, kept_total)
        binding.kvs_select_rows(self.ctx, layer, total, total.shape[2], counts, n_recent, keep, kept_total, keep.shape[2],
                                total.shape[0], self._stream())
        return keep, kept_total

    def evict_by_weight(self, layer, total, n_keep, n_recent, stride=None):
        """``select_rows`` and ``evict`` in one: the layer's slot keeps n_keep rows per unit.  Returns their totals,
        zeros behind them up to ``stride`` entries per unit (None: the largest n_keep; the slot's capacity leaves room
        for rows appended later)."""
        keep = None
        if stride is not None:
            keep = self._torch.zeros(*total.shape[:2], stride, dtype=self._torch.int32, device=self.device)
        keep, kept = self.select_rows(layer, total, n_keep, n_recent, keep)
        self.evict(layer, keep, n_keep)
        return kept

    def read_rows(self, layer, first=0, n_rows=None, batch=None):
        """Rows of the slot the layer reads, as ``append`` takes them: k, v ``[batch][n_rows][n_kv_heads][head_dim]`` (of a
        4-bit cache: the values its rows stand for).  None: all rows, all cached sequences."""
        if n_rows is None:
            n_rows = self.seq_len(layer) - first
        if batch is None:
            batch = binding.kvs_cached_batch(self.ctx)
        shape = (batch, n_rows, self.shape[2], self.shape[3])
        k, v = (self._torch.empty(shape, dtype=self.dtype, device=self.device) for _ in range(2))
        binding.kvs_read_rows(self.ctx, layer, first, n_rows, k, v, batch, self._stream())
        return k, v

    def beam_select(self, logits, scores, n_beams, n_out, out=None):
        """The n_out best continuations of every request's n_beams beams.  logits: bf16 or float32 ``[rows][vocab]`` (rows may be
        strided), rows = requests * n_beams; scores: float32 of as many elements, the beams' log-probabilities so far.  Returns
        (or fills ``out``) scores float32, tokens int32 and parents int32 (sequence numbers, as ``reorder`` takes them), each
        ``[requests][n_out]``, best first."""
        torch = self._torch
        assert logits.ndim == 2 and logits.dtype in (torch.bfloat16, torch.float32)
        rows, vocab = logits.shape
        assert n_beams >= 1 and rows % n_beams == 0 and (vocab == 1 or logits.stride(1) == 1), "a row's logits must be contiguous"
        assert scores.dtype == torch.float32 and scores.is_contiguous() and scores.numel() == rows and self._here(logits, scores)
        shape = (rows // n_beams, n_out)
        if out is None:
            out = scores.new_empty(shape), scores.new_empty(shape, dtype=torch.int32), scores.new_empty(shape, dtype=torch.int32)
        else:
            for x, d in zip(out, (torch.float32, torch.int32, torch.int32)):
                assert x.dtype == d and x.is_contiguous() and x.shape == shape and self._here(x)
        binding.kvs_beam_select(self.ctx, logits, KVS_BF16 if logits.dtype == torch.bfloat16 else KVS_F32,
                                logits.stride(0) if rows > 1 else vocab, vocab, scores, shape[0], n_beams, n_out, *out, self._stream())
        return out

    def reorder(self, parent, first_row=0):
        """Every sequence b of every slot becomes what sequence ``parent[b]`` was, rows first_row and on.  parent: device int32
        ``[batch]``; the batch may grow (fork) or shrink (compaction)."""
        assert parent.dtype == self._torch.int32 and parent.is_contiguous() and parent.ndim == 1 and self._here(parent)
        binding.kvs_reorder(self.ctx, parent, first_row, parent.shape[0], self._stream())

    def unit_len(self, layer, b, h):
        return binding.kvs_unit_len(self.ctx, layer, b, h)

    def layer_distances(self, batch=None):
        """float32 ``[L][L]`` distances between the layers' sample-mean K/V representations."""
        torch = self._torch
        L = self.shape[0]
        dist = torch.empty(L, L, dtype=torch.float32, device=self.device)
        if batch is None:
            batch = self._cached_batch()
        binding.kvs_layer_distances(self.ctx, batch, dist, self._stream())
        return dist

    def _cached_batch(self):
        b = 0
        while b < self.max_batch and self.unit_len(0, b, 0) > 0:
            b += 1
        return b

    def mean_cosine(self, a, b):
        """cos(mean over samples of a, mean over samples of b) for ``[S][dim]`` device tensors (float32 scalar tensor)."""
        torch = self._torch
        assert a.shape == b.shape and a.ndim == 2 and a.is_contiguous() and b.is_contiguous() and a.dtype == self.dtype
        out = torch.empty(1, dtype=torch.float32, device=self.device)
        binding.kvs_mean_cosine(self.ctx, a, b, a.shape[0], a.shape[1], out, self._stream())
        return out

    def replay_advance(self):
        binding.kvs_replay_advance(self.ctx, self._stream())

    def replay_commit(self, times_run):
        binding.kvs_replay_commit(self.ctx, times_run, self._stream())

    def step_host(self, q_host, k_host, v_host, out_host):
        """One decode step over all layers from host tensors (see ``kvs_step_host``)."""
        return binding.kvs_step_host(self.ctx, q_host, k_host, v_host, out_host, q_host.shape[1], self._stream())

    def plane(self, slot, kv):
        """View of plane (slot, kv) as ``[max_batch][n_kv_heads][row_stride][head_dim]`` (of a 4-bit cache: its bytes,
        ``[max_batch][n_kv_heads][row_stride][16 + head_dim / 2]``)."""
        if self._planes is None or self._planes[0] is not self.pool:
            self._planes = self.pool, {}
        seen = self._planes[1].get((slot, kv))
        if seen is None:
            off, nbytes = binding.kvs_plane_offset(self.ctx, slot, kv), binding.kvs_plane_offset(self.ctx, 0, 1)
            rs = binding.kvs_row_stride(self.ctx)
            plane = self.pool[off:off + nbytes]
            if self.cache_format == KVS_CACHE_PLAIN:
                plane = plane.view(self.dtype)
            seen = plane.view(self.max_batch, self.shape[2], rs, -1)
            self._planes[1][slot, kv] = seen
        return seen.detach()        # a tensor of its own for every caller

    # plain forwards
    def num_slots(self):
        return binding.kvs_num_slots(self.ctx)

    def slot_of_layer(self, layer):
        return binding.kvs_slot_of_layer(self.ctx, layer)

    def seq_len(self, layer):
        return binding.kvs_seq_len(self.ctx, layer)

    def reset(self):
        binding.kvs_reset(self.ctx)

    def truncate(self, n_tokens):
        """Cut every slot back to at most ``n_tokens`` rows (host bookkeeping only)."""
        binding.kvs_truncate(self.ctx, n_tokens)

    def clear_device_status(self):
        binding.kvs_clear_device_status(self.ctx, self._stream())

    def selftest_wait_timeout(self, limit_us=1000):
        """Make one bounded device-side wait run out; returns the nanoseconds it lasted."""
        return binding.kvs_selftest_wait_timeout(self.ctx, limit_us, self._stream())

    def stats(self):
        return binding.kvs_stats(self.ctx)

    def device_status(self):
        return binding.kvs_last_device_status(self.ctx)

    def set_option(self, option, value):
        binding.kvs_set_option(self.ctx, option, value)

    def last_launch(self):
        return binding.kvs_last_launch(self.ctx)
