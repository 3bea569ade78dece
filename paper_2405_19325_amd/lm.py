"""The language model's own step around the mixture: cache append, attention of drafts, sampling.

Like the rest of the package this only marshals arguments; the HIP kernels
behind include/knnlm.h do the work.  Each class keeps the buffers, the planning
hints and the workspace of repeated calls; run() takes the tensors' contents as
they are when the stream gets there, so it can be captured into a graph and
replayed on new ones.  The function of each is a one-shot call.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence, Tuple

import torch

from . import _lib
from . import _dtype_code, _need, _ptr, _stream
from ._lib import load


def _on_device(first: torch.Tensor, **named: Optional[torch.Tensor]) -> int:
    """Checks that the tensors given are on the current GPU (that of `first`) and returns its index."""
    _need(first.is_cuda, "device tensors are needed")
    for name, t in named.items():
        if t is not None:
            _need(t.is_cuda and t.device == first.device, f"{name} must be on {first.device}")
    index = first.device.index
    _need(index == torch.cuda.current_device(), f"the tensors are on {first.device}, which is not the current device")
    return index


def _flat(name: str, t: Optional[torch.Tensor], dtype: torch.dtype, shape: Tuple[int, ...]):
    if t is not None:
        _need(t.dtype == dtype and tuple(t.shape) == shape and t.is_contiguous(),
              f"{name}: contiguous {list(shape)} {dtype} tensor")


class _Call:
    """A call that is made again and again on one GPU, with the same buffers where they are.  Its runs share their
    outputs and workspace, so they follow each other on one stream or wait for each other.  A stream that it runs on for
    the first time waits for the one that was current when it was made: what that one still does may be with the memory
    that the outputs and the workspace were given.  A graph that captured one replays on its buffers: keep the object as
    long as the graph."""

    def _keep(self, index: int, name: str, args: Sequence, tensors: Sequence, own: Sequence[torch.Tensor]):
        """`name`: the library's function; `args`: its arguments but the stream, converted once; `tensors`: what they
        point to; `own`: those of them that this object allocated."""
        fn = getattr(load(), name)
        self._name, self._fn = name, fn
        self._args = tuple(a if a is None else kind(a) for kind, a in zip(fn.argtypes, args))
        self._index, self._tensors, self._own = index, tuple(tensors), tuple(own)
        self._home = _stream(None)
        self._known = {self._home}

    def _call(self, stream):
        if torch.cuda.current_device() != self._index:
            raise ValueError(f"made for cuda:{self._index}, which is not the current device")
        h = _stream(stream)
        if h not in self._known:  # the allocator has to know who else uses what this object allocated
            if not torch.cuda.is_current_stream_capturing():
                s, home = (torch.cuda.ExternalStream(i) if i else torch.cuda.default_stream() for i in (h, self._home))
                if self._own:
                    s.wait_stream(home)
                for t in self._own:
                    t.record_stream(s)
                self._known.add(h)
        st = self._fn(*self._args, h)
        if st != _lib.KNN_OK:
            _lib.check(self._name, st)


def _paged(k_cache: torch.Tensor, v_cache: torch.Tensor, pages: torch.Tensor, row_offsets: torch.Tensor,
           cache_lens: torch.Tensor) -> Tuple[int, int, int, int, int]:
    """Checks the cache's tensors: (S, n_pages, kv_heads, page_size, head_dim)."""
    _need(k_cache.dim() == 4 and k_cache.is_contiguous(),
          "k_cache: contiguous [n_pages, kv_heads, page_size, head_dim]")
    _flat("v_cache", v_cache, k_cache.dtype, tuple(k_cache.shape))
    _need(pages.dim() == 2, "pages: [S, table_width]")
    _flat("pages", pages, torch.int32, tuple(pages.shape))
    S = pages.shape[0]
    _flat("row_offsets", row_offsets, torch.int64, (S + 1,))
    _flat("cache_lens", cache_lens, torch.int32, (S,))
    n_pages, kv_heads, page_size, d = k_cache.shape
    return S, n_pages, kv_heads, page_size, d


class KVAppend(_Call):
    """knn_kv_append on these buffers: the rows' keys and values into the paged cache, keys and queries rotated.

    k, v [source rows, kv_heads, d] and q [source rows, q_heads, d] (bf16 or f16) may be views with any row and head
    stride, such as the parts of one projection's output; k_cache, v_cache [n_pages, kv_heads, page_size, d]; pages
    [S, width] int32, row_offsets [S+1] int64, cache_lens [S] int32 as the header says.  positions [rows] int32
    (default: the cache index); inv_freq [rotated elements / 2] fp32 (None: no rotation); interleaved: pairs
    (2i, 2i+1); source_rows [rows] int32: the row that each row is read from.  q_out [rows, q_heads, d] is
    allocated where it is not given (it may be q where q is dense and there are no source_rows).  What is read lies
    apart from the caches.
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                 pages: torch.Tensor, row_offsets: torch.Tensor, cache_lens: torch.Tensor,
                 q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 positions: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None,
                 interleaved: bool = False, source_rows: Optional[torch.Tensor] = None):
        index = _on_device(k, v=v, k_cache=k_cache, v_cache=v_cache, pages=pages, row_offsets=row_offsets,
                           cache_lens=cache_lens, q=q, q_out=q_out, positions=positions, inv_freq=inv_freq,
                           source_rows=source_rows)
        S, n_pages, kv_heads, page_size, d = _paged(k_cache, v_cache, pages, row_offsets, cache_lens)
        source = k.shape[0]
        for name, t in (("k", k), ("v", v)):
            _need(t.dim() == 3 and t.dtype == k_cache.dtype and tuple(t.shape) == (source, kv_heads, d) and
                  t.stride(2) == 1, f"{name}: [rows, {kv_heads}, {d}] {k_cache.dtype} with dense heads")
        rows = source if source_rows is None else source_rows.numel()
        _flat("source_rows", source_rows, torch.int32, (rows,))
        _flat("positions", positions, torch.int32, (rows,))
        q_heads, own = 0, ()
        if q is not None:
            _need(q.dim() == 3 and q.dtype == k.dtype and q.shape[0] == source and q.shape[2] == d and
                  q.stride(2) == 1, f"q: [{source}, q_heads, {d}] {k.dtype} with dense heads")
            q_heads = q.shape[1]
            if q_out is None:
                q_out = torch.empty((rows, q_heads, d), dtype=q.dtype, device=q.device)
                own = (q_out,)
            _flat("q_out", q_out, q.dtype, (rows, q_heads, d))
        else:
            _need(q_out is None, "q_out without q")
        half = 0
        if inv_freq is not None:
            half = inv_freq.numel()
            _flat("inv_freq", inv_freq, torch.float32, (half,))
        self.q_out = q_out
        tensors = (q, k, v, row_offsets, cache_lens, pages, positions, inv_freq, source_rows)
        strides = [t.stride(i) if t is not None else 0 for t in (q, k, v) for i in (0, 1)]
        args = (*map(_ptr, tensors), rows, source, S, q_heads, kv_heads, d, 2 * half, int(bool(interleaved)), *strides,
                n_pages, page_size, pages.shape[1], _dtype_code(k), *map(_ptr, (q_out, k_cache, v_cache)))
        self._keep(index, "knn_kv_append", args, (*tensors, q_out, k_cache, v_cache), own)

    def run(self, stream=None) -> Optional[torch.Tensor]:
        """One call; returns q_out (the rotated queries), valid after stream sync."""
        self._call(stream)
        return self.q_out


def kv_append(k, v, k_cache, v_cache, pages, row_offsets, cache_lens, q=None, q_out=None, positions=None,
              inv_freq=None, interleaved=False, source_rows=None, stream=None):
    """One-shot knn_kv_append: writes the caches and returns the rotated queries (None without q)."""
    return KVAppend(k, v, k_cache, v_cache, pages, row_offsets, cache_lens, q, q_out, positions, inv_freq,
                    interleaved, source_rows).run(stream)


def tree_words(parents: Sequence[int], device) -> torch.Tensor:
    """The masks of one sequence's rows as knn_tree_attention reads them, [rows, words] int32: every row sees itself
    and its ancestors, parents[i] < i being the row that row i hangs under (-1: none)."""
    n = len(parents)
    words = torch.zeros((n, (n + 31) // 32), dtype=torch.int64)
    for i, p in enumerate(parents):
        _need(-1 <= p < i, "parents: each row's parent comes before it")
        if p >= 0:
            words[i] = words[p]
        words[i, i // 32] |= 1 << (i % 32)
    return (words - ((words >> 31) << 32)).to(torch.int32).to(device)


class TreeAttention(_Call):
    """knn_tree_attention on these buffers: rows of drafts over the paged cache.

    q [rows, q_heads, d] (bf16 or f16; any row and head stride that is a multiple of 8), the cache's tensors as in
    KVAppend.  max_rows and max_keys bound the rows of a sequence and its tokens with them, in every run; where they are
    not given they are what can be at all: all rows (and bits of a mask's row) and the table's room.  Bounds near the
    truth are faster, since they decide how the work is split.  tree_mask [rows, words] int32 (see tree_words) or None
    for chains.  out and lse ([rows, q_heads] fp32; only with want_lse) are allocated where they are not given.
    """

    def __init__(self, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, pages: torch.Tensor,
                 row_offsets: torch.Tensor, cache_lens: torch.Tensor, max_rows: Optional[int] = None,
                 max_keys: Optional[int] = None, tree_mask: Optional[torch.Tensor] = None,
                 scale: Optional[float] = None, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                 want_lse: bool = False):
        index = _on_device(q, k_cache=k_cache, v_cache=v_cache, pages=pages, row_offsets=row_offsets,
                           cache_lens=cache_lens, tree_mask=tree_mask, out=out, lse=lse)
        S, n_pages, kv_heads, page_size, d = _paged(k_cache, v_cache, pages, row_offsets, cache_lens)
        _need(q.dim() == 3 and q.dtype == k_cache.dtype and q.shape[2] == d and q.stride(2) == 1,
              f"q: [rows, q_heads, {d}] {k_cache.dtype} with dense heads")
        rows, q_heads = q.shape[0], q.shape[1]
        words = 0
        if tree_mask is not None:
            _need(tree_mask.dim() == 2, "tree_mask: [rows, words]")
            words = tree_mask.shape[1]
            _flat("tree_mask", tree_mask, torch.int32, (rows, words))
        if max_rows is None:
            max_rows = rows if tree_mask is None else min(rows, 32 * words)
            _need(max_rows <= 65535, "max_rows: to be given for more than 65535 rows (a sequence has that many at most)")
        if max_keys is None:
            max_keys = min(pages.shape[1] * page_size, 2 ** 31 - 1)
        own = []
        if out is None:
            out = torch.empty((rows, q_heads, d), dtype=q.dtype, device=q.device)
            own.append(out)
        if lse is None and want_lse:
            lse = torch.empty((rows, q_heads), dtype=torch.float32, device=q.device)
            own.append(lse)
        _flat("out", out, q.dtype, (rows, q_heads, d))
        _flat("lse", lse, torch.float32, (rows, q_heads))
        self.out, self.lse = out, lse
        need = load().knn_tree_attention_workspace_size(rows, S, q_heads, kv_heads, d, int(max_rows), int(max_keys))
        self.workspace = torch.empty(max(int(need), 256), dtype=torch.uint8, device=q.device)
        own.append(self.workspace)
        tensors = (q, k_cache, v_cache, pages, row_offsets, cache_lens, tree_mask)
        args = (*map(_ptr, tensors), rows, S, q_heads, kv_heads, d, q.stride(0), q.stride(1), n_pages, page_size,
                pages.shape[1], words, int(max_rows), int(max_keys), _dtype_code(q),
                float(1.0 / math.sqrt(d) if scale is None else scale), _ptr(out), _ptr(lse), _ptr(self.workspace),
                self.workspace.numel())
        self._keep(index, "knn_tree_attention", args, (*tensors, out, lse), own)

    def run(self, stream=None) -> torch.Tensor:
        """One call; returns out (and fills lse, where there is one), valid after stream sync."""
        self._call(stream)
        return self.out


def tree_attention(q, k_cache, v_cache, pages, row_offsets, cache_lens, max_rows=None, max_keys=None, tree_mask=None,
                   scale=None, out=None, lse=None, want_lse=False, stream=None):
    """One-shot knn_tree_attention: out, or (out, lse) with an lse.  max_rows and max_keys that are not given come from the
    tensors' present contents, which are copied to the host for that."""
    if max_rows is None or max_keys is None:
        _flat("row_offsets", row_offsets, torch.int64, (pages.shape[0] + 1,))
        _flat("cache_lens", cache_lens, torch.int32, (pages.shape[0],))
        count = row_offsets.diff()
        if max_rows is None:
            max_rows = max(1, int(count.max()))
        if max_keys is None:
            max_keys = max(1, int((cache_lens + count).max()))
    call = TreeAttention(q, k_cache, v_cache, pages, row_offsets, cache_lens, max_rows, max_keys, tree_mask, scale, out,
                         lse, want_lse)
    call.run(stream)
    return call.out if call.lse is None else (call.out, call.lse)


class Sampler(_Call):
    """knn_sample on these buffers: a token of each row of scores [rows, V] (f32, bf16 or f16, dense rows).

    scores are logits, or a distribution with probabilities=True (p_m of a MixtureProblem, say); uniforms [rows] fp32.
    temperature, top_p, min_p [rows] fp32 and top_k [rows] int32, or None: 1, 1, 0 and 0 (off).
    """

    def __init__(self, scores: torch.Tensor, uniforms: torch.Tensor, probabilities: bool = False,
                 temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
                 top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None):
        index = _on_device(scores, uniforms=uniforms, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
        _need(scores.dim() == 2 and (scores.stride(1) == 1 or scores.shape[1] == 1),
              "scores: [rows, V] with dense rows")
        rows, V = scores.shape
        for name, t, dtype in (("uniforms", uniforms, torch.float32), ("temperature", temperature, torch.float32),
                               ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                               ("min_p", min_p, torch.float32)):
            _flat(name, t, dtype, (rows,))
        dev = scores.device
        self.token = torch.empty(rows, dtype=torch.int32, device=dev)
        self.prob = torch.empty(rows, dtype=torch.float32, device=dev)
        self.kept = torch.empty(rows, dtype=torch.int32, device=dev)
        code = _dtype_code(scores)
        need = load().knn_sample_workspace_size(rows, V, code)
        self.workspace = torch.empty(max(int(need), 256), dtype=torch.uint8, device=dev)
        tensors = (scores, uniforms, temperature, top_k, top_p, min_p)
        own = (self.token, self.prob, self.kept, self.workspace)
        args = (*map(_ptr, tensors), rows, V, scores.stride(0), int(bool(probabilities)), code, *map(_ptr, own),
                self.workspace.numel())
        self._keep(index, "knn_sample", args, tensors, own)

    def run(self, stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """One call; returns (token, its probability among those kept, how many were kept), valid after stream sync."""
        self._call(stream)
        return self.token, self.prob, self.kept


def sample(scores, uniforms, probabilities=False, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
    """One-shot knn_sample: (token [rows], its probability among those kept, how many were kept)."""
    return Sampler(scores, uniforms, probabilities, temperature, top_k, top_p, min_p).run(stream)
