"""The operators of a decoder step around the multiply (include/biq.h, its last part): rotary positions, the paged 8-bit
cache, attention over it, verification of drafted tokens.

Each comes as a function and as a class whose objects are the call with its arguments converted once, for programs that keep
their buffers (calling the object only crosses the C ABI).  Tensors give their own sizes, types and strides.  A prepared call
uses the stream that it is given or torch's current one at preparation; its tensors must stay alive and in place (it keeps
references to them).

Ragged calls take starts (int32 [seqs + 1]) and max_rows, the most rows that a sequence has.  Left open, max_rows is all rows: right,
but single tokens then run as prompts do.

Checked here is what the C functions cannot see of tensors: their number of dimensions, sizes that have to agree, types, devices.
"""
from __future__ import annotations

import ctypes
import math

from . import binding

FORMATS = {"int8": 0, "fp8": 1}
SCALINGS = {"plain": 0, "linear": 1, "base": 2, "by_parts": 3}
I, P, L = ctypes.c_int, ctypes.c_void_p, ctypes.c_int64


class _Rows(ctypes.Structure):
    _fields_ = [("data", P), ("row_stride", L), ("head_stride", L)]


class _Rotation(ctypes.Structure):
    _fields_ = [("angles", P), ("positions", I), ("rot", I), ("interleaved", I)]


class _Cache(ctypes.Structure):
    _fields_ = [("store", P), ("table", P), ("lens", P), ("num_pages", I), ("page_tokens", I), ("table_stride", I), ("seqs", I),
                ("heads", I), ("head_dim", I), ("format", I)]


class _Ragged(ctypes.Structure):
    _fields_ = [("starts", P), ("rows", I), ("max_rows", I)]


class _RotaryArgs(ctypes.Structure):
    _fields_ = [("x", _Rows), ("y", _Rows), ("positions", P), ("rotation", _Rotation), ("type", I), ("rows", I), ("heads", I),
                ("head_dim", I), ("inverse", I)]


class _AppendArgs(ctypes.Structure):
    _fields_ = [("cache", _Cache), ("k", _Rows), ("v", _Rows), ("ragged", _Ragged), ("rotation", _Rotation), ("type", I)]


class _ReadArgs(ctypes.Structure):
    _fields_ = [("cache", _Cache), ("k", _Rows), ("v", _Rows), ("ragged", _Ragged), ("type", I)]


class _AttentionArgs(ctypes.Structure):
    _fields_ = [("cache", _Cache), ("q", _Rows), ("out", _Rows), ("lse", P), ("ragged", _Ragged), ("type", I), ("q_heads", I),
                ("max_len", I), ("causal", I), ("window", I), ("scale", ctypes.c_float)]


class _SharedArgs(ctypes.Structure):
    _fields_ = [("attention", _AttentionArgs), ("shared", I)]


class _VerifyArgs(ctypes.Structure):
    _fields_ = [("p", P), ("q", P), ("p_seq_stride", L), ("p_stride", L), ("q_seq_stride", L), ("q_stride", L),
                ("draft_tokens", P), ("draft_lens", P), ("uniform", P), ("tokens", P), ("accepted", P), ("type", I), ("seqs", I),
                ("drafts", I), ("vocab", I)]


# ---- what tensors have to be -----------------------------------------------------------------------------

_types = None


def _type(t) -> int:
    global _types
    if _types is None:
        import torch

        _types = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    if t.dtype not in _types:
        raise ValueError("float32, bfloat16 or float16 expected, not %s" % t.dtype)
    return _types[t.dtype]


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _rows(t, name, like=None, heads=None, dim=None, rows=None) -> _Rows:
    """[rows][heads][dim] with adjacent elements."""
    _need(t.dim() == 3, "%s: [rows, heads, head_dim] expected" % name)
    _need(t.shape[2] <= 1 or t.stride(2) == 1, "%s: the elements of a head have to be adjacent" % name)
    _need(heads is None or t.shape[1] == heads, "%s: %s heads expected" % (name, heads))
    _need(dim is None or t.shape[2] == dim, "%s: heads of %s expected" % (name, dim))
    _need(rows is None or t.shape[0] == rows, "%s: %s rows expected" % (name, rows))
    _need(like is None or (t.dtype == like.dtype and t.device == like.device), "%s: another type or device" % name)
    return _Rows(t.data_ptr(), t.stride(0), t.stride(1))


def _whole(t, name, dtype, shape, device):
    """A dense tensor of that type and shape on that device."""
    _need(str(t.dtype) == "torch." + dtype and tuple(t.shape) == tuple(shape) and t.is_contiguous() and t.device == device,
          "%s: dense %s %s on %s expected" % (name, dtype, list(shape), device))
    return t.data_ptr()


def _rotation(angles, interleaved, device) -> _Rotation:
    if angles is None:
        return _Rotation(None, 0, 0, 0)
    _need(angles.dim() == 3 and angles.shape[2] == 2, "angles: [positions, rot / 2, 2] expected")
    return _Rotation(_whole(angles, "angles", "float32", angles.shape, device), angles.shape[0], 2 * angles.shape[1], int(bool(interleaved)))


def _ragged(starts, max_rows, rows, cache) -> _Ragged:
    if starts is None:
        each = rows // cache.seqs
        _need(rows == each * cache.seqs, "rows are no multiple of the sequences: starts expected")
        _need(max_rows is None or max_rows == each, "max_rows: %d rows a sequence without starts" % each)
        return _Ragged(None, rows, each)
    return _Ragged(_whole(starts, "starts", "int32", [cache.seqs + 1], cache.store.device), rows,
                   min(rows, rows if max_rows is None else max_rows))


class _Prepared:
    """A call with its descriptor built once."""

    def __init__(self, name, args, keep, workspace=None, takes_workspace=False, device=None, stream=None):
        _need(workspace is None or (workspace.is_contiguous() and workspace.device == device), "workspace: dense memory on %s expected" % device)
        lib = binding.load_library()
        from ._calls import Operation

        self._keep, self._args = (keep, workspace), args
        space = None
        if takes_workspace:
            space = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
        self._call = Operation(ctypes.cast(getattr(lib, name), P).value, name, ctypes.addressof(args), space, binding._check,
                               binding._stream(stream) or 0)

    def __call__(self) -> None:
        self._call()


# ---- rotary positions --------------------------------------------------------------------------------------

def biq_rotary_frequencies(rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, trained: int = 1,
                           slow: float = 1.0, fast: float = 32.0):
    """Turns per position of every pair, a float64 tensor on the host."""
    import torch

    _need(scaling in SCALINGS, "scaling: one of %s" % ", ".join(SCALINGS))
    turns = torch.empty(max(rot // 2, 1), dtype=torch.float64)
    binding._check(binding.load_library().biq_rotary_frequencies(turns.data_ptr(), rot, base, SCALINGS[scaling], factor, trained,
                                                                 slow, fast), "biq_rotary_frequencies")
    return turns


def biq_rotary_table(turns, angles, first: int = 0, amplitude: float = 1.0, stream=None) -> None:
    """angles [positions, rot / 2, 2] = amplitude (cos, sin) of the positions from `first` on; turns float64 [rot / 2]."""
    _need(angles.dim() == 3 and angles.shape[2] == 2, "angles: [positions, rot / 2, 2] expected")
    lib = binding.load_library()
    binding._check(lib.biq_rotary_table(_whole(turns, "turns", "float64", [angles.shape[1]], angles.device),
                                        _whole(angles, "angles", "float32", angles.shape, angles.device), 2 * angles.shape[1], first,
                                        angles.shape[0], amplitude, binding._stream(stream)), "biq_rotary_table")


class PreparedRotary(_Prepared):
    """biq_rotary: y = x turned by the angles of positions (int32 [rows]); inverse: the gradient.  y may be x."""

    def __init__(self, x, y, positions, angles, interleaved=False, inverse=False, stream=None):
        a = _RotaryArgs(x=_rows(x, "x"), y=_rows(y, "y", x, x.shape[1], x.shape[2], x.shape[0]),
                        positions=_whole(positions, "positions", "int32", [x.shape[0]], x.device),
                        rotation=_rotation(angles, interleaved, x.device), type=_type(x), rows=x.shape[0], heads=x.shape[1],
                        head_dim=x.shape[2], inverse=int(bool(inverse)))
        super().__init__("biq_rotary", a, (x, y, positions, angles), stream=stream)


def biq_rotary(x, y, positions, angles, interleaved=False, inverse=False, stream=None) -> None:
    PreparedRotary(x, y, positions, angles, interleaved, inverse, stream)()


# ---- the cache ---------------------------------------------------------------------------------------------

def biq_cache_page_bytes(page_tokens: int, heads: int, head_dim: int) -> int:
    return binding.load_library().biq_cache_page_bytes(page_tokens, heads, head_dim)


class KvCache:
    """A paged 8-bit cache on given buffers: store uint8 [pages, biq_cache_page_bytes], table int32 [seqs, width] of page numbers, lens
    int32 [seqs] (with the rows of the call that uses them).  format: "int8" or "fp8"."""

    def __init__(self, store, table, lens, page_tokens: int, heads: int, head_dim: int, format: str = "int8"):
        _need(format in FORMATS, "format: int8 or fp8")
        page = biq_cache_page_bytes(page_tokens, heads, head_dim)
        _need(page > 0, "page_tokens and head_dim: multiples of 16 up to 256")
        _need(store.dim() == 2 and store.shape[1] == page, "store: pages of %d bytes expected" % page)
        _need(table.dim() == 2 and table.numel() > 0, "table: [seqs, pages of a sequence] expected")
        self.store, self.table, self.lens = store, table, lens
        self.seqs, self.page_tokens, self.heads, self.head_dim, self.format = table.shape[0], page_tokens, heads, head_dim, format
        self._c = _Cache(_whole(store, "store", "uint8", store.shape, store.device),
                         _whole(table, "table", "int32", table.shape, store.device),
                         _whole(lens, "lens", "int32", [table.shape[0]], store.device), store.shape[0], page_tokens, table.shape[1],
                         table.shape[0], heads, head_dim, FORMATS[format])


class PreparedAppend(_Prepared):
    """biq_cache_append: k and v [rows, heads, head_dim] become the last tokens of their sequences; angles: keys are turned."""

    def __init__(self, cache, k, v, starts=None, max_rows=None, angles=None, interleaved=False, stream=None):
        _need(k.device == cache.store.device, "k: another device than the cache's")
        a = _AppendArgs(cache=cache._c, k=_rows(k, "k", None, cache.heads, cache.head_dim),
                        v=_rows(v, "v", k, cache.heads, cache.head_dim, k.shape[0]),
                        ragged=_ragged(starts, max_rows, k.shape[0], cache), rotation=_rotation(angles, interleaved, k.device), type=_type(k))
        super().__init__("biq_cache_append", a, (cache, k, v, starts, angles), stream=stream)


def biq_cache_append(cache, k, v, starts=None, max_rows=None, angles=None, interleaved=False, stream=None) -> None:
    PreparedAppend(cache, k, v, starts, max_rows, angles, interleaved, stream)()


class PreparedRead(_Prepared):
    """biq_cache_read: the last tokens of every sequence into k and v [rows, heads, head_dim]."""

    def __init__(self, cache, k, v, starts=None, max_rows=None, stream=None):
        _need(k.device == cache.store.device, "k: another device than the cache's")
        a = _ReadArgs(cache=cache._c, k=_rows(k, "k", None, cache.heads, cache.head_dim),
                      v=_rows(v, "v", k, cache.heads, cache.head_dim, k.shape[0]),
                      ragged=_ragged(starts, max_rows, k.shape[0], cache), type=_type(k))
        super().__init__("biq_cache_read", a, (cache, k, v, starts), stream=stream)


def biq_cache_read(cache, k, v, starts=None, max_rows=None, stream=None) -> None:
    PreparedRead(cache, k, v, starts, max_rows, stream)()


# ---- attention -----------------------------------------------------------------------------------------------

def _attention_args(cache, q, scale, starts, max_rows, max_len, causal, window):
    _need(q.device == cache.store.device, "q: another device than the cache's")
    rows = _rows(q, "q", None, None, cache.head_dim)
    return _AttentionArgs(cache=cache._c, q=rows, ragged=_ragged(starts, max_rows, q.shape[0], cache), type=_type(q), q_heads=q.shape[1],
                          max_len=max_len, causal=int(bool(causal)), window=window,
                          scale=1.0 / math.sqrt(cache.head_dim) if scale is None else scale)


def biq_attention_workspace_bytes(cache, q, scale=None, starts=None, max_rows=None, max_len=0, causal=True, window=0) -> int:
    """Bytes for PreparedAttention / biq_attention with the same arguments."""
    a = _attention_args(cache, q, scale, starts, max_rows, max_len, causal, window)
    return binding.load_library().biq_attention_workspace_bytes(ctypes.addressof(a))


class PreparedAttention(_Prepared):
    """biq_attention: q, out [rows, q_heads, head_dim], lse float32 [rows, q_heads] or None; scale None: 1 / sqrt(head_dim)."""

    def __init__(self, cache, q, out, lse=None, scale=None, starts=None, max_rows=None, max_len=0, causal=True, window=0,
                 workspace=None, stream=None):
        a = _attention_args(cache, q, scale, starts, max_rows, max_len, causal, window)
        a.out = _rows(out, "out", q, q.shape[1], q.shape[2], q.shape[0])
        a.lse = None if lse is None else _whole(lse, "lse", "float32", q.shape[:2], q.device)
        super().__init__("biq_attention", a, (cache, q, out, lse, starts), workspace, True, q.device, stream)


def biq_attention(cache, q, out, lse=None, scale=None, starts=None, max_rows=None, max_len=0, causal=True, window=0,
                  workspace=None, stream=None) -> None:
    PreparedAttention(cache, q, out, lse, scale, starts, max_rows, max_len, causal, window, workspace, stream)()


def biq_attention_shared_workspace_bytes(cache, q, shared, scale=None, starts=None, max_rows=None, max_len=0, causal=True, window=0) -> int:
    """Bytes for PreparedSharedAttention / biq_attention_shared with the same arguments."""
    a = _SharedArgs(_attention_args(cache, q, scale, starts, max_rows, max_len, causal, window), shared)
    return binding.load_library().biq_attention_shared_workspace_bytes(ctypes.addressof(a))


class PreparedSharedAttention(_Prepared):
    """biq_attention_shared: as PreparedAttention, where the first `shared` tokens of all sequences are those of the cache's sequence 0."""

    def __init__(self, cache, q, out, shared, lse=None, scale=None, starts=None, max_rows=None, max_len=0, causal=True, window=0,
                 workspace=None, stream=None):
        a = _SharedArgs(_attention_args(cache, q, scale, starts, max_rows, max_len, causal, window), shared)
        a.attention.out = _rows(out, "out", q, q.shape[1], q.shape[2], q.shape[0])
        a.attention.lse = None if lse is None else _whole(lse, "lse", "float32", q.shape[:2], q.device)
        super().__init__("biq_attention_shared", a, (cache, q, out, lse, starts), workspace, True, q.device, stream)


def biq_attention_shared(cache, q, out, shared, lse=None, scale=None, starts=None, max_rows=None, max_len=0, causal=True, window=0,
                         workspace=None, stream=None) -> None:
    PreparedSharedAttention(cache, q, out, shared, lse, scale, starts, max_rows, max_len, causal, window, workspace, stream)()


# ---- drafted tokens ----------------------------------------------------------------------------------------

def biq_verify_workspace_bytes(seqs: int, vocab: int) -> int:
    return binding.load_library().biq_verify_workspace_bytes(seqs, vocab)


class PreparedVerify(_Prepared):
    """biq_verify_drafts: p [seqs, drafts + 1, vocab], q [seqs, drafts, vocab] or None, draft_tokens int32 [seqs, drafts], uniform float32
    [seqs, drafts + 1] -> tokens int32 [seqs, drafts + 1], accepted int32 [seqs]."""

    def __init__(self, p, q, draft_tokens, uniform, tokens, accepted, draft_lens=None, workspace=None, stream=None):
        _need(p.dim() == 3 and (p.shape[2] <= 1 or p.stride(2) == 1), "p: [seqs, drafts + 1, vocab] with adjacent tokens expected")
        seqs, drafts, vocab = p.shape[0], p.shape[1] - 1, p.shape[2]
        if q is not None:
            _need(tuple(q.shape) == (seqs, drafts, vocab) and (vocab <= 1 or q.stride(2) == 1) and q.dtype == p.dtype and
                  q.device == p.device, "q: %s like p expected" % [seqs, drafts, vocab])
        a = _VerifyArgs(p=p.data_ptr(), q=None if q is None else q.data_ptr(), p_seq_stride=p.stride(0), p_stride=p.stride(1),
                        q_seq_stride=0 if q is None else q.stride(0), q_stride=0 if q is None else q.stride(1),
                        draft_tokens=_whole(draft_tokens, "draft_tokens", "int32", [seqs, drafts], p.device),
                        draft_lens=None if draft_lens is None else _whole(draft_lens, "draft_lens", "int32", [seqs], p.device),
                        uniform=_whole(uniform, "uniform", "float32", [seqs, drafts + 1], p.device),
                        tokens=_whole(tokens, "tokens", "int32", [seqs, drafts + 1], p.device),
                        accepted=_whole(accepted, "accepted", "int32", [seqs], p.device), type=_type(p), seqs=seqs, drafts=drafts,
                        vocab=vocab)
        super().__init__("biq_verify_drafts", a, (p, q, draft_tokens, draft_lens, uniform, tokens, accepted), workspace, True, p.device, stream)


def biq_verify_drafts(p, q, draft_tokens, uniform, tokens, accepted, draft_lens=None, workspace=None, stream=None) -> None:
    PreparedVerify(p, q, draft_tokens, uniform, tokens, accepted, draft_lens, workspace, stream)()
