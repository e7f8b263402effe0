"""Binding of the fusion scorer's operators (``include/lightbeam_scorer.h``): the names of
the C ABI, over torch tensors.

The functions check what the C side cannot see of a tensor (its type, shape, device and
layout), raise ``LBError`` for it as for the library's own refusals, allocate the outputs
and workspaces that are not given, and enqueue the call on ``stream`` (None: torch's
current stream of the tensors' device).  Every step runs in the library's HIP kernels.  No
gradients are recorded: where torch records them, a tensor that requires one is refused,
and tensors of the caller's that a call writes to count as changed in place.

A call on few rows is mostly this file's work, so what a function has made itself is not
checked again, and nothing that the common case does not need is called.
"""

from __future__ import annotations

import ctypes
import functools
from typing import Optional

LB_F32, LB_BF16, LB_F16 = 0, 1, 2
LB_ROPE_HALF, LB_ROPE_INTERLEAVED = 0, 1
LB_ROPE_PLAIN, LB_ROPE_LINEAR, LB_ROPE_BLEND = 0, 1, 2
LB_KV_BAD_PAGE, LB_KV_BAD_LENGTH = 1, 2
LB_MAX_RULE_IDS = 4096

SCORER_EXPORTED = ("lb_rope_table", "lb_kv_append", "lb_kv_read", "lb_kv_attend_workspace", "lb_kv_attend",
                   "lb_lora_workspace", "lb_lora_add", "lb_logits_workspace", "lb_logits_adjust")

_P, _I, _L, _F, _D = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double


class lb_kv_cache(ctypes.Structure):
    _fields_ = [("pages", _P), ("n_pages", _L), ("page_tokens", _I), ("kv_heads", _I), ("head_dim", _I),
                ("reserved", _I), ("flags", _P)]


class lb_kv_batch(ctypes.Structure):
    _fields_ = [("starts", _P), ("lengths", _P), ("pages", _P), ("n_seqs", _I), ("n_rows", _I), ("max_pages", _I),
                ("max_new", _I)]


class lb_rope(ctypes.Structure):
    _fields_ = [("cos", _P), ("sin", _P), ("positions", _I), ("rot_dim", _I), ("layout", _I), ("reserved", _I)]


class lb_logit_rules(ctypes.Structure):
    _fields_ = [("temperature", _F), ("repetition", _F), ("presence", _F), ("frequency", _F), ("history", _P),
                ("bias_ids", _P), ("bias_values", _P), ("mask", _P), ("mask_row", _P), ("history_width", _I),
                ("bias_width", _I), ("bias_per_row", _I), ("mask_rows", _I)]


def declare(L) -> None:
    """Argument types of the loaded library's scorer functions."""
    at = {
        "lb_rope_table": [_I, _I, _D, _I, _D, _D, _D, _D, _P, _P],
        "lb_kv_append": [_P, _P, _P, _I, _I, _P, _L, _P, _L, _P, _L, _P, _L, _P],
        "lb_kv_read": [_P, _P, _I, _P, _L, _P, _L, _P],
        "lb_kv_attend_workspace": [_P, _P, _I, _P],
        "lb_kv_attend": [_P, _P, _I, _I, _P, _L, _F, _I, _P, _L, _P, _P, _L, _P],
        "lb_lora_workspace": [_L, _I, _I, _I, _P],
        "lb_lora_add": [_I, _L, _I, _I, _I, _I, _P, _L, _P, _L, _P, _P, _P, _P, _P, _L, _P, _L, _P],
        "lb_logits_workspace": [_L, _I, _P],
        "lb_logits_adjust": [_I, _L, _I, _P, _L, _P, _P, _P, _L, _P, _P, _P, _L, _P],
    }
    for name in SCORER_EXPORTED:
        f = getattr(L, name)
        f.restype = _I
        f.argtypes = at[name]


# torch, this package, torch's current raw stream of a device, its current device, whether it records gradients
# and what counts a tensor as changed, set by _load() before the first use: the package can be imported without
# torch, and a call of a few microseconds has no time for an import statement in each helper
torch = _lbm = _raw_stream = _current_device = _recording = _changed = None
_DTYPE = {}


def _load() -> None:
    global torch, _lbm, _raw_stream, _current_device, _recording, _changed
    if torch is not None:
        return
    import torch as t
    import paper_2603_14002_amd as lbm
    _DTYPE.update({t.float32: LB_F32, t.bfloat16: LB_BF16, t.float16: LB_F16})
    _lbm, _current_device, _recording, _changed = lbm, t.cuda.current_device, t.is_grad_enabled, t.autograd.graph.increment_version
    # what torch.cuda.current_stream(i).cuda_stream reads, without making a Stream object (2.8 us)
    _raw_stream = getattr(t._C, "_cuda_getCurrentRawStream", None) or (lambda i: t.cuda.current_stream(i).cuda_stream)
    torch = t


def _bad(msg: str):
    _load()
    raise _lbm.LBError(_lbm.LB_ERR_INVALID_ARG, msg)


def _dtype(t, name: str) -> int:
    if torch is None:
        _load()
    d = _DTYPE.get(t.dtype)
    if d is None:
        _bad(f"{name} must be float32, bfloat16 or float16")
    return d


def _call(g: int, stream, name: str, *args) -> None:
    """Calls an entry point with `stream` last, on the tensors' device."""
    if g < 0:
        _bad(f"{name}: the tensors must be on a GPU")
    f = getattr(_lbm._lib or _lbm.lib(), name)
    if g == _current_device():
        st = f(*args, _raw_stream(g) if stream is None else _lbm._stream_ptr(stream))
    else:
        with torch.cuda.device(g):
            st = f(*args, _raw_stream(g) if stream is None else _lbm._stream_ptr(stream))
    if st:
        raise _lbm.LBError(st, _lbm.lb_last_error())


def _elsewhere(g: int, **tensors) -> None:
    """Refuses the call for the first of its tensors that is not on device `g` (-1: not on a GPU)."""
    for name, t in tensors.items():
        if t is not None and t.get_device() != g:
            _bad(f"{name} is on {t.device}, the call's other tensors are on {f'cuda:{g}' if g >= 0 else 'cpu'}")


def _counts(**values) -> None:
    """Refuses the call for the first number that is negative or past 31 bits, of which ctypes would drop the rest."""
    for name, n in values.items():
        if n >> 31:
            _bad(f"{name} must be in 0..2^31 - 1")


def _no_gradient(**tensors) -> None:
    """Refuses the call for the first of its tensors that requires a gradient."""
    for name, t in tensors.items():
        if t is not None and t.requires_grad:
            _bad(f"{name} requires a gradient, and none is recorded: call under torch.no_grad(), or detach it")


def _empty(shape, dtype, like, stream):
    """A new tensor on `like`'s device for a call on `stream`.  For another stream than torch's current one it
    comes from that stream's own pool (a block of the current stream's pool may still be in use by work queued
    there), and it is also kept for work that the current stream has been given when it is dropped."""
    if stream is None:
        return torch.empty(*shape, dtype=dtype, device=like.device)  # sizes one by one: parsed sooner than a tuple
    with torch.cuda.device(like.device):
        here = torch.cuda.current_stream()
        with torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream):
            t = torch.empty(*shape, dtype=dtype, device=like.device)
        t.record_stream(here)
    return t


def _scratch(like, stream, nbytes: int, given, name: str):
    """The workspace given, or a new one: its address (None: none is needed), its size and the tensor itself,
    which has to live until the call has been enqueued."""
    if given is not None:
        if given.get_device() != like.get_device() or not given.is_contiguous():
            _bad(f"{name}: the workspace must be contiguous, on {like.device}")
        return given.data_ptr(), given.numel() * given.element_size(), given
    if nbytes == 0:
        return None, 0, None
    ws = _empty((nbytes,), torch.uint8, like, stream)
    return ws.data_ptr(), nbytes, ws


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _ints(t, name: str, shape) -> None:
    """A contiguous int32 tensor; None in `shape`: any size there."""
    if t.dtype is not torch.int32 or not t.is_contiguous():
        _bad(f"{name} must be a contiguous int32 tensor")
    at = t.shape
    if len(at) != len(shape):
        _bad(f"{name} has shape {tuple(at)}, expected {tuple('any' if n is None else n for n in shape)}")
    for n, m in zip(shape, at):
        if n is not None and n != m:
            _bad(f"{name} has shape {tuple(at)}, expected {tuple('any' if n is None else n for n in shape)}")


def _heads(t, name: str, rows: int, heads: Optional[int], dim: int, dtype) -> int:
    """Row stride of [rows, heads, dim] whose heads and channels lie together."""
    if t.dtype is not dtype:
        _bad(f"{name} is {t.dtype}, expected {dtype}")
    at = t.shape
    if len(at) != 3 or at[0] != rows or at[2] != dim or (heads is not None and at[1] != heads):
        _bad(f"{name} has shape {tuple(at)}, expected ({rows}, {'heads' if heads is None else heads}, {dim})")
    s0, s1, s2 = t.stride()
    if rows and ((at[1] > 1 and s1 != dim) or s2 != 1):
        _bad(f"{name}: the heads of a row must lie one after the other")
    return s0 if rows > 1 else at[1] * dim


def _rows(t, name: str, rows: int, width: int, dtype) -> int:
    """Row stride of [rows, width] whose rows are contiguous."""
    if t.dtype is not dtype:
        _bad(f"{name} is {t.dtype}, expected {dtype}")
    at = t.shape
    if len(at) != 2 or at[0] != rows or at[1] != width:
        _bad(f"{name} has shape {tuple(at)}, expected ({rows}, {width})")
    s0, s1 = t.stride()
    if width > 1 and rows and s1 != 1:
        _bad(f"{name}: the values of a row must lie one after the other")
    return s0 if rows > 1 else width


# ------------------------------------------------------------------ descriptors


class KVCache:
    """A paged 4-bit cache in the caller's memory (``lb_kv_cache``): `pages` uint8
    [n_pages, kv_heads, page_tokens * (head_dim + head_dim / 16)], `flags` None or an int32
    tensor of one element that faults of the data are or-ed into."""

    __slots__ = ("pages", "flags", "page_tokens", "kv_heads", "head_dim", "device", "sizes", "desc", "ref")

    def __init__(self, pages, page_tokens: int, kv_heads: int, head_dim: int, flags=None):
        if torch is None:
            _load()
        if pages.dtype is not torch.uint8 or not pages.is_contiguous():
            _bad("pages must be a contiguous uint8 tensor")
        at = pages.shape
        if len(at) != 3 or at[1] != kv_heads or at[2] != page_tokens * (head_dim + head_dim // 16):
            _bad(f"pages has shape {tuple(at)}, expected (pages, {kv_heads}, {self.page_bytes(page_tokens, 1, head_dim)})")
        if (page_tokens | kv_heads | head_dim) >> 31:
            _counts(page_tokens=page_tokens, kv_heads=kv_heads, head_dim=head_dim)
        self.device = pages.get_device()
        if flags is not None and (flags.dtype is not torch.int32 or flags.numel() != 1 or flags.get_device() != self.device):
            _bad("flags must be one int32 on the pages' device")
        self.pages, self.flags = pages, flags
        self.sizes = self.page_tokens, self.kv_heads, self.head_dim = page_tokens, kv_heads, head_dim
        self.desc = lb_kv_cache(pages.data_ptr(), at[0], page_tokens, kv_heads, head_dim, 0, _ptr(flags))
        self.ref = ctypes.addressof(self.desc)

    @staticmethod
    def page_bytes(page_tokens: int, kv_heads: int, head_dim: int) -> int:
        return kv_heads * page_tokens * (head_dim + head_dim // 16)

    @classmethod
    def empty(cls, n_pages: int, page_tokens: int, kv_heads: int, head_dim: int, device="cuda"):
        """A cache in new memory, with a flags word."""
        _load()
        pages = torch.empty((n_pages, kv_heads, cls.page_bytes(page_tokens, 1, head_dim)), dtype=torch.uint8, device=device)
        return cls(pages, page_tokens, kv_heads, head_dim, torch.zeros(1, dtype=torch.int32, device=device))

    def status(self) -> int:
        """The LB_KV_* faults found so far (waits for the device)."""
        return 0 if self.flags is None else int(self.flags.item())


class KVBatch:
    """A ragged batch (``lb_kv_batch``): int32 device tensors starts [n_seqs + 1], lengths
    [n_seqs] and pages [n_seqs, max_pages]; `n_rows` rows of activations, at most `max_new`
    new tokens a sequence.  The tensors may be changed between calls."""

    __slots__ = ("starts", "lengths", "pages", "n_rows", "max_pages", "device", "sizes", "desc", "ref")

    def __init__(self, starts, lengths, pages, n_rows: int, max_new: int):
        if torch is None:
            _load()
        i32, at = torch.int32, pages.shape
        n = at[0] if len(at) == 2 else -1
        if starts.dtype is not i32 or lengths.dtype is not i32 or pages.dtype is not i32 or starts.shape != (n + 1,) or lengths.shape != (n,) \
                or not starts.is_contiguous() or not lengths.is_contiguous() or not pages.is_contiguous():
            n = lengths.shape[0] if lengths.dim() else 0
            _ints(starts, "starts", (n + 1,))
            _ints(lengths, "lengths", (n,))
            _ints(pages, "the page table", (n, None))
        if (n | n_rows | at[1] | max_new) >> 31:
            _counts(n_seqs=n, n_rows=n_rows, max_pages=at[1], max_new=max_new)
        self.device = g = starts.get_device()
        if lengths.get_device() != g or pages.get_device() != g:
            _elsewhere(g, lengths=lengths, pages=pages)
        self.starts, self.lengths, self.pages, self.n_rows, self.max_pages = starts, lengths, pages, n_rows, at[1]
        self.sizes = (n, n_rows, at[1], max_new)
        self.desc = lb_kv_batch(starts.data_ptr(), lengths.data_ptr(), pages.data_ptr(), n, n_rows, at[1], max_new)
        self.ref = ctypes.addressof(self.desc)


class Rope:
    """Angles of the rotation (``lb_rope``): cos and sin, float32 [positions, rot_dim / 2]."""

    __slots__ = ("cos", "sin", "device", "desc", "ref")

    def __init__(self, cos, sin, layout: int = LB_ROPE_HALF):
        if torch is None:
            _load()
        if cos.dtype is not torch.float32 or sin.dtype is not torch.float32 or cos.dim() != 2 or cos.shape != sin.shape \
                or not cos.is_contiguous() or not sin.is_contiguous() or cos.device != sin.device:
            _bad("cos and sin must be contiguous float32 [positions, rot_dim / 2] on one device")
        if (cos.shape[0] | 2 * cos.shape[1] | layout) >> 31:
            _counts(positions=cos.shape[0], rot_dim=2 * cos.shape[1], layout=layout)
        self.cos, self.sin, self.device = cos, sin, cos.get_device()
        self.desc = lb_rope(cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1], layout, 0)
        self.ref = ctypes.addressof(self.desc)


class LogitRules:
    """What ``lb_logits_adjust`` does before the log-softmax (``lb_logit_rules``): history int32
    [rows, width]; bias_ids int32 and bias_values float32 [rows or 1, width]; mask int32 (32
    classes a word) [masks, (classes + 31) // 32] and mask_row int32 [rows]."""

    __slots__ = ("history", "bias_ids", "bias_values", "mask", "mask_row", "desc", "ref")

    def __init__(self, temperature: float = 1.0, history=None, repetition: float = 1.0, presence: float = 0.0,
                 frequency: float = 0.0, bias_ids=None, bias_values=None, mask=None, mask_row=None):
        if torch is None:
            _load()
        self.history, self.bias_ids, self.bias_values, self.mask, self.mask_row = history, bias_ids, bias_values, mask, mask_row
        i32 = torch.int32
        h = bi = bv = mk = mr = None
        hw = bw = per_row = masks = 0
        if history is not None:
            at = history.shape
            if history.dtype is not i32 or len(at) != 2 or not history.is_contiguous():
                _ints(history, "history", (None, None))
            h, hw = history.data_ptr(), at[1]
        if (bias_ids is None) != (bias_values is None):
            _bad("bias_ids and bias_values belong together")
        if bias_ids is not None:
            at = bias_ids.shape
            if bias_ids.dtype is not i32 or len(at) != 2 or not bias_ids.is_contiguous():
                _ints(bias_ids, "bias_ids", (None, None))
            if bias_values.dtype is not torch.float32 or bias_values.shape != at or not bias_values.is_contiguous():
                _bad("bias_values must be contiguous float32 of bias_ids' shape")
            bi, bv, bw, per_row = bias_ids.data_ptr(), bias_values.data_ptr(), at[1], 0 if at[0] == 1 else 1
        if mask is not None:
            at = mask.shape
            if mask.dtype is not i32 or len(at) != 2 or not mask.is_contiguous():
                _ints(mask, "mask", (None, None))
            mk, masks = mask.data_ptr(), at[0]
        if mask_row is not None:
            if mask is None:
                _bad("mask_row needs a mask")
            if mask_row.dtype is not i32 or len(mask_row.shape) != 1 or not mask_row.is_contiguous():
                _ints(mask_row, "mask_row", (None,))
            mr = mask_row.data_ptr()
        if (hw | bw | masks) >> 31:
            _counts(history_width=hw, bias_width=bw, mask_rows=masks)
        self.desc = lb_logit_rules(temperature, repetition, presence, frequency, h, bi, bv, mk, mr, hw, bw, per_row, masks)
        self.ref = ctypes.addressof(self.desc)


# ------------------------------------------------------------------ C-ABI wrappers (same names)


def lb_rope_table(positions: int, rot_dim: int, base: float = 10000.0, scaling: int = LB_ROPE_PLAIN, factor: float = 1.0,
                  trained: float = 0.0, low: float = 1.0, high: float = 4.0):
    """Host tables (cos, sin), float32 [positions, rot_dim / 2]."""
    _load()
    _counts(positions=positions, rot_dim=rot_dim, scaling=scaling)
    cos = torch.empty((positions, rot_dim // 2), dtype=torch.float32)
    sin = torch.empty_like(cos)
    _lbm._check(_lbm.lib().lb_rope_table(positions, rot_dim, base, scaling, factor, trained, low, high, cos.data_ptr(),
                                         sin.data_ptr()))
    return cos, sin


def lb_kv_append(cache: KVCache, batch: KVBatch, q, k, v, rope: Optional[Rope] = None, q_out=None, stream=None):
    """Appends the batch's new keys and values ([n_rows, kv_heads, head_dim]) to the cache, rotated
    if `rope` is given; q [n_rows, q_heads, head_dim] or None.  Returns the rotated queries (q_out,
    which may be q itself, or a new tensor)."""
    dt, dtype, n, H, D, g = _dtype(k, "k"), k.dtype, batch.n_rows, cache.kv_heads, cache.head_dim, cache.device
    ks, vs = _heads(k, "k", n, H, D, dtype), _heads(v, "v", n, H, D, dtype)
    if batch.device != g or k.get_device() != g or v.get_device() != g or (rope is not None and rope.device != g):
        _elsewhere(g, starts=batch.starts, k=k, v=v, cos=None if rope is None else rope.cos)
    if _recording() and (k.requires_grad or v.requires_grad or (q is not None and q.requires_grad) or (q_out is not None and q_out.requires_grad)
                         or (rope is not None and (rope.cos.requires_grad or rope.sin.requires_grad))):
        _no_gradient(q=q, k=k, v=v, q_out=q_out, cos=None if rope is None else rope.cos, sin=None if rope is None else rope.sin)
    hq = qs = os = 0
    written = cache.pages if q_out is None else (cache.pages, q_out)
    if q is not None:
        qs, hq = _heads(q, "q", n, None, D, dtype), q.shape[1]
        if q.get_device() != g or (q_out is not None and q_out.get_device() != g):
            _elsewhere(g, q=q, q_out=q_out)
        if q_out is None:
            q_out, os = _empty((n, hq, D), dtype, q, stream), hq * D
        else:
            os = _heads(q_out, "q_out", n, hq, D, dtype)
    elif q_out is not None:
        _bad("q_out needs q")
    _call(g, stream, "lb_kv_append", cache.ref, batch.ref, None if rope is None else rope.ref, dt, hq, _ptr(q), qs,
          k.data_ptr(), ks, v.data_ptr(), vs, _ptr(q_out), os)
    _changed(written)
    return q_out


def lb_kv_read(cache: KVCache, batch: KVBatch, dtype=None, k_out=None, v_out=None, stream=None):
    """The keys and values that the cache holds of the batch's new tokens, [n_rows, kv_heads, head_dim] each
    (k_out and v_out, or new tensors of `dtype`, float32 if None; of rows that are padding nothing is written)."""
    n, H, D, g = batch.n_rows, cache.kv_heads, cache.head_dim, cache.device
    if dtype is None:
        given = k_out if k_out is not None else v_out
        dtype = torch.float32 if given is None else given.dtype
    ks = vs = H * D
    if batch.device != g:
        _elsewhere(g, starts=batch.starts)
    written = [t for t in (k_out, v_out) if t is not None]
    if written and _recording():
        _no_gradient(k_out=k_out, v_out=v_out)
    if k_out is None:
        k_out = _empty((n, H, D), dtype, cache.pages, stream)
    else:
        ks = _heads(k_out, "k_out", n, H, D, dtype)
        _elsewhere(g, k_out=k_out)
    if v_out is None:
        v_out = _empty((n, H, D), dtype, cache.pages, stream)
    else:
        vs = _heads(v_out, "v_out", n, H, D, dtype)
        _elsewhere(g, v_out=v_out)
    _call(g, stream, "lb_kv_read", cache.ref, batch.ref, _dtype(k_out, "k_out"), k_out.data_ptr(), ks, v_out.data_ptr(), vs)
    if written:
        _changed(written)
    return k_out, v_out


def lb_kv_attend_workspace(cache: KVCache, batch: KVBatch, q_heads: int) -> int:
    _counts(q_heads=q_heads)
    need = _L()
    _lbm._check((_lbm._lib or _lbm.lib()).lb_kv_attend_workspace(cache.ref, batch.ref, q_heads, ctypes.addressof(need)))
    return need.value


_attend_bytes = {}  # what the library has said of these sizes


def lb_kv_attend(cache: KVCache, batch: KVBatch, q, scale: float, window: int = 0, out=None, lse=None, want_lse: bool = False,
                 workspace=None, stream=None):
    """Attention of the batch's new tokens, q [n_rows, q_heads, head_dim].  Returns (out, lse): out (or a
    new tensor) as q, lse float32 [n_rows, q_heads] or None."""
    dt, dtype, n, D, g = _dtype(q, "q"), q.dtype, batch.n_rows, cache.head_dim, cache.device
    qs = _heads(q, "q", n, None, D, dtype)
    hq = q.shape[1]
    if batch.device != g or q.get_device() != g:
        _elsewhere(g, starts=batch.starts, q=q)
    if (hq | window) >> 31:
        _counts(q_heads=hq, window=window)
    written = () if out is None and lse is None else [t for t in (out, lse) if t is not None]
    if _recording() and (q.requires_grad or written):
        _no_gradient(q=q, out=out, lse=lse)
    if out is None:
        out, os = _empty((n, hq, D), dtype, q, stream), hq * D
    else:
        os = _heads(out, "out", n, hq, D, dtype)
        _elsewhere(g, out=out)
    if lse is not None:
        if lse.dtype is not torch.float32 or lse.shape != (n, hq) or not lse.is_contiguous():
            _bad(f"lse must be contiguous float32 ({n}, {hq})")
        _elsewhere(g, lse=lse)
    elif want_lse:
        lse = _empty((n, hq), torch.float32, q, stream)
    need = 0
    if workspace is None:
        sizes = (cache.sizes, batch.sizes, hq)
        need = _attend_bytes.get(sizes)
        if need is None:
            need = lb_kv_attend_workspace(cache, batch, hq)
            if len(_attend_bytes) >= 4096:
                _attend_bytes.clear()
            _attend_bytes[sizes] = need
    ws, nbytes, _held = _scratch(q, stream, need, workspace, "lb_kv_attend")
    _call(g, stream, "lb_kv_attend", cache.ref, batch.ref, dt, hq, q.data_ptr(), qs, scale, window, out.data_ptr(), os,
          _ptr(lse), ws, nbytes)
    if written:
        _changed(written)
    return out, lse


@functools.lru_cache(maxsize=4096)
def lb_lora_workspace(rows: int, d_in: int, d_out: int, rank: int) -> int:
    _load()
    _counts(d_in=d_in, d_out=d_out, rank=rank)
    need = _L()
    _lbm._check((_lbm._lib or _lbm.lib()).lb_lora_workspace(rows, d_in, d_out, rank, ctypes.addressof(need)))
    return need.value


def lb_lora_add(y, x, a, b, adapter, scale=None, out=None, workspace=None, stream=None):
    """y [rows, d_out] + scale[adapter] * b[adapter] (a[adapter] x), x [rows, d_in], a [n, rank, d_in],
    b [n, d_out, rank], adapter int32 [rows], scale float32 [n] or None.  Written to `out` (None: y itself),
    which is returned."""
    dt, dtype, g = _dtype(y, "y"), y.dtype, y.get_device()
    if x.dim() != 2 or y.dim() != 2 or a.dim() != 3 or b.dim() != 3:
        _bad("x and y must have 2 dimensions, a and b 3")
    (rows, d_out), d_in, (n, rank, _) = y.shape, x.shape[1], a.shape
    if (d_in | d_out | rank | n) >> 31:
        _counts(d_in=d_in, d_out=d_out, rank=rank, n_adapters=n)
    xs, ys = _rows(x, "x", rows, d_in, dtype), _rows(y, "y", rows, d_out, dtype)
    if out is None:
        out, os = y, ys
    else:
        os = _rows(out, "out", rows, d_out, dtype)
    if a.dtype is not dtype or a.shape != (n, rank, d_in) or not a.is_contiguous():
        _bad(f"a must be contiguous {dtype} ({n}, {rank}, {d_in})")
    if b.dtype is not dtype or b.shape != (n, d_out, rank) or not b.is_contiguous():
        _bad(f"b must be contiguous {dtype} ({n}, {d_out}, {rank})")
    _ints(adapter, "adapter", (rows,))
    if scale is not None and (scale.dtype is not torch.float32 or scale.shape != (n,) or not scale.is_contiguous()):
        _bad(f"scale must be contiguous float32 ({n},)")
    if x.get_device() != g or a.get_device() != g or b.get_device() != g or adapter.get_device() != g or out.get_device() != g \
            or (scale is not None and scale.get_device() != g):
        _elsewhere(g, x=x, a=a, b=b, adapter=adapter, scale=scale, out=out)
    if _recording() and (y.requires_grad or x.requires_grad or a.requires_grad or b.requires_grad or out.requires_grad
                         or (scale is not None and scale.requires_grad)):
        _no_gradient(y=y, x=x, a=a, b=b, scale=scale, out=out)
    xp, op = x.data_ptr(), out.data_ptr()
    need = 0 if workspace is not None else lb_lora_workspace(rows, d_in, d_out, rank)
    if need == 0 and -4 * rows * os < op - xp < 4 * rows * xs:  # at most 4 B a value: they may overlap
        need = 4 * rows * rank
    ws, nbytes, _held = _scratch(y, stream, need, workspace, "lb_lora_add")
    _call(g, stream, "lb_lora_add", dt, rows, d_in, d_out, rank, n, xp, xs, y.data_ptr(), ys, a.data_ptr(),
          b.data_ptr(), adapter.data_ptr(), _ptr(scale), op, os, ws, nbytes)
    _changed(out)
    return out


@functools.lru_cache(maxsize=4096)
def lb_logits_workspace(rows: int, classes: int) -> int:
    _load()
    _counts(classes=classes)
    need = _L()
    _lbm._check((_lbm._lib or _lbm.lib()).lb_logits_workspace(rows, classes, ctypes.addressof(need)))
    return need.value


def lb_logits_adjust(logits, rules: Optional[LogitRules] = None, target=None, want_logprobs: bool = True, logprobs=None,
                     workspace=None, stream=None):
    """Adjusted log-probabilities of logits [rows, classes].  Returns (logprobs, score, lse): float32
    [rows, classes] (None unless wanted or given), float32 [rows] at target int32 [rows] (None without
    one), and float32 [rows]."""
    dt, g = _dtype(logits, "logits"), logits.get_device()
    if logits.dim() != 2:
        _bad("logits must have 2 dimensions")
    rows, classes = logits.shape
    if classes >> 31:
        _counts(classes=classes)
    stride = _rows(logits, "logits", rows, classes, logits.dtype)
    if _recording() and (logits.requires_grad or logprobs is not None or rules is not None):
        _no_gradient(logits=logits, logprobs=logprobs, bias_values=None if rules is None else rules.bias_values)
    written = logprobs
    os = classes
    if logprobs is not None:
        os = _rows(logprobs, "logprobs", rows, classes, torch.float32)
        if logprobs.get_device() != g:
            _elsewhere(g, logprobs=logprobs)
    elif want_logprobs:
        logprobs = _empty((rows, classes), torch.float32, logits, stream)
    score = None
    if target is not None:
        _ints(target, "target", (rows,))
        if target.get_device() != g:
            _elsewhere(g, target=target)
        score = _empty((rows,), torch.float32, logits, stream)
    lse = _empty((rows,), torch.float32, logits, stream)
    ref = None
    if rules is not None:
        h, b, m, r = rules.history, rules.bias_ids, rules.mask, rules.mask_row
        if h is not None and (h.shape[0] != rows or h.get_device() != g):
            _elsewhere(g, history=h)
            _bad(f"history has {h.shape[0]} rows, the logits {rows}")
        if b is not None and ((b.shape[0] != 1 and b.shape[0] != rows) or b.get_device() != g or rules.bias_values.get_device() != g):
            _elsewhere(g, bias_ids=b, bias_values=rules.bias_values)
            _bad(f"bias_ids has {b.shape[0]} rows, the logits {rows}")
        if m is not None and (m.shape[1] != (classes + 31) // 32 or m.get_device() != g):
            _elsewhere(g, mask=m)
            _bad(f"mask has {m.shape[1]} words a row, expected {(classes + 31) // 32}")
        if r is not None and (r.shape[0] != rows or r.get_device() != g):
            _elsewhere(g, mask_row=r)
            _bad(f"mask_row has {r.shape[0]} entries, expected {rows}")
        ref = rules.ref
    ws, nbytes, _held = _scratch(logits, stream, 0 if workspace is not None else lb_logits_workspace(rows, classes), workspace, "lb_logits_adjust")
    _call(g, stream, "lb_logits_adjust", dt, rows, classes, logits.data_ptr(), stride, ref, _ptr(target), _ptr(logprobs), os,
          _ptr(score), _ptr(lse), ws, nbytes)
    if written is not None:
        _changed(written)
    return logprobs, score, lse
