"""Binding of the fusion scorer's operators (``include/lightbeam_scorer.h``): the names of
the C ABI, over torch tensors.

The functions check what the C side cannot see of a tensor (its type, shape, device and
layout), raise ``LBError`` for it as for the library's own refusals, allocate the outputs
and workspaces that are not given, and enqueue the call on ``stream`` (None: torch's
current stream of the tensors' device).  Every step runs in the library's HIP kernels.
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


def _binding():
    import paper_2603_14002_amd as lbm
    return lbm


@functools.lru_cache(maxsize=None)
def _dtypes():
    import torch
    return {torch.float32: LB_F32, torch.bfloat16: LB_BF16, torch.float16: LB_F16}


def _bad(msg: str):
    lbm = _binding()
    raise lbm.LBError(lbm.LB_ERR_INVALID_ARG, msg)


def _dtype(t, name: str) -> int:
    d = _dtypes().get(t.dtype)
    if d is None:
        _bad(f"{name} must be float32, bfloat16 or float16")
    return d


def _call(dev, stream, name: str, *args) -> None:
    """Calls an entry point with `stream` last, on the tensors' device."""
    import torch
    lbm = _binding()
    if dev.type != "cuda":
        _bad(f"{name}: the tensors must be on a GPU")
    f = getattr(lbm.lib(), name)
    here = torch.cuda.current_device()
    if dev.index is None or dev.index == here:
        st = f(*args, lbm._stream_ptr(stream))
    else:
        with torch.cuda.device(dev):
            st = f(*args, lbm._stream_ptr(stream))
    if st != lbm.LB_OK:
        raise lbm.LBError(st, lbm.lb_last_error())


def _same_device(dev, **tensors) -> None:
    for name, t in tensors.items():
        if t is not None and t.device != dev:
            _bad(f"{name} is on {t.device}, the call's other tensors are on {dev}")


def _scratch(dev, stream, nbytes: int, given, name: str):
    """The workspace given, or a new one that lives until the stream is done with it."""
    import torch
    if given is not None:
        if given.device != dev or not given.is_contiguous():
            _bad(f"{name}: the workspace must be contiguous, on {dev}")
        return given, given.numel() * given.element_size()
    if nbytes == 0:
        return None, 0
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    if stream is not None:
        with torch.cuda.device(dev):
            ws.record_stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream)
    return ws, nbytes


def _empty(like, stream, shape, dtype=None):
    """A new output, safe to drop while `stream` still writes it."""
    import torch
    out = torch.empty(shape, dtype=dtype or like.dtype, device=like.device)
    if stream is not None:
        with torch.cuda.device(like.device):
            out.record_stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream)
    return out


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _ints(t, name: str, shape) -> None:
    """A contiguous int32 tensor; None in `shape`: any size there."""
    import torch
    if t.dtype != torch.int32 or not t.is_contiguous():
        _bad(f"{name} must be a contiguous int32 tensor")
    if t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        _bad(f"{name} has shape {tuple(t.shape)}, expected {tuple('any' if n is None else n for n in shape)}")


def _heads(t, name: str, rows: int, heads: Optional[int], dim: int, dtype) -> int:
    """Row stride of [rows, heads, dim] whose heads and channels lie together."""
    if t.dtype != dtype:
        _bad(f"{name} is {t.dtype}, expected {dtype}")
    if t.dim() != 3 or t.shape[0] != rows or t.shape[2] != dim or (heads is not None and t.shape[1] != heads):
        _bad(f"{name} has shape {tuple(t.shape)}, expected ({rows}, {'heads' if heads is None else heads}, {dim})")
    if rows and ((t.shape[1] > 1 and t.stride(1) != dim) or t.stride(2) != 1):
        _bad(f"{name}: the heads of a row must lie one after the other")
    return t.stride(0) if rows > 1 else t.shape[1] * dim


def _rows(t, name: str, rows: int, width: int, dtype) -> int:
    """Row stride of [rows, width] whose rows are contiguous."""
    if t.dtype != dtype:
        _bad(f"{name} is {t.dtype}, expected {dtype}")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != width:
        _bad(f"{name} has shape {tuple(t.shape)}, expected ({rows}, {width})")
    if width > 1 and rows and t.stride(1) != 1:
        _bad(f"{name}: the values of a row must lie one after the other")
    return t.stride(0) if rows > 1 else width


# ------------------------------------------------------------------ descriptors


class KVCache:
    """A paged 4-bit cache in the caller's memory (``lb_kv_cache``): `pages` uint8
    [n_pages, kv_heads, page_tokens * (head_dim + head_dim / 16)], `flags` None or an int32
    tensor of one element that faults of the data are or-ed into."""

    __slots__ = ("pages", "flags", "page_tokens", "kv_heads", "head_dim", "desc", "ref")

    def __init__(self, pages, page_tokens: int, kv_heads: int, head_dim: int, flags=None):
        import torch
        if pages.dtype != torch.uint8 or not pages.is_contiguous():
            _bad("pages must be a contiguous uint8 tensor")
        if pages.dim() != 3 or pages.shape[1] != kv_heads or pages.shape[2] != self.page_bytes(page_tokens, 1, head_dim):
            _bad(f"pages has shape {tuple(pages.shape)}, expected (pages, {kv_heads}, {self.page_bytes(page_tokens, 1, head_dim)})")
        if flags is not None and (flags.dtype != torch.int32 or flags.numel() != 1 or flags.device != pages.device):
            _bad("flags must be one int32 on the pages' device")
        self.pages, self.flags = pages, flags
        self.page_tokens, self.kv_heads, self.head_dim = page_tokens, kv_heads, head_dim
        self.desc = lb_kv_cache(pages.data_ptr(), pages.shape[0], page_tokens, kv_heads, head_dim, 0, _ptr(flags))
        self.ref = ctypes.addressof(self.desc)

    @staticmethod
    def page_bytes(page_tokens: int, kv_heads: int, head_dim: int) -> int:
        return kv_heads * page_tokens * (head_dim + head_dim // 16)

    @classmethod
    def empty(cls, n_pages: int, page_tokens: int, kv_heads: int, head_dim: int, device="cuda"):
        """A cache in new memory, with a flags word."""
        import torch
        pages = torch.empty((n_pages, kv_heads, cls.page_bytes(page_tokens, 1, head_dim)), dtype=torch.uint8, device=device)
        return cls(pages, page_tokens, kv_heads, head_dim, torch.zeros(1, dtype=torch.int32, device=device))

    def status(self) -> int:
        """The LB_KV_* faults found so far (waits for the device)."""
        return 0 if self.flags is None else int(self.flags.item())


class KVBatch:
    """A ragged batch (``lb_kv_batch``): int32 device tensors starts [n_seqs + 1], lengths
    [n_seqs] and pages [n_seqs, max_pages]; `n_rows` rows of activations, at most `max_new`
    new tokens a sequence.  The tensors may be changed between calls."""

    __slots__ = ("starts", "lengths", "pages", "n_rows", "desc", "ref")

    def __init__(self, starts, lengths, pages, n_rows: int, max_new: int):
        n = lengths.shape[0] if lengths.dim() else 0
        _ints(starts, "starts", (n + 1,))
        _ints(lengths, "lengths", (n,))
        _ints(pages, "the page table", (n, None))
        _same_device(starts.device, lengths=lengths, pages=pages)
        self.starts, self.lengths, self.pages, self.n_rows = starts, lengths, pages, n_rows
        self.desc = lb_kv_batch(starts.data_ptr(), lengths.data_ptr(), pages.data_ptr(), n, n_rows, pages.shape[1], max_new)
        self.ref = ctypes.addressof(self.desc)


class Rope:
    """Angles of the rotation (``lb_rope``): cos and sin, float32 [positions, rot_dim / 2]."""

    __slots__ = ("cos", "sin", "desc", "ref")

    def __init__(self, cos, sin, layout: int = LB_ROPE_HALF):
        import torch
        if cos.dtype != torch.float32 or sin.dtype != torch.float32 or cos.dim() != 2 or cos.shape != sin.shape \
                or not cos.is_contiguous() or not sin.is_contiguous() or cos.device != sin.device:
            _bad("cos and sin must be contiguous float32 [positions, rot_dim / 2] on one device")
        self.cos, self.sin = cos, sin
        self.desc = lb_rope(cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1], layout, 0)
        self.ref = ctypes.addressof(self.desc)


class LogitRules:
    """What ``lb_logits_adjust`` does before the log-softmax (``lb_logit_rules``): history int32
    [rows, width]; bias_ids int32 and bias_values float32 [rows or 1, width]; mask int32 (32
    classes a word) [masks, (classes + 31) // 32] and mask_row int32 [rows]."""

    __slots__ = ("history", "bias_ids", "bias_values", "mask", "mask_row", "desc", "ref")

    def __init__(self, temperature: float = 1.0, history=None, repetition: float = 1.0, presence: float = 0.0,
                 frequency: float = 0.0, bias_ids=None, bias_values=None, mask=None, mask_row=None):
        import torch
        self.history, self.bias_ids, self.bias_values, self.mask, self.mask_row = history, bias_ids, bias_values, mask, mask_row
        if history is not None:
            _ints(history, "history", (None, None))
        if (bias_ids is None) != (bias_values is None):
            _bad("bias_ids and bias_values belong together")
        if bias_ids is not None:
            _ints(bias_ids, "bias_ids", (None, None))
            if bias_values.dtype != torch.float32 or bias_values.shape != bias_ids.shape or not bias_values.is_contiguous():
                _bad("bias_values must be contiguous float32 of bias_ids' shape")
        if mask is not None:
            _ints(mask, "mask", (None, None))
        if mask_row is not None:
            if mask is None:
                _bad("mask_row needs a mask")
            _ints(mask_row, "mask_row", (None,))
        self.desc = lb_logit_rules(temperature, repetition, presence, frequency, _ptr(history), _ptr(bias_ids),
                                   _ptr(bias_values), _ptr(mask), _ptr(mask_row),
                                   0 if history is None else history.shape[1], 0 if bias_ids is None else bias_ids.shape[1],
                                   0, 0 if mask is None else mask.shape[0])
        self.ref = ctypes.addressof(self.desc)


# ------------------------------------------------------------------ C-ABI wrappers (same names)


def lb_rope_table(positions: int, rot_dim: int, base: float = 10000.0, scaling: int = LB_ROPE_PLAIN, factor: float = 1.0,
                  trained: float = 0.0, low: float = 1.0, high: float = 4.0):
    """Host tables (cos, sin), float32 [positions, rot_dim / 2]."""
    import torch
    lbm = _binding()
    cos = torch.empty((max(positions, 0), max(rot_dim, 0) // 2), dtype=torch.float32)
    sin = torch.empty_like(cos)
    lbm._check(lbm.lib().lb_rope_table(positions, rot_dim, base, scaling, factor, trained, low, high, cos.data_ptr(),
                                       sin.data_ptr()))
    return cos, sin


def lb_kv_append(cache: KVCache, batch: KVBatch, q, k, v, rope: Optional[Rope] = None, q_out=None, stream=None):
    """Appends the batch's new keys and values ([n_rows, kv_heads, head_dim]) to the cache, rotated
    if `rope` is given; q [n_rows, q_heads, head_dim] or None.  Returns the rotated queries (q_out,
    which may be q itself, or a new tensor)."""
    dt, n, H, D = _dtype(k, "k"), batch.n_rows, cache.kv_heads, cache.head_dim
    dev = cache.pages.device
    _same_device(dev, starts=batch.starts, k=k, v=v, q=q, q_out=q_out, cos=None if rope is None else rope.cos)
    ks, vs = _heads(k, "k", n, H, D, k.dtype), _heads(v, "v", n, H, D, k.dtype)
    hq = qs = os = 0
    if q is not None:
        qs, hq = _heads(q, "q", n, None, D, k.dtype), q.shape[1]
        if q_out is None:
            q_out = _empty(q, stream, (n, hq, D))
        os = _heads(q_out, "q_out", n, hq, D, k.dtype)
    elif q_out is not None:
        _bad("q_out needs q")
    _call(dev, stream, "lb_kv_append", cache.ref, batch.ref, None if rope is None else rope.ref, dt, hq, _ptr(q), qs,
          k.data_ptr(), ks, v.data_ptr(), vs, _ptr(q_out), os)
    return q_out


def lb_kv_read(cache: KVCache, batch: KVBatch, dtype=None, k_out=None, v_out=None, stream=None):
    """The keys and values that the cache holds of the batch's new tokens, [n_rows, kv_heads, head_dim] each
    (k_out and v_out, or new tensors of `dtype`, float32 if None; of rows that are padding nothing is written)."""
    import torch
    n, H, D, dev = batch.n_rows, cache.kv_heads, cache.head_dim, cache.pages.device
    if dtype is None:
        given = k_out if k_out is not None else v_out
        dtype = torch.float32 if given is None else given.dtype
    k_out = _empty(cache.pages, stream, (n, H, D), dtype) if k_out is None else k_out
    v_out = _empty(cache.pages, stream, (n, H, D), dtype) if v_out is None else v_out
    _same_device(dev, starts=batch.starts, k_out=k_out, v_out=v_out)
    ks, vs = _heads(k_out, "k_out", n, H, D, dtype), _heads(v_out, "v_out", n, H, D, dtype)
    _call(dev, stream, "lb_kv_read", cache.ref, batch.ref, _dtype(k_out, "k_out"), k_out.data_ptr(), ks, v_out.data_ptr(), vs)
    return k_out, v_out


def lb_kv_attend_workspace(cache: KVCache, batch: KVBatch, q_heads: int) -> int:
    lbm = _binding()
    need = ctypes.c_int64()
    lbm._check(lbm.lib().lb_kv_attend_workspace(cache.ref, batch.ref, q_heads, ctypes.addressof(need)))
    return need.value


def lb_kv_attend(cache: KVCache, batch: KVBatch, q, scale: float, window: int = 0, out=None, lse=None, want_lse: bool = False,
                 workspace=None, stream=None):
    """Attention of the batch's new tokens, q [n_rows, q_heads, head_dim].  Returns (out, lse): out (or a
    new tensor) as q, lse float32 [n_rows, q_heads] or None."""
    import torch
    dt, n, D, dev = _dtype(q, "q"), batch.n_rows, cache.head_dim, cache.pages.device
    qs = _heads(q, "q", n, None, D, q.dtype)
    hq = q.shape[1]
    if out is None:
        out = _empty(q, stream, (n, hq, D))
    os = _heads(out, "out", n, hq, D, q.dtype)
    if lse is None and want_lse:
        lse = _empty(q, stream, (n, hq), torch.float32)
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (n, hq) or not lse.is_contiguous()):
        _bad(f"lse must be contiguous float32 ({n}, {hq})")
    _same_device(dev, starts=batch.starts, q=q, out=out, lse=lse)
    ws, nbytes = _scratch(dev, stream, 0 if workspace is not None else lb_kv_attend_workspace(cache, batch, hq), workspace, "lb_kv_attend")
    _call(dev, stream, "lb_kv_attend", cache.ref, batch.ref, dt, hq, q.data_ptr(), qs, scale, window, out.data_ptr(), os,
          _ptr(lse), _ptr(ws), nbytes)
    return out, lse


def lb_lora_workspace(rows: int, d_in: int, d_out: int, rank: int) -> int:
    lbm = _binding()
    need = ctypes.c_int64()
    lbm._check(lbm.lib().lb_lora_workspace(rows, d_in, d_out, rank, ctypes.addressof(need)))
    return need.value


def lb_lora_add(y, x, a, b, adapter, scale=None, out=None, workspace=None, stream=None):
    """y [rows, d_out] + scale[adapter] * b[adapter] (a[adapter] x), x [rows, d_in], a [n, rank, d_in],
    b [n, d_out, rank], adapter int32 [rows], scale float32 [n] or None.  Written to `out` (None: y itself),
    which is returned."""
    import torch
    dt, dev = _dtype(y, "y"), y.device
    if x.dim() != 2 or y.dim() != 2 or a.dim() != 3 or b.dim() != 3:
        _bad("x and y must have 2 dimensions, a and b 3")
    rows, d_in, d_out, (n, rank) = y.shape[0], x.shape[1], y.shape[1], a.shape[:2]
    out = y if out is None else out
    xs, ys, os = _rows(x, "x", rows, d_in, y.dtype), _rows(y, "y", rows, d_out, y.dtype), _rows(out, "out", rows, d_out, y.dtype)
    if a.dtype != y.dtype or tuple(a.shape) != (n, rank, d_in) or not a.is_contiguous():
        _bad(f"a must be contiguous {y.dtype} ({n}, {rank}, {d_in})")
    if b.dtype != y.dtype or tuple(b.shape) != (n, d_out, rank) or not b.is_contiguous():
        _bad(f"b must be contiguous {y.dtype} ({n}, {d_out}, {rank})")
    _ints(adapter, "adapter", (rows,))
    if scale is not None and (scale.dtype != torch.float32 or tuple(scale.shape) != (n,) or not scale.is_contiguous()):
        _bad(f"scale must be contiguous float32 ({n},)")
    _same_device(dev, x=x, a=a, b=b, adapter=adapter, scale=scale, out=out)
    ws, nbytes = _scratch(dev, stream, 0 if workspace is not None else lb_lora_workspace(rows, d_in, d_out, rank), workspace, "lb_lora_add")
    _call(dev, stream, "lb_lora_add", dt, rows, d_in, d_out, rank, n, x.data_ptr(), xs, y.data_ptr(), ys, a.data_ptr(),
          b.data_ptr(), adapter.data_ptr(), _ptr(scale), out.data_ptr(), os, _ptr(ws), nbytes)
    return out


def lb_logits_workspace(rows: int, classes: int) -> int:
    lbm = _binding()
    need = ctypes.c_int64()
    lbm._check(lbm.lib().lb_logits_workspace(rows, classes, ctypes.addressof(need)))
    return need.value


def lb_logits_adjust(logits, rules: Optional[LogitRules] = None, target=None, want_logprobs: bool = True, logprobs=None,
                     workspace=None, stream=None):
    """Adjusted log-probabilities of logits [rows, classes].  Returns (logprobs, score, lse): float32
    [rows, classes] (None unless wanted or given), float32 [rows] at target int32 [rows] (None without
    one), and float32 [rows]."""
    import torch
    dt, dev = _dtype(logits, "logits"), logits.device
    if logits.dim() != 2:
        _bad("logits must have 2 dimensions")
    rows, classes = logits.shape
    stride = _rows(logits, "logits", rows, classes, logits.dtype)
    os = classes
    if logprobs is None and want_logprobs:
        logprobs = _empty(logits, stream, (rows, classes), torch.float32)
    if logprobs is not None:
        os = _rows(logprobs, "logprobs", rows, classes, torch.float32)
    score = None
    if target is not None:
        _ints(target, "target", (rows,))
        score = _empty(logits, stream, (rows,), torch.float32)
    lse = _empty(logits, stream, (rows,), torch.float32)
    ref = None
    if rules is not None:
        if rules.history is not None and rules.history.shape[0] != rows:
            _bad(f"history has {rules.history.shape[0]} rows, the logits {rows}")
        if rules.bias_ids is not None:
            if rules.bias_ids.shape[0] not in (1, rows):
                _bad(f"bias_ids has {rules.bias_ids.shape[0]} rows, the logits {rows}")
            rules.desc.bias_per_row = int(rules.bias_ids.shape[0] != 1)
        if rules.mask is not None and rules.mask.shape[1] != (classes + 31) // 32:
            _bad(f"mask has {rules.mask.shape[1]} words a row, expected {(classes + 31) // 32}")
        if rules.mask_row is not None and rules.mask_row.shape[0] != rows:
            _bad(f"mask_row has {rules.mask_row.shape[0]} entries, expected {rows}")
        _same_device(dev, history=rules.history, bias_ids=rules.bias_ids, bias_values=rules.bias_values, mask=rules.mask,
                     mask_row=rules.mask_row)
        ref = rules.ref
    _same_device(dev, target=target, logprobs=logprobs)
    ws, nbytes = _scratch(dev, stream, 0 if workspace is not None else lb_logits_workspace(rows, classes), workspace, "lb_logits_adjust")
    _call(dev, stream, "lb_logits_adjust", dt, rows, classes, logits.data_ptr(), stride, ref, _ptr(target), _ptr(logprobs), os,
          _ptr(score), _ptr(lse), _ptr(ws), nbytes)
    return logprobs, score, lse
