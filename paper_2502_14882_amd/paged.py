"""The paged 8-bit KV cache of libcq (include/cq_paged.h): same names as the C ABI, argument marshalling only.

What a serving program keeps between steps - the cache, its view of the batch, the rotary frequencies - is an object made once
(PagedCache, PagedBatch, Rope); their tensors are checked then, and their C structs built.  The calls

    cqp_rotate      turn queries and keys by their positions (or gradients back)
    cqp_append_kv   write new keys and values into the pages, turn the step's queries beside them
    cqp_attn        attend to the cache

run on the current stream of the tensors' device.  There is no fallback: if libcq.so is missing or a call fails, an exception is
raised.
"""
from __future__ import annotations

import ctypes
import struct
from typing import Optional, Sequence, Tuple, Union

import torch

from . import binding
from .binding import CqError  # noqa: F401  (what the calls raise)

CQP_F16, CQP_BF16 = 0, 1
CQP_PAIRS_HALVES, CQP_PAIRS_ADJACENT = 0, 1
PAGES = (16, 32, 64, 128, 256)

_DTYPES = {torch.float16: CQP_F16, torch.bfloat16: CQP_BF16}


class CqpHeads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("n_heads", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class CqpCache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "page", "n_kv_heads", "head_dim")] + \
               [(n, ctypes.c_void_p) for n in ("k_codes", "v_codes", "k_scale", "v_scale")]


class CqpBatch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "max_pages", "max_new", "max_len")] + \
               [(n, ctypes.c_void_p) for n in ("page_table", "seq_lens", "q_start")]


class CqpRope(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rot_dim", "n_axes", "pairs", "reserved")] + \
               [("inv_freq", ctypes.c_void_p), ("axis_of", ctypes.c_uint8 * 128)]


_fns = None


class _Calls:
    """The library's cqp_* functions, as function objects of their own that take every struct as an address or as packed bytes."""
    __slots__ = ("rotate", "append_kv", "attn_workspace_bytes", "attn")

    def __init__(self, L):
        I, V, S = ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
        for name, result, args in (("rotate", ctypes.c_int, [V, V, I, I, I, I, V, V, I, V]),
                                   ("append_kv", ctypes.c_int, [V, V, I, I, V, V, V, V, V, V, V]),
                                   ("attn_workspace_bytes", S, [V, V, I, I]),
                                   ("attn", ctypes.c_int, [V, V, I, I, V, V, V, I, ctypes.c_float, V, S, V])):
            f = L["cqp_" + name]
            f.restype, f.argtypes = result, args
            setattr(self, name, f)


_packed: Optional[_Calls] = None


def _calls() -> _Calls:
    global _packed
    if _packed is None or binding._lib is None:
        _packed = _Calls(binding.lib())
    return _packed


def lib():
    """The library's cqp_* functions (cq_* ones: binding.lib())."""
    global _fns
    if _fns is None or binding._lib is None:
        L = binding.lib()
        P, I, V = ctypes.POINTER, ctypes.c_int32, ctypes.c_void_p
        heads, cache, batch, rope = P(CqpHeads), P(CqpCache), P(CqpBatch), P(CqpRope)
        L.cqp_rotate.restype = ctypes.c_int
        L.cqp_rotate.argtypes = [rope, V, I, I, I, I, heads, heads, I, V]
        L.cqp_append_kv.restype = ctypes.c_int
        L.cqp_append_kv.argtypes = [cache, batch, I, I, heads, heads, rope, V, heads, heads, V]
        L.cqp_attn_workspace_bytes.restype = ctypes.c_size_t
        L.cqp_attn_workspace_bytes.argtypes = [cache, batch, I, I]
        L.cqp_attn.restype = ctypes.c_int
        L.cqp_attn.argtypes = [cache, batch, I, I, heads, heads, V, I, ctypes.c_float, V, ctypes.c_size_t, V]
        _fns = L
    return _fns


def _need(ok: bool, text: str, *args) -> None:
    if not ok:
        raise ValueError(text % args)


class PagedCache:
    """The pages: codes float8_e4m3fn (or uint8) [n_pages, Hkv, page, d] of the keys and [n_pages, Hkv, d, page] of the values,
    scales float32 [n_pages, Hkv].  Nothing has to be cleared."""
    __slots__ = ("k_codes", "v_codes", "k_scale", "v_scale", "n_pages", "page", "n_kv_heads", "head_dim", "device", "index", "c", "at")

    def __init__(self, k_codes: torch.Tensor, v_codes: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        _need(k_codes.dim() == 4, "k_codes are %s, [n_pages, Hkv, page, d] is wanted", tuple(k_codes.shape))
        self.n_pages, self.n_kv_heads, self.page, self.head_dim = k_codes.shape
        _need(v_codes.shape == (self.n_pages, self.n_kv_heads, self.head_dim, self.page),
              "v_codes are %s, [n_pages, Hkv, d, page] is wanted", tuple(v_codes.shape))
        for t in (k_codes, v_codes):
            _need(t.dtype in (torch.float8_e4m3fn, torch.uint8), "codes are float8_e4m3fn or uint8, not %s", t.dtype)
        for t in (k_scale, v_scale):
            _need(t.dtype == torch.float32 and t.shape == (self.n_pages, self.n_kv_heads),
                  "scales are float32 [n_pages, Hkv], not %s %s", t.dtype, tuple(t.shape))
        _need(self.page in PAGES, "a page holds 16, 32, 64, 128 or 256 tokens, not %d", self.page)
        for t in (k_codes, v_codes, k_scale, v_scale):
            _need(t.is_contiguous() and t.device == k_codes.device, "the cache's tensors are contiguous and on one device")
        self.k_codes, self.v_codes, self.k_scale, self.v_scale = k_codes, v_codes, k_scale, v_scale
        self.device = k_codes.device
        self.c = CqpCache(self.n_pages, self.page, self.n_kv_heads, self.head_dim, k_codes.data_ptr(), v_codes.data_ptr(),
                          k_scale.data_ptr(), v_scale.data_ptr())
        self.index, self.at = k_codes.get_device(), ctypes.addressof(self.c)


def alloc_cache(n_pages: int, n_kv_heads: int, head_dim: int, page: int = 64, device="cuda") -> PagedCache:
    shape = (n_pages, n_kv_heads)
    return PagedCache(torch.empty(shape + (page, head_dim), dtype=torch.float8_e4m3fn, device=device),
                      torch.empty(shape + (head_dim, page), dtype=torch.float8_e4m3fn, device=device),
                      torch.empty(shape, dtype=torch.float32, device=device),
                      torch.empty(shape, dtype=torch.float32, device=device))


class PagedBatch:
    """The sequences of a step: page_table int32 [B, max_pages], seq_lens int32 [B] (tokens in the cache, the new ones
    included), q_start int32 [B + 1] (rows of the new tokens), all on the device, and the host's bounds of the new
    tokens of a sequence and of seq_lens.  The tensors' contents may change between calls (and replays)."""
    __slots__ = ("page_table", "seq_lens", "q_start", "max_new", "max_len", "device", "index", "c", "at")

    def __init__(self, page_table: torch.Tensor, seq_lens: torch.Tensor, q_start: torch.Tensor, max_new: int, max_len: int):
        _need(page_table.dim() == 2, "page_table is %s, [B, max_pages] is wanted", tuple(page_table.shape))
        b = page_table.shape[0]
        _need(seq_lens.shape == (b,) and q_start.shape == (b + 1,), "seq_lens is %s and q_start %s for %d sequences",
              tuple(seq_lens.shape), tuple(q_start.shape), b)
        for t in (page_table, seq_lens, q_start):
            _need(t.dtype == torch.int32 and t.is_contiguous() and t.device == page_table.device,
                  "the batch's tensors are contiguous int32 on one device")
        self.page_table, self.seq_lens, self.q_start = page_table, seq_lens, q_start
        self.max_new, self.max_len, self.device = int(max_new), int(max_len), page_table.device
        self.c = CqpBatch(b, page_table.shape[1], self.max_new, self.max_len, page_table.data_ptr(), seq_lens.data_ptr(),
                          q_start.data_ptr())
        self.index, self.at = page_table.get_device(), ctypes.addressof(self.c)


class Rope:
    """Rotary frequencies: inv_freq float32 [rot_dim / 2] on the device; axis_of says which axis of the positions each of them
    belongs to (None: one axis); pairs: CQP_PAIRS_HALVES or CQP_PAIRS_ADJACENT."""
    __slots__ = ("inv_freq", "n_axes", "device", "index", "c", "at")

    def __init__(self, inv_freq: torch.Tensor, axis_of: Optional[Sequence[int]] = None, pairs: int = CQP_PAIRS_HALVES,
                 n_axes: Optional[int] = None):
        _need(inv_freq.dim() == 1 and inv_freq.dtype == torch.float32 and inv_freq.is_contiguous(),
              "inv_freq is a contiguous float32 vector")
        half = inv_freq.shape[0]
        axis_of = [0] * half if axis_of is None else [int(a) for a in axis_of]
        _need(len(axis_of) == half and half <= 128, "axis_of has %d entries for %d frequencies (at most 128)", len(axis_of), half)
        _need(all(0 <= a < 4 for a in axis_of), "axes are 0 to 3")
        self.inv_freq, self.device = inv_freq, inv_freq.device
        self.n_axes = (max(axis_of) + 1 if axis_of else 1) if n_axes is None else int(n_axes)
        self.c = CqpRope(2 * half, self.n_axes, int(pairs), 0, inv_freq.data_ptr(), (ctypes.c_uint8 * 128)(*axis_of))
        self.index, self.at = inv_freq.get_device(), ctypes.addressof(self.c)


# The checks run on every call, in the time the GPU could already be working: texts are only made on failure, devices are compared
# by index, rows of heads are packed as bytes.

_pack_heads = struct.Struct("PqqiI").pack            # a cqp_heads_t


def _heads(t: torch.Tensor, what: str, head_dim: int, n_tokens: int, dtype, index: int) -> bytes:
    shape = t.shape
    if len(shape) != 3 or shape[2] != head_dim or shape[0] != n_tokens:
        raise ValueError("%s is %s, [%d, heads, %d] is wanted" % (what, tuple(shape), n_tokens, head_dim))
    if t.dtype is not dtype or t.get_device() != index:
        raise ValueError("%s is %s on %s, the call's are %s on GPU %d" % (what, t.dtype, t.device, dtype, index))
    token, head, channel = t.stride()
    if channel != 1:
        raise ValueError("the channels of %s are not contiguous" % what)
    heads = shape[1]
    # a dimension of one entry is never stepped over, whatever stride it has
    return _pack_heads(t.data_ptr(), token if n_tokens > 1 else 0, head if heads > 1 else 0, heads, 0)


def _own_heads(t: torch.Tensor) -> bytes:
    """The same of a tensor that was allocated here, dense."""
    _, heads, d = t.shape
    return _pack_heads(t.data_ptr(), heads * d, d, heads, 0)


def _dtype(t: torch.Tensor) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError("elements are float16 or bfloat16, not %s" % t.dtype)
    return code


def _positions(positions: torch.Tensor, rope: Rope, n_tokens: int, index: int) -> int:
    shape = positions.shape
    if (positions.dtype is not torch.int32 or not positions.is_contiguous() or positions.get_device() != index
            or (shape != (rope.n_axes, n_tokens) and not (rope.n_axes == 1 and shape == (n_tokens,)))):
        raise ValueError("positions are %s %s on %s, contiguous int32 [%d, %d] is wanted" % (
            positions.dtype, tuple(shape), positions.device, rope.n_axes, n_tokens))
    if rope.index != index:
        raise ValueError("the rope's frequencies are on %s, the call's tensors on GPU %d" % (rope.device, index))
    return positions.data_ptr()


def _dense_like(t: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _run(index: int, call, *args) -> None:
    """One call on the current stream of GPU `index`, which is made the current one for it."""
    if index < 0:
        raise ValueError("the tensors are on the CPU, a GPU is wanted")
    if index == torch._C._cuda_getDevice():
        status = call(*args, torch._C._cuda_getCurrentRawStream(index) or None)
    else:
        with torch.cuda.device(index):
            status = call(*args, torch._C._cuda_getCurrentRawStream(index) or None)
    if status:
        binding._check(status)


def cqp_rotate(rope: Rope, positions: torch.Tensor, x: Union[torch.Tensor, Sequence[torch.Tensor]], out=None,
               backward: bool = False):
    """Turn the heads of x - a tensor [tokens, heads, d], or two of them (queries and keys) - by their positions int32 [n_axes,
    tokens]; backward: by the opposite angles, which takes the gradient of the result to that of x.  out: like x (x itself:
    in place), allocated here if None.  Returns out."""
    single = isinstance(x, torch.Tensor)
    xs = (x,) if single else tuple(x)
    if not 1 <= len(xs) <= 2:
        raise ValueError("one or two tensors are turned at once, not %d" % len(xs))
    first = xs[0]
    shape, dtype, index = first.shape, first.dtype, first.get_device()
    if len(shape) != 3:
        raise ValueError("x is %s, [tokens, heads, d] is wanted" % (tuple(shape),))
    n, _, d = shape
    ins = b"".join([_heads(t, "x", d, n, dtype, index) for t in xs])
    if out is None:
        outs = [_dense_like(t) for t in xs]
        res = b"".join([_own_heads(t) for t in outs])
    else:
        outs = [out] if single else list(out)
        if len(outs) != len(xs):
            raise ValueError("%d tensors, %d results" % (len(xs), len(outs)))
        res = b"".join([_heads(t, "out", d, n, dtype, index) for t in outs])
    _run(index, _calls().rotate, rope.at, _positions(positions, rope, n, index), n, d, _dtype(first), 1 if backward else 0, ins, res,
         len(xs))
    return outs[0] if single else outs


def _check_step(cache: PagedCache, batch: PagedBatch) -> None:
    if cache.index != batch.index:
        raise ValueError("the cache is on %s, the batch on %s" % (cache.device, batch.device))


def cqp_append_kv(cache: PagedCache, batch: PagedBatch, k: torch.Tensor, v: torch.Tensor, rope: Optional[Rope] = None,
                  positions: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
                  q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Write the new keys and values [tokens, Hkv, d] into the cache, the keys turned by `positions` if a rope is given; with q
    [tokens, Hq, d] the queries are turned in the same launch, into q_out (q itself: in place; allocated here if None), which is
    returned."""
    _check_step(cache, batch)
    n, d, index, dtype = k.shape[0], cache.head_dim, cache.index, k.dtype
    ks, vs = _heads(k, "k", d, n, dtype, index), _heads(v, "v", d, n, dtype, index)
    if (rope is None) != (positions is None):
        raise ValueError("rope and positions go together")
    where = turn = qs = os = None
    if rope is not None:
        turn, where = rope.at, _positions(positions, rope, n, index)
    if q is not None:
        if rope is None:
            raise ValueError("queries are turned by a rope: none is given")
        qs = _heads(q, "q", d, n, dtype, index)
        if q_out is None:
            q_out = _dense_like(q)
            os = _own_heads(q_out)
        else:
            os = _heads(q_out, "q_out", d, n, dtype, index)
    elif q_out is not None:
        raise ValueError("q_out without q")
    _run(index, _calls().append_kv, cache.at, batch.at, n, _dtype(k), ks, vs, turn, where, qs, os)
    return q_out


def cqp_attn_workspace_bytes(cache: PagedCache, batch: PagedBatch, n_tokens: int, n_q_heads: int) -> int:
    return int(_calls().attn_workspace_bytes(cache.at, batch.at, int(n_tokens), int(n_q_heads)))


def cqp_attn(cache: PagedCache, batch: PagedBatch, q: torch.Tensor, causal: bool = True, softmax_scale: float = 0.0,
             out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, return_lse: bool = False,
             workspace: Optional[torch.Tensor] = None) -> Union[torch.Tensor, Tuple[torch.Tensor, torch.Tensor]]:
    """Attention of the new tokens' queries [tokens, Hq, d] over the cache; returns out [tokens, Hq, d], and with return_lse
    (or lse, a float32 [tokens, Hq] to write to) the logarithms of the rows' sums of weights.  Rows behind the last sequence
    are not written (those of an `out` allocated here are undefined)."""
    _check_step(cache, batch)
    shape, dtype, index = q.shape, q.dtype, cache.index
    if len(shape) != 3:
        raise ValueError("q is %s, [tokens, heads, d] is wanted" % (tuple(shape),))
    n, heads, _ = shape
    qs = _heads(q, "q", cache.head_dim, n, dtype, index)
    if out is None:
        out = _dense_like(q)
        os = _own_heads(out)
    else:
        os = _heads(out, "out", cache.head_dim, n, dtype, index)
    if lse is not None:
        if lse.dtype is not torch.float32 or lse.shape != (n, heads) or not lse.is_contiguous() or lse.get_device() != index:
            raise ValueError("lse is a contiguous float32 [tokens, heads] on the cache's device")
    elif return_lse:
        lse = torch.empty((n, heads), dtype=torch.float32, device=q.device)
    calls = _calls()
    if workspace is None:
        workspace = torch.empty(calls.attn_workspace_bytes(cache.at, batch.at, n, heads), dtype=torch.uint8, device=q.device)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError("the workspace is contiguous and on the cache's device")
    _run(index, calls.attn, cache.at, batch.at, n, _dtype(q), qs, os, None if lse is None else lse.data_ptr(), 1 if causal else 0,
         softmax_scale, workspace.data_ptr(), workspace.nbytes)
    return out if lse is None else (out, lse)
