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


def lib():
    """The library's cqp_* functions (cq_* ones: binding.lib())."""
    global _fns
    if _fns is None:
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
    __slots__ = ("k_codes", "v_codes", "k_scale", "v_scale", "n_pages", "page", "n_kv_heads", "head_dim", "device", "c")

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
    __slots__ = ("page_table", "seq_lens", "q_start", "max_new", "max_len", "device", "c")

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


class Rope:
    """Rotary frequencies: inv_freq float32 [rot_dim / 2] on the device; axis_of says which axis of the positions each of them
    belongs to (None: one axis); pairs: CQP_PAIRS_HALVES or CQP_PAIRS_ADJACENT."""
    __slots__ = ("inv_freq", "n_axes", "device", "c")

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


def _heads(t: torch.Tensor, what: str, head_dim: int, n_tokens: int, dtype, device) -> CqpHeads:
    _need(t.dim() == 3 and t.shape[2] == head_dim and t.shape[0] == n_tokens, "%s is %s, [%d, heads, %d] is wanted", what,
          tuple(t.shape), n_tokens, head_dim)
    _need(t.dtype == dtype and t.device == device, "%s is %s on %s, the call's are %s on %s", what, t.dtype, t.device, dtype, device)
    st, sh, sc = t.stride()
    _need(sc == 1, "the channels of %s are not contiguous", what)
    # a dimension of one entry is never stepped over, whatever stride it has
    return CqpHeads(t.data_ptr(), st if t.shape[0] > 1 else 0, sh if t.shape[1] > 1 else 0, t.shape[1], 0)


def _dtype(t: torch.Tensor) -> int:
    code = _DTYPES.get(t.dtype)
    _need(code is not None, "elements are float16 or bfloat16, not %s", t.dtype)
    return code


def _positions(positions: torch.Tensor, rope: Rope, n_tokens: int, device) -> int:
    _need(positions.dtype == torch.int32 and positions.is_contiguous() and positions.device == device
          and positions.numel() == rope.n_axes * n_tokens and positions.shape[-1] == n_tokens and positions.dim() <= 2,
          "positions are %s %s, contiguous int32 [%d, %d] is wanted", positions.dtype, tuple(positions.shape), rope.n_axes, n_tokens)
    _need(rope.device == device, "the rope's frequencies are on %s, the call's tensors on %s", rope.device, device)
    return positions.data_ptr()


def _run(device, call, *args) -> None:
    """One call on the current stream of `device`, which is made the current one for it."""
    if device.type == "cuda":
        if device.index is not None and device.index != torch.cuda.current_device():
            with torch.cuda.device(device):
                status = call(*args, torch._C._cuda_getCurrentRawStream(device.index) or None)
        else:
            status = call(*args, torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None)
    else:
        raise ValueError("the tensors are on %s, a GPU is wanted" % device)
    if status:
        binding._check(status)


def cqp_rotate(rope: Rope, positions: torch.Tensor, x: Union[torch.Tensor, Sequence[torch.Tensor]], out=None,
               backward: bool = False):
    """Turn the heads of x - a tensor [tokens, heads, d], or two of them (queries and keys) - by their positions int32 [n_axes,
    tokens]; backward: by the opposite angles, which takes the gradient of the result to that of x.  out: like x (x itself:
    in place), allocated here if None.  Returns out."""
    single = isinstance(x, torch.Tensor)
    xs = [x] if single else list(x)
    _need(1 <= len(xs) <= 2, "one or two tensors are turned at once, not %d", len(xs))
    outs = [torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in xs] if out is None else [out] if single else list(out)
    _need(len(outs) == len(xs), "%d tensors, %d results", len(xs), len(outs))
    first = xs[0]
    _need(first.dim() == 3, "x is %s, [tokens, heads, d] is wanted", tuple(first.shape))
    n, _, d = first.shape
    args = [(CqpHeads * 2)(*[_heads(t, "x" if ts is xs else "out", d, n, first.dtype, first.device) for t in ts]) for ts in (xs, outs)]
    _run(first.device, lib().cqp_rotate, ctypes.byref(rope.c), _positions(positions, rope, n, first.device), n, d, _dtype(first),
         int(bool(backward)), args[0], args[1], len(xs))
    return outs[0] if single else outs


def _check_step(cache: PagedCache, batch: PagedBatch) -> None:
    _need(cache.device == batch.device, "the cache is on %s, the batch on %s", cache.device, batch.device)


def cqp_append_kv(cache: PagedCache, batch: PagedBatch, k: torch.Tensor, v: torch.Tensor, rope: Optional[Rope] = None,
                  positions: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
                  q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Write the new keys and values [tokens, Hkv, d] into the cache, the keys turned by `positions` if a rope is given; with q
    [tokens, Hq, d] the queries are turned in the same launch, into q_out (q itself: in place; allocated here if None), which is
    returned."""
    _check_step(cache, batch)
    n, d, dev = k.shape[0], cache.head_dim, cache.device
    ks, vs = _heads(k, "k", d, n, k.dtype, dev), _heads(v, "v", d, n, k.dtype, dev)
    _need((rope is None) == (positions is None), "rope and positions go together")
    _need(q is not None or q_out is None, "q_out without q")
    qs = os = None
    if q is not None:
        _need(rope is not None, "queries are turned by a rope: none is given")
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        qs, os = _heads(q, "q", d, n, k.dtype, dev), _heads(q_out, "q_out", d, n, k.dtype, dev)
    _run(dev, lib().cqp_append_kv, ctypes.byref(cache.c), ctypes.byref(batch.c), n, _dtype(k), ctypes.byref(ks),
         ctypes.byref(vs), ctypes.byref(rope.c) if rope is not None else None,
         _positions(positions, rope, n, dev) if rope is not None else None,
         ctypes.byref(qs) if qs is not None else None, ctypes.byref(os) if os is not None else None)
    return q_out


def cqp_attn_workspace_bytes(cache: PagedCache, batch: PagedBatch, n_tokens: int, n_q_heads: int) -> int:
    return int(lib().cqp_attn_workspace_bytes(ctypes.byref(cache.c), ctypes.byref(batch.c), int(n_tokens), int(n_q_heads)))


def cqp_attn(cache: PagedCache, batch: PagedBatch, q: torch.Tensor, causal: bool = True, softmax_scale: float = 0.0,
             out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, return_lse: bool = False,
             workspace: Optional[torch.Tensor] = None) -> Union[torch.Tensor, Tuple[torch.Tensor, torch.Tensor]]:
    """Attention of the new tokens' queries [tokens, Hq, d] over the cache; returns out [tokens, Hq, d], and with return_lse
    (or lse, a float32 [tokens, Hq] to write to) the logarithms of the rows' sums of weights.  Rows behind the last sequence
    are not written (those of an `out` allocated here are undefined)."""
    _check_step(cache, batch)
    _need(q.dim() == 3, "q is %s, [tokens, heads, d] is wanted", tuple(q.shape))
    n, heads, d = q.shape
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None and return_lse:
        lse = torch.empty((n, heads), dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse.dtype == torch.float32 and lse.shape == (n, heads) and lse.is_contiguous() and lse.device == q.device,
              "lse is a contiguous float32 [tokens, heads]")
    dev = cache.device
    qs, os = _heads(q, "q", cache.head_dim, n, q.dtype, dev), _heads(out, "out", cache.head_dim, n, q.dtype, dev)
    _need(out.shape[1] == heads, "out has %d heads, q %d", out.shape[1], heads)
    if workspace is None:
        workspace = torch.empty(cqp_attn_workspace_bytes(cache, batch, n, heads), dtype=torch.uint8, device=dev)
    else:
        _need(workspace.device == dev and workspace.is_contiguous(), "the workspace is contiguous and on the cache's device")
    _run(dev, lib().cqp_attn, ctypes.byref(cache.c), ctypes.byref(batch.c), n, _dtype(q), ctypes.byref(qs), ctypes.byref(os),
         None if lse is None else lse.data_ptr(), int(bool(causal)), float(softmax_scale), workspace.data_ptr(),
         workspace.nbytes)
    return out if lse is None else (out, lse)
