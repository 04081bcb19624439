"""The attention calls of libqmoe.so (include/qattn.h) on torch tensors: argument marshalling only.

Queries, keys, values and outputs are bfloat16 tensors [tokens, heads, dim] with any token and head stride (multiples of 8
elements) and dense heads.  Outputs are the caller's tensors.  All tensors of a call are on one device, which need not be the current
one; the call enqueues on PyTorch's current stream of that device.  A tensor that belongs to another stream's work is the caller's to order, as
with any kernel."""
from __future__ import annotations

import ctypes as C
import struct
import threading
from typing import Optional

import torch

from .binding import MOE_E_ARG, MoeError, _check, lib

ATTN_BF16, ATTN_FP8 = 0, 1
ATTN_ROPE = {"half": 0, "interleaved": 1}
ATTN_SCALE = {"none": 0, "linear": 1, "base": 2, "ramp": 3, "waves": 4}


class _Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("n_pages", C.c_int32),
                ("heads_kv", C.c_int32), ("page_tokens", C.c_int32), ("dim", C.c_int32), ("format", C.c_int32)]


class _Rope(C.Structure):
    _fields_ = [("inv_freq", C.c_void_p), ("dims", C.c_int32), ("layout", C.c_int32), ("mscale", C.c_float)]


# attn_rows and attn_place are passed as slices of one array of 64-bit numbers, a thread's own, written anew by every call: a structure
# object for each of a call's tensors costs more than its kernel's launch, an array object a call a tenth of the call.
_ROWS, _PLACE = 3, 4
_MOST = 5 * _ROWS + _PLACE
_pack2, _pack2p, _pack4, _pack5p = (struct.Struct(f"{n}q").pack_into for n in (2 * _ROWS, 2 * _ROWS + _PLACE, 4 * _ROWS, _MOST))


class _Numbers(threading.local):
    def __init__(self):
        self.to = (C.c_int64 * _MOST)()
        self.at = C.addressof(self.to)


_numbers = _Numbers()

_ready = None


def _lib():
    global _ready
    if _ready is None:
        L = lib()
        P, I, F = C.c_void_p, C.c_int32, C.c_float
        L.attn_rope_frequencies.argtypes = [I, C.c_double, I, C.c_double, C.c_double, C.c_double, C.c_double, P, C.POINTER(F)]
        L.attn_append.argtypes = [P, P, P, P, P, P, I, I, P, P, P, P]
        L.attn_read.argtypes = [P, P, I, P, P, P, P]
        L.attn_prompt.argtypes = [P, P, P, P, P, P, P, I, I, I, I, I, I, F, I, P, C.c_size_t, P]
        L.attn_decode.argtypes = [P, P, P, P, I, I, P, I, P, F, P, C.c_size_t, P, P]
        for f in ("attn_rope_frequencies", "attn_append", "attn_read", "attn_prompt", "attn_decode"):
            getattr(L, f).restype = I
        for f, n in (("attn_prompt_workspace_bytes", 6), ("attn_decode_workspace_bytes", 4), ("attn_decode_counter_bytes", 3)):
            getattr(L, f).argtypes = [I] * n
            getattr(L, f).restype = C.c_size_t
        _ready = L
    return _ready


def _bad(text: str):
    raise MoeError(MOE_E_ARG, text)


def _device(t, name: str) -> int:
    d = t.get_device()
    if d < 0:
        _bad(f"{name} must be on the GPU")
    return d


def _heads(t, name: str, T: int, H: int, D: int, dev: Optional[int] = None):
    """A bfloat16 tensor [T, H, D] on this device (None: any) as rows: address, token stride, head stride."""
    if dev is None:
        dev = _device(t, name)
    if t.dtype is not torch.bfloat16 or t.shape != (T, H, D) or t.get_device() != dev:
        _bad(f"{name} must be a bfloat16 tensor {[T, H, D]} on GPU {dev}, not {t.dtype} {list(t.shape)} on {t.device}")
    ts, hs, ds = t.stride()
    if ds != 1:
        _bad(f"the elements of a head of {name} must be dense")
    return t.data_ptr(), ts if T > 1 else 0, hs if H > 1 else 0


def _whole(t, name: str, dtype, shape, dev: int) -> int:
    """The address of a dense tensor of this type and shape on this device."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _bad(f"{name} must be a dense {dtype} tensor {list(shape)} on GPU {dev}, not {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def _optional(t, name: str, dtype, shape, dev: int):
    return None if t is None else _whole(t, name, dtype, shape, dev)


def _three(t, name: str):
    s = t.shape
    if len(s) != 3:
        _bad(f"{name} must be [tokens, heads, dim]")
    if s[0] >> 31:
        _long(name)
    return s


def _long(name: str):
    """Counts are int32 in the library; ctypes would cut them off."""
    _bad(f"{name} has 2^31 rows or more")


# torch.cuda.current_stream() builds a stream object, 2 us of a call's 8.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _enqueue(f, dev: int, *args) -> int:
    """f(*args, stream) on the current stream of this device, with the device current: a launch on a default stream goes to the current device's."""
    if _current_device() == dev:
        return _check(f(*args, _raw_stream(dev)))
    with torch.cuda.device(dev):
        return _check(f(*args, _raw_stream(dev)))


class AttnCache:
    """Pages of keys and values: k and v [n_pages, heads_kv, page_tokens, dim], bfloat16, or float8_e4m3fn (or its bytes as uint8)
    with the scale bytes k_scale and v_scale [n_pages, heads_kv, page_tokens]."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        if k.dim() != 4:
            _bad("k must be [n_pages, heads_kv, page_tokens, dim]")
        if k.dtype not in (torch.bfloat16, torch.float8_e4m3fn, torch.uint8):
            _bad("a cache is bfloat16 or float8_e4m3fn")
        shape = tuple(k.shape)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.heads_kv, self.page_tokens, self.dim = shape
        self.fp8 = k.dtype != torch.bfloat16
        if self.fp8 != (k_scale is not None) or self.fp8 != (v_scale is not None):
            _bad("a float8 cache needs k_scale and v_scale, a bfloat16 cache has none")
        self._device = d = _device(k, "k")
        self._c = _Cache(_whole(k, "k", k.dtype, shape, d), _whole(v, "v", k.dtype, shape, d), _optional(k_scale, "k_scale", torch.uint8, shape[:3], d),
                         _optional(v_scale, "v_scale", torch.uint8, shape[:3], d), *shape, ATTN_FP8 if self.fp8 else ATTN_BF16)
        self._at = C.addressof(self._c)

    @classmethod
    def empty(cls, n_pages: int, heads_kv: int, page_tokens: int, dim: int, fp8: bool = False, device="cuda:0") -> "AttnCache":
        """A cache in memory of its own; its slots hold nothing until tokens are appended."""
        shape = (n_pages, heads_kv, page_tokens, dim)
        k, v = (torch.empty(shape, dtype=torch.uint8 if fp8 else torch.bfloat16, device=device) for _ in range(2))
        return cls(k, v, *((torch.empty(shape[:3], dtype=torch.uint8, device=device) for _ in range(2)) if fp8 else ()))


class AttnRope:
    """Rotary positions: inv_freq [dims/2] float64 on the GPU (see attn_rope_frequencies), pairs "half" a rotation apart or
    "interleaved", mscale on cos and sin."""

    def __init__(self, inv_freq, layout: str = "half", mscale: float = 1.0):
        if layout not in ATTN_ROPE:
            _bad("layout must be half or interleaved")
        self.inv_freq = inv_freq
        self._device = _device(inv_freq, "inv_freq")
        self._c = _Rope(_whole(inv_freq, "inv_freq", torch.float64, (inv_freq.numel(),), self._device), 2 * inv_freq.numel(), ATTN_ROPE[layout], mscale)
        self._at = C.addressof(self._c)


def attn_rope_frequencies(dims: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained: float = 4096.0,
                          fast: float = 32.0, slow: float = 1.0):
    """(frequencies as a list, factor on cos and sin); the scalings are those of include/qattn.h.  Host only."""
    if scaling not in ATTN_SCALE:
        _bad(f"scaling must be one of {', '.join(ATTN_SCALE)}")
    f, m = (C.c_double * max(1, dims // 2))(), C.c_float()
    _check(_lib().attn_rope_frequencies(dims, base, ATTN_SCALE[scaling], factor, trained, fast, slow, f, C.byref(m)))
    return list(f), float(m.value)


def _place(seq, pos, pages, T: int, dev: int):
    """seq, pos and pages as attn_place."""
    if pages.dim() != 2:
        _bad("pages must be [n_seqs, seq_pages]")
    n, m = pages.shape
    if (n | m) >> 31:
        _long("pages")
    return (_optional(seq, "seq", torch.int32, (T,), dev) or 0, _whole(pos, "pos", torch.int32, (T,), dev), _whole(pages, "pages", torch.int32, (n, m), dev), n | m << 32)


def attn_append(cache: AttnCache, q, k, v, seq, pos, pages, rope: Optional[AttnRope], q_out, k_out=None, bad=None) -> int:
    """Rotates q into q_out and k into k_out (may be None) and writes k and v to the cache.  seq (None: token t is sequence t's),
    pos int32 [tokens], pages int32 [n_seqs, seq_pages]; bad int32 [1] counts tokens that are out of range.  q and q_out may be None.
    No two tokens of a call have the same slot: what it holds afterwards is not specified."""
    T, Hk, D, dev = _three(k, "k")[0], cache.heads_kv, cache.dim, cache._device
    if (q is None) != (q_out is None):
        _bad("q and q_out go together")
    if rope is not None and rope._device != dev:
        _bad(f"inv_freq must be on GPU {dev}")
    Hq = 0 if q is None else _three(q, "q")[1]
    none = (0, 0, 0)
    w = _numbers
    _pack5p(w.to, 0, *_heads(k, "k", T, Hk, D, dev), *_heads(v, "v", T, Hk, D, dev), *_place(seq, pos, pages, T, dev),
            *(none if q is None else _heads(q, "q", T, Hq, D, dev)), *(none if q is None else _heads(q_out, "q_out", T, Hq, D, dev)),
            *(none if k_out is None else _heads(k_out, "k_out", T, Hk, D, dev)))
    at = w.at
    return _enqueue(_lib().attn_append, dev, cache._at, at + 80 if q is not None else None, at, at + 24, at + 104 if q is not None else None,
                    at + 128 if k_out is not None else None, Hq, T, at + 48, None if rope is None else rope._at,
                    _optional(bad, "bad", torch.int32, (1,), dev))


def attn_read(cache: AttnCache, seq, pos, pages, k_out, v_out, bad=None) -> int:
    """Keys and values of the tokens at (seq, pos) out of the cache, as bfloat16."""
    T, Hk, D, dev = pos.shape[0], cache.heads_kv, cache.dim, cache._device
    if T >> 31:
        _long("pos")
    w = _numbers
    _pack2p(w.to, 0, *_heads(k_out, "k_out", T, Hk, D, dev), *_heads(v_out, "v_out", T, Hk, D, dev), *_place(seq, pos, pages, T, dev))
    at = w.at
    return _enqueue(_lib().attn_read, dev, cache._at, at + 48, T, at, at + 24, _optional(bad, "bad", torch.int32, (1,), dev))


def attn_prompt(q, k, v, cu_q, cu_k, out, scale: Optional[float] = None, causal: bool = True, lse=None) -> int:
    """Attention over packed prompts; cu_q, cu_k int32 [n_seqs + 1] on the GPU; scale None: dim ** -0.5; lse float32 [n_q, heads_q].
    Where queries are few and keys many the call takes scratch memory from PyTorch's allocator, for the time of its kernels."""
    (n_q, Hq, D), (n_k, Hk, _) = _three(q, "q"), _three(k, "k")
    n = cu_q.shape[0] - 1
    if n >> 31 > 0:
        _long("cu_q")
    if n < 0:
        _bad("cu_q has no entry")
    L, dev = _lib(), _device(q, "q")
    w = _numbers
    _pack4(w.to, 0, *_heads(q, "q", n_q, Hq, D, dev), *_heads(k, "k", n_k, Hk, D, dev), *_heads(v, "v", n_k, Hk, D, dev), *_heads(out, "out", n_q, Hq, D, dev))
    nb = L.attn_prompt_workspace_bytes(n, n_q, n_k, Hq, Hk, D)
    ws = None if nb == 0 else torch.empty(nb, dtype=torch.uint8, device=q.device)
    at = w.at
    return _enqueue(L.attn_prompt, dev, at, at + 24, at + 48, at + 72, _optional(lse, "lse", torch.float32, (n_q, Hq), dev),
                    _whole(cu_q, "cu_q", torch.int32, (n + 1,), dev), _whole(cu_k, "cu_k", torch.int32, (n + 1,), dev), n, n_q, n_k, Hq, Hk, D,
                    D ** -0.5 if scale is None else scale, 1 if causal else 0, None if ws is None else ws.data_ptr(), nb)


def attn_decode_workspace(cache: AttnCache, n_seqs: int, heads_q: int):
    """Workspace for attn_decode calls of up to n_seqs sequences, its counters zeroed; for one stream at a time, and passed whole by each call."""
    n = int(_lib().attn_decode_workspace_bytes(n_seqs, heads_q, cache.heads_kv, cache.dim))
    if n == 0:
        raise MoeError(MOE_E_ARG, _lib().moe_last_error().decode())
    return torch.zeros(n, dtype=torch.uint8, device=cache.k.device)


def attn_decode(cache: AttnCache, q, pages, lens, out, workspace, scale: Optional[float] = None, lse=None, bad=None) -> int:
    """One query a sequence (q [n_seqs, heads_q, dim]) over the first lens[b] tokens of its pages."""
    n, Hq, D = _three(q, "q")
    if pages.dim() != 2 or D != cache.dim:
        _bad("pages must be [n_seqs, seq_pages], q [n_seqs, heads_q, dim of the cache]")
    m, nb, dev = pages.shape[1], workspace.numel(), cache._device
    if m >> 31:
        _long("pages")
    w = _numbers
    _pack2(w.to, 0, *_heads(q, "q", n, Hq, D, dev), *_heads(out, "out", n, Hq, D, dev))
    at = w.at
    return _enqueue(_lib().attn_decode, dev, cache._at, at, at + 24, _optional(lse, "lse", torch.float32, (n, Hq), dev), n, Hq,
                    _whole(pages, "pages", torch.int32, (n, m), dev), m, _whole(lens, "lens", torch.int32, (n,), dev),
                    D ** -0.5 if scale is None else scale, _whole(workspace, "workspace", torch.uint8, (nb,), dev), nb,
                    _optional(bad, "bad", torch.int32, (1,), dev))
