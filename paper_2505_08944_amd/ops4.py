"""The operators on values in 4 bits (OCP MXFP4: blocks of 32 share a power of two):
the quantiser, the dense product with 4-bit weights, and the paged cache of keys
and values with the attention that reads it.

Tensors, streams and devices as in ``ops``: a call runs on the device of its
tensors, on torch's current stream there, and needs no context.  Forward only.
"""

from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple

import torch

from . import _lib as L
from .ops import _CODE, _FN, _Fixed, _int32, _ld, _rows, arg32

# (torch's own types for these bytes are newer than all else that the package needs of it)
_CODES = (torch.uint8, getattr(torch, "float4_e2m1fn_x2", torch.uint8))
_SCALES = (torch.uint8, getattr(torch, "float8_e8m0fnu", torch.uint8))
_F32_BF16 = (torch.float32, torch.bfloat16)


def _bytes_matrix(t, name, dtypes, shape, dev) -> None:
    _rows(t, name, dtypes, shape, dev)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


_seen = {}  # what was checked of the quantiser's tensors: shapes, strides, types and devices


def _checked(key, check) -> None:
    """Runs check() for what was not checked before."""
    if key not in _seen:
        check()
        if len(_seen) >= 1024:
            _seen.clear()
        _seen[key] = True


def _number(n, what: str, call: str) -> int:
    """A whole number as an int: what calls are known by must not change as a tensor's value can."""
    return n if type(n) is int else arg32(n, what, call)


def quantize_mx4(x: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """x [n, k] float32 or bfloat16 to codes [n, (k + 1) // 2] and scales [n, (k +
    31) // 32], both uint8 (``aep_mx4_quantize``).  Rows may be strided."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError("x must be a CUDA (HIP) tensor")
    dev, dtype = x.device, x.dtype

    def check():
        _rows(x, "x", _F32_BF16, (None, None), dev)
        if x.shape[1] < 1:
            raise ValueError(f"x has shape {tuple(x.shape)}")
        _int32(x.shape[1], 1 << 30, "columns", "aep_mx4_quantize")

    _checked((x.shape, x.stride(), dtype, dev), check)
    n, k = x.shape
    if dev.index != L.current_device():
        with torch.cuda.device(dev):
            return quantize_mx4(x)
    codes = torch.empty((n, (k + 1) // 2), dtype=torch.uint8, device=dev)
    scale = torch.empty((n, (k + 31) // 32), dtype=torch.uint8, device=dev)
    st = L.lib().aep_mx4_quantize(x.data_ptr(), _CODE[dtype], _ld(x), n, k, codes.data_ptr(), scale.data_ptr(),
                                  L.raw_stream(dev.index))
    if st:
        L.check(st, "aep_mx4_quantize")
    return codes, scale


def dequantize_mx4(codes: torch.Tensor, scale: torch.Tensor, k: int, *, dtype: torch.dtype = torch.bfloat16,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values [n, k] of codes and scales (``aep_mx4_dequantize``), exactly, as
    bfloat16 or float32."""
    if not isinstance(codes, torch.Tensor) or not codes.is_cuda:
        raise ValueError("codes must be a CUDA (HIP) tensor")
    if not isinstance(scale, torch.Tensor):
        raise ValueError("scale must be a tensor")
    dev = codes.device
    k = _number(k, "k", "aep_mx4_dequantize")

    def check():
        if arg32(k, "k", "aep_mx4_dequantize") < 1:
            raise ValueError(f"k is {k}")
        _bytes_matrix(codes, "codes", _CODES, (None, (k + 1) // 2), dev)
        _bytes_matrix(scale, "scale", _SCALES, (codes.shape[0], (k + 31) // 32), dev)
        if dtype not in _F32_BF16:
            raise ValueError(f"dtype {dtype}, expected torch.bfloat16 or torch.float32")
        if out is not None:
            _rows(out, "out", (dtype,), (codes.shape[0], k), dev)

    _checked((k, codes.shape, codes.stride(), codes.dtype, dev, scale.shape, scale.stride(), scale.dtype, scale.device,
              dtype, out is None or (out.shape, out.stride(), out.dtype, out.device)), check)
    n = codes.shape[0]
    if dev.index != L.current_device():
        with torch.cuda.device(dev):
            return dequantize_mx4(codes, scale, k, dtype=dtype, out=out)
    if out is None:
        out = torch.empty((n, k), dtype=dtype, device=dev)
    st = L.lib().aep_mx4_dequantize(codes.data_ptr(), scale.data_ptr(), n, k, out.data_ptr(), _CODE[dtype], _ld(out),
                                    L.raw_stream(dev.index))
    if st:
        L.check(st, "aep_mx4_dequantize")
    return out


class Linear4(_Fixed):
    """y = f(x W^T + bias) + residual with W [n, k] in 4 bits (``aep_linear4``).

    codes [n, (k + 1) // 2] and scale [n, (k + 31) // 32] as ``quantize_mx4`` makes
    them (uint8, or torch's float4_e2m1fn_x2 and float8_e8m0fnu); k is needed where
    it is odd.  They are laid out anew on the current stream and not kept: later changes to
    them do not count.  bias [n] float32 or bfloat16 is kept, not copied, as
    ``Linear`` keeps its tensors.  x is bfloat16; out_dtype bfloat16 (the default)
    or float32.
    """

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor, k: Optional[int] = None, *,
                 bias: Optional[torch.Tensor] = None, activation: str = "none",
                 out_dtype: torch.dtype = torch.bfloat16):
        if not isinstance(codes, torch.Tensor) or not codes.is_cuda:
            raise ValueError("codes must be a CUDA (HIP) tensor")
        dev = codes.device
        _bytes_matrix(codes, "codes", _CODES, (None, None), dev)
        n, half = codes.shape
        k = 2 * half if k is None else arg32(k, "k", "aep_linear4")
        if n < 1 or k < 1 or half != (k + 1) // 2:
            raise ValueError(f"codes have shape {tuple(codes.shape)}, expected [n, {(k + 1) // 2}] for k = {k}")
        _int32(max(n, k), 1 << 30, "channels", "aep_linear4")
        _bytes_matrix(scale, "scale", _SCALES, (n, (k + 31) // 32), dev)
        if bias is not None:
            _rows(bias, "bias", _F32_BF16, (n,), dev)
        if activation not in _FN:
            raise ValueError(f"activation {activation!r}, expected one of {', '.join(_FN)}")
        if out_dtype not in _F32_BF16:
            raise ValueError(f"out_dtype {out_dtype}, expected torch.bfloat16 or torch.float32")
        self.bias, self.activation, self.out_dtype, self.device = bias, activation, out_dtype, dev
        self.n, self.k = n, k
        self._lib = L.lib()
        need = ctypes.c_size_t()
        L.check(self._lib.aep_linear4_packed_bytes(n, k, ctypes.byref(need)), "aep_linear4_packed_bytes")
        with torch.cuda.device(dev):
            self.packed = torch.empty(need.value, dtype=torch.uint8, device=dev)
            L.check(self._lib.aep_linear4_pack(codes.data_ptr(), scale.data_ptr(), n, k, self.packed.data_ptr(),
                                               L.raw_stream(dev.index)), "aep_linear4_pack")
        self._kept = None if bias is None else (bias.shape, bias.stride(), bias.dtype, bias.device)
        self._calls = {}  # by what is checked of the tensors: what _describe makes of such a call

    def __call__(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [m, k] bfloat16 -> [m, n].  residual [m, n] float32 or bfloat16; out may be
        the residual itself, and must not overlap anything else."""
        dev, bias = self.device, self.bias
        if dev.index != L.current_device():
            with torch.cuda.device(dev):
                return self(x, residual, out)
        if bias is not None and (bias.shape, bias.stride(), bias.dtype, bias.device) != self._kept:
            raise ValueError("the bias has another shape, stride, type or device than it had: make a new Linear4")
        # a call like one before, in all that is checked and in its alignment, needs no checks
        try:
            at = x.data_ptr()
            key = (x.shape, x.stride(), x.dtype, x.device, at & 15,
                   residual is None or (residual.shape, residual.stride(), residual.dtype, residual.device,
                                        residual.data_ptr() & 15),
                   out is None or (out.shape, out.stride(), out.dtype, out.device, out.data_ptr() & 15))
        except AttributeError:
            raise ValueError("x, residual and out must be tensors") from None
        desc, need, shape = self._calls.get(key) or self._describe(key, x, residual, out)
        if out is None:
            out = torch.empty(shape, dtype=self.out_dtype, device=dev)
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None  # held until the launch is in the stream
        st = self._lib.aep_linear4(desc, at, self.packed.data_ptr(), None if bias is None else bias.data_ptr(),
                                   None if residual is None else residual.data_ptr(), out.data_ptr(),
                                   None if ws is None else ws.data_ptr(), need, L.raw_stream(dev.index))
        if st:
            L.check(st, "aep_linear4")
        return out

    def _describe(self, key, x, residual, out):
        """(description, bytes of scratch, shape of the result) of a checked call, kept for the next ones like it."""
        n, k, dev = self.n, self.k, self.device
        _rows(x, "x", (torch.bfloat16,), (None, k), dev)
        m = x.shape[0]
        _int32(m, 1 << 30, "rows", "aep_linear4")
        if residual is not None:
            _rows(residual, "residual", _F32_BF16, (m, n), dev)
        if out is not None:
            _rows(out, "out", (self.out_dtype,), (m, n), dev)
        y_dtype = _CODE[self.out_dtype]
        d = L.Linear4Desc(m, n, k, y_dtype, L.AEP_F32 if self.bias is None else _CODE[self.bias.dtype],
                          y_dtype if residual is None else _CODE[residual.dtype], _FN[self.activation], _ld(x),
                          n if out is None else _ld(out), n if residual is None else _ld(residual))
        b = ctypes.c_size_t()
        # (an output that torch allocates is aligned)
        L.check(self._lib.aep_linear4_workspace(ctypes.byref(d), x.data_ptr(),
                                                None if residual is None else residual.data_ptr(),
                                                16 if out is None else out.data_ptr(), ctypes.byref(b)),
                "aep_linear4_workspace")
        if len(self._calls) >= 1024:
            self._calls.clear()
        call = self._calls[key] = (ctypes.byref(d), b.value, (m, n))
        return call


def _heads(t, name, shape, dev) -> None:
    """A bfloat16 tensor [rows, heads, d] on ``dev`` whose d values are contiguous."""
    if not isinstance(t, torch.Tensor) or t.device != dev:
        raise ValueError(f"{name} must be a tensor on {dev}")
    if t.dtype != torch.bfloat16:
        raise ValueError(f"{name} has dtype {t.dtype}, expected torch.bfloat16")
    if t.dim() != 3 or any(s is not None and s != h for s, h in zip(shape, t.shape)):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
    if t.stride(2) != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")


def _tables(pages, lens, rows, flag):
    """What is checked of a call's sequences."""
    return (pages.shape, pages.stride(), pages.dtype, pages.device, lens.shape, lens.stride(), lens.dtype, lens.device,
            rows is None or (rows.shape, rows.stride(), rows.dtype, rows.device),
            flag is None or (flag.shape, flag.stride(), flag.dtype, flag.device))


def _seqs(pages, lens, rows, flag, sizes):
    return ctypes.byref(L.Cache4Seqs(pages.data_ptr(), lens.data_ptr(), None if rows is None else rows.data_ptr(),
                                     None if flag is None else flag.data_ptr(), *sizes))


class Cache4(_Fixed):
    """A paged cache of keys and values in 4 bits (``aep_cache4``) and the attention
    over it.

    n_pages pages of page_size tokens (a power of two from 32 on) of n_heads heads
    of head_dim (64, 128 or 256) values.  ``data`` holds it all.

    The calls name their sequences alike: ``pages`` [B, max_pages] int32, the pages
    of each sequence in order; ``lens`` [B] int32, all its tokens, those of this
    call among them.  The rows of a call are the sequences' newest tokens, sequence
    behind sequence: as many each, or, with ``rows`` [B + 1] int32 (ascending),
    rows[b] .. rows[b + 1] - 1 of sequence b.  These are tensors on the cache's
    device and are not looked at by the host; ``flag`` (int32 [1]) is set to 1 where
    one of them is out of range.
    """

    def __init__(self, n_pages: int, n_heads: int, head_dim: int, *, page_size: int = 64, device="cuda"):
        n_pages, n_heads, head_dim, page_size = (
            arg32(n, what, "aep_cache4") for n, what in
            ((n_pages, "n_pages"), (n_heads, "n_heads"), (head_dim, "head_dim"), (page_size, "page_size")))
        self.n_pages, self.n_heads, self.head_dim, self.page_size = n_pages, n_heads, head_dim, page_size
        self._desc = L.Cache4Desc(n_pages, page_size, n_heads, head_dim)
        self._at = ctypes.byref(self._desc)
        self._lib = L.lib()
        need = ctypes.c_size_t()
        L.check(self._lib.aep_cache4_bytes(self._at, ctypes.byref(need)), "aep_cache4_bytes")
        self.data = torch.zeros(need.value, dtype=torch.uint8, device=device)
        self.device = self.data.device
        if self.device.type != "cuda":
            raise ValueError(f"a cache on {self.device}, expected a CUDA (HIP) device")
        self._mem = self.data.data_ptr()
        self._calls = {}  # calls by what is checked of their tensors

    def _sizes(self, pages, lens, rows, flag, total) -> Tuple[int, int, int, int]:
        """(distance of the pages' rows, pages, sequences, rows) of a call, checked."""
        dev = self.device
        _rows(pages, "pages", (torch.int32,), (None, None), dev)
        B = pages.shape[0]
        for t, name, n in ((lens, "lens", B), (rows, "rows", B + 1), (flag, "flag", 1)):
            if t is not None:
                _rows(t, name, (torch.int32,), (n,), dev)
        if lens is None:
            raise ValueError("lens must be a tensor")
        if rows is None and (total % B if B else total):
            raise ValueError(f"{total} rows for {B} sequences: rows says whose they are")
        _int32(max(total, pages.shape[1] * self.page_size), 1 << 30, "rows, or tokens of a sequence", "aep_cache4")
        _int32(B, 1 << 24, "sequences", "aep_cache4")
        return _ld(pages), pages.shape[1], B, total

    def _keep(self, key, call):
        if len(self._calls) >= 1024:
            self._calls.clear()
        self._calls[key] = call
        return call

    def append(self, k: torch.Tensor, v: torch.Tensor, pages: torch.Tensor, lens: torch.Tensor,
               rows: Optional[torch.Tensor] = None, *, flag: Optional[torch.Tensor] = None) -> None:
        """Quantise rows of keys and values [T, n_heads, head_dim] bfloat16 into the
        cache (``aep_cache4_append``).  Rows and heads may be strided.  A row whose token
        has no page in the table, or one outside the cache, is left out."""
        dev = self.device
        if dev.index != L.current_device():
            with torch.cuda.device(dev):
                return self.append(k, v, pages, lens, rows, flag=flag)
        # a call like one before, in all that is checked, needs no checks
        try:
            key = ("append", k.shape, k.stride(), k.dtype, k.device, v.shape, v.stride(), v.dtype, v.device,
                   _tables(pages, lens, rows, flag))
        except AttributeError:
            raise ValueError("k, v, pages, lens, rows and flag must be tensors") from None
        fixed = self._calls.get(key)
        if fixed is None:
            _heads(k, "k", (None, self.n_heads, self.head_dim), dev)
            _heads(v, "v", tuple(k.shape), dev)
            fixed = self._keep(key, self._sizes(pages, lens, rows, flag, k.shape[0]))
        st = self._lib.aep_cache4_append(self._at, self._mem, _seqs(pages, lens, rows, flag, fixed), k.data_ptr(), k.stride(0),
                                         k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), L.raw_stream(dev.index))
        if st:
            L.check(st, "aep_cache4_append")

    def read(self, pages: torch.Tensor, lens: torch.Tensor, n_rows: int, rows: Optional[torch.Tensor] = None, *,
             k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
             flag: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """The newest tokens' keys and values [n_rows, n_heads, head_dim] bfloat16
        (``aep_cache4_read``): what the cache keeps of them, zeros where a sequence has
        no token for a row.  Rows of no sequence are left as they were in k and v, and are
        zeros in new tensors."""
        dev = self.device
        if dev.index != L.current_device():
            with torch.cuda.device(dev):
                return self.read(pages, lens, n_rows, rows, k=k, v=v, flag=flag)
        n_rows = _number(n_rows, "n_rows", "aep_cache4_read")
        try:
            key = ("read", n_rows, k is None or (k.shape, k.stride(), k.dtype, k.device, k.data_ptr() & 15),
                   v is None or (v.shape, v.stride(), v.dtype, v.device, v.data_ptr() & 15),
                   _tables(pages, lens, rows, flag))
        except AttributeError:
            raise ValueError("pages, lens, rows, k, v and flag must be tensors") from None
        fixed = self._calls.get(key)
        shape = (n_rows, self.n_heads, self.head_dim)
        if fixed is None:
            if arg32(n_rows, "n_rows", "aep_cache4_read") < 0:
                raise ValueError(f"n_rows is {n_rows}")
            for t, name in ((k, "k"), (v, "v")):
                if t is not None:
                    _heads(t, name, shape, dev)
                    if not t.is_contiguous():
                        raise ValueError(f"{name} must be contiguous")
            fixed = self._keep(key, self._sizes(pages, lens, rows, flag, n_rows))
        new = torch.empty if rows is None else torch.zeros  # (with rows, some may be of no sequence)
        if k is None:
            k = new(shape, dtype=torch.bfloat16, device=dev)
        if v is None:
            v = new(shape, dtype=torch.bfloat16, device=dev)
        st = self._lib.aep_cache4_read(self._at, self._mem, _seqs(pages, lens, rows, flag, fixed), k.data_ptr(), v.data_ptr(),
                                       L.raw_stream(dev.index))
        if st:
            L.check(st, "aep_cache4_read")
        return k, v

    def attend(self, q: torch.Tensor, pages: torch.Tensor, lens: torch.Tensor, rows: Optional[torch.Tensor] = None, *,
               scale: Optional[float] = None, window: int = 0, max_rows: int = 0, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None, flag: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of rows of queries [T, heads, head_dim] bfloat16 to the tokens of
        their sequences up to their own (``aep_cache4_attend``); heads a multiple of n_heads.

        scale defaults to head_dim^-0.5.  window: how many tokens a row sees, the last
        ones (0: all).  max_rows: with ``rows``, the most of a sequence where that is known
        (0: not known); it may save launches, and must hold.  out [T, heads, head_dim] bfloat16 (rows and heads may be strided);
        lse [T, heads] float32 receives the logarithms of the sums.  A row without a token
        gets 0, and -inf; rows of no sequence are left as they were, and are zeros in a new
        tensor (with ``rows``: a fill, some 2 us, that ``out`` saves)."""
        dev = self.device
        if dev.index != L.current_device():
            with torch.cuda.device(dev):
                return self.attend(q, pages, lens, rows, scale=scale, window=window, max_rows=max_rows, out=out, lse=lse,
                                   flag=flag)
        window = _number(window, "window", "aep_cache4_attend")
        max_rows = _number(max_rows, "max_rows", "aep_cache4_attend")
        if scale is not None and type(scale) is not float:
            scale = float(scale)
        # a call like one before, in all that is checked, needs no checks
        try:
            key = (q.shape, q.stride(), q.dtype, q.device, scale, window, max_rows,
                   out is None or (out.shape, out.stride(), out.dtype, out.device),
                   lse is None or (lse.shape, lse.stride(), lse.dtype, lse.device), _tables(pages, lens, rows, flag))
        except AttributeError:
            raise ValueError("q, pages, lens, rows, out, lse and flag must be tensors") from None
        need, desc, sizes = self._calls.get(key) or self._describe(key, q, pages, lens, rows, scale, window, max_rows, out,
                                                                   lse, flag)
        if out is None:
            # (with rows, some may be of no sequence)
            out = (torch.empty if rows is None else torch.zeros)(q.shape, dtype=torch.bfloat16, device=dev)
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None  # held until the launch is in the stream
        st = self._lib.aep_cache4_attend(self._at, self._mem, _seqs(pages, lens, rows, flag, sizes), desc, q.data_ptr(),
                                         out.data_ptr(), None if lse is None else lse.data_ptr(),
                                         None if ws is None else ws.data_ptr(), need, L.raw_stream(dev.index))
        if st:
            L.check(st, "aep_cache4_attend")
        return out

    def _describe(self, key, q, pages, lens, rows, scale, window, max_rows, out, lse, flag):
        """(bytes of scratch, description, sizes of the sequences) of a checked call, kept for the next ones like it."""
        dev = self.device
        _heads(q, "q", (None, None, self.head_dim), dev)
        T, H, _ = q.shape
        if H < 1 or H % self.n_heads:
            raise ValueError(f"{H} heads of queries for {self.n_heads} of the cache")
        if out is not None:
            _heads(out, "out", tuple(q.shape), dev)
        if lse is not None:
            _bytes_matrix(lse, "lse", (torch.float32,), (T, H), dev)
        window, max_rows = (arg32(n, what, "aep_cache4_attend") for n, what in ((window, "window"), (max_rows, "max_rows")))
        scale = self.head_dim ** -0.5 if scale is None else scale
        if window < 0 or max_rows < 0 or not math.isfinite(scale) or scale <= 0:
            raise ValueError(f"window {window}, max_rows {max_rows}, scale {scale}")
        sizes = self._sizes(pages, lens, rows, flag, T)
        o = (H * self.head_dim, self.head_dim) if out is None else (out.stride(0), out.stride(1))
        d = L.Attend4Desc(H, window, max_rows, scale, q.stride(0), q.stride(1), *o)
        b = ctypes.c_size_t()
        L.check(self._lib.aep_cache4_attend_workspace(self._at, _seqs(pages, lens, rows, flag, sizes), ctypes.byref(d),
                                                      ctypes.byref(b)), "aep_cache4_attend_workspace")
        return self._keep(key, (b.value, ctypes.byref(d), sizes))
