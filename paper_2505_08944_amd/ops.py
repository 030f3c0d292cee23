"""The operators in front of the queues that need no context: the dense
product with its epilogue and routing by scores.

As in ``context``, torch provides memory and the stream, and the work runs in
libaep.  A call runs on the device of its tensors, on torch's current stream
there.  Tensors are read on that stream: a caller that uses tensors of another
stream orders the two, as for any torch operation.  Forward only: results do
not take part in autograd.
"""

from __future__ import annotations

import ctypes
import operator
from typing import Optional, Tuple

import torch

from . import _lib as L

_CODE = {torch.float32: L.AEP_F32, torch.bfloat16: L.AEP_BF16, torch.float8_e4m3fn: L.AEP_FP8_E4M3,
         torch.uint8: L.AEP_FP8_E4M3}
_FN = {"none": L.AEP_FN_NONE, "relu": L.AEP_FN_RELU, "silu": L.AEP_FN_SILU, "gelu": L.AEP_FN_GELU,
       "gelu_tanh": L.AEP_FN_GELU_TANH}
_SCORE = {"softmax": L.AEP_SCORE_SOFTMAX, "sigmoid": L.AEP_SCORE_SIGMOID}


def _rows(t: torch.Tensor, name: str, dtypes, shape, device) -> None:
    """A matrix (or vector) on ``device`` whose rows are contiguous and apart."""
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise ValueError(f"{name} must be a tensor on {device}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    have = t.shape
    if len(have) != len(shape) or have[-1] != shape[-1] and shape[-1] is not None or \
            have[0] != shape[0] and shape[0] is not None:
        raise ValueError(f"{name} has shape {tuple(have)}, expected {shape}")
    step = t.stride()
    if step[-1] != 1 and have[-1] > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    if len(have) == 2 and have[0] > 1 and step[0] < have[1]:
        raise ValueError(f"{name}: rows must not overlap")


def _ld(t: torch.Tensor) -> int:
    """Elements from one row to the next (a single row has no next one)."""
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _int32(n: int, most: int, what: str, call: str) -> None:
    # (ctypes cuts larger values off)
    if n > most:
        raise L.AEPError(L.AEP_ERR_UNSUPPORTED, f"{call}: {n} {what}")


def arg32(n, what: str, call: str) -> int:
    """n, a whole number that an int32 argument holds."""
    n = operator.index(n)
    if not -(1 << 31) <= n < 1 << 31:
        raise L.AEPError(L.AEP_ERR_INVALID_ARG, f"{call}: {what} {n}")
    return n


class _Fixed:
    """Attributes are set once: what is kept for calls goes with them."""

    def __setattr__(self, name, value):
        if name in self.__dict__:
            raise AttributeError(f"{type(self).__name__}.{name} is fixed: make a new {type(self).__name__}")
        self.__dict__[name] = value


class Linear(_Fixed):
    """y = f(scale * (x W^T) + bias) + residual (``aep_linear``).

    weight [n, k]: float32 (x float32), bfloat16 or float8_e4m3fn / uint8 codes
    (x bfloat16), the latter with scale [n] bfloat16; rows may be strided.
    bias [n] float32 or bfloat16.  activation: none, relu, silu, gelu or
    gelu_tanh.  out_dtype: x's type (the default) or float32.  The tensors are
    kept, not copied: values written to them later are used by later calls;
    with another shape, stride, type or device than they had they are refused.
    """

    def __init__(self, weight: torch.Tensor, *, scale: Optional[torch.Tensor] = None,
                 bias: Optional[torch.Tensor] = None, activation: str = "none",
                 out_dtype: Optional[torch.dtype] = None):
        if not isinstance(weight, torch.Tensor) or not weight.is_cuda:
            raise ValueError("weight must be a CUDA (HIP) tensor")
        dev = weight.device
        _rows(weight, "weight", (torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.uint8), (None, None), dev)
        n, k = weight.shape
        if n < 1 or k < 1:
            raise ValueError(f"weight has shape {tuple(weight.shape)}")
        _int32(max(n, k), 1 << 30, "channels", "aep_linear")
        fp8 = _CODE[weight.dtype] == L.AEP_FP8_E4M3
        if fp8 != (scale is not None):
            raise ValueError("scale goes with fp8 weights, and only with them")
        for t, name, dtypes in ((scale, "scale", (torch.bfloat16,)),
                                (bias, "bias", (torch.float32, torch.bfloat16))):
            if t is not None:
                _rows(t, name, dtypes, (n,), dev)
        if activation not in _FN:
            raise ValueError(f"activation {activation!r}, expected one of {', '.join(_FN)}")
        self.x_dtype = torch.float32 if weight.dtype == torch.float32 else torch.bfloat16
        out_dtype = out_dtype or self.x_dtype
        if out_dtype not in (torch.float32, self.x_dtype):
            raise ValueError(f"out_dtype {out_dtype}, expected {self.x_dtype} or torch.float32")
        self.weight, self.scale, self.bias = weight, scale, bias
        self.activation, self.out_dtype, self.device = activation, out_dtype, dev
        self.n, self.k = n, k
        self._lib = L.lib()
        self._fixed = (n, k, _CODE[self.x_dtype], _CODE[weight.dtype], _CODE[out_dtype],
                       L.AEP_F32 if bias is None else _CODE[bias.dtype])
        self._fn = _FN[activation]
        self._ldw = _ld(weight)
        self._kept = tuple((t, t.shape, t.stride(), t.dtype) for t in (weight, scale, bias) if t is not None)
        self._calls = {}  # by what is checked of the tensors: what _describe makes of such a call

    def __call__(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [m, k] -> [m, n].  residual [m, n] float32 or bfloat16; out may be
        the residual itself, and must not overlap anything else."""
        dev = self.device
        if dev.index != L.current_device():
            with torch.cuda.device(dev):
                return self(x, residual, out)
        # (a module's conversions set the data of its parameters; 0.3 .. 0.4 us per tensor, of some 6)
        for t, shape, stride, dtype in self._kept:
            if t.dtype is not dtype or t.stride() != stride or t.shape != shape or t.get_device() != dev.index:
                raise ValueError("the weight, its scale or the bias has another shape, stride, type or device than it "
                                 "had: make a new Linear")
        # a call like one before, in all that is checked and in its alignment, which the
        # scratch goes by, needs no checks
        try:
            at, w_at = x.data_ptr(), self.weight.data_ptr()
            key = (x.shape, x.stride(), x.dtype, x.device, (at & 15) << 4 | w_at & 15,
                   residual is None or (residual.shape, residual.stride(), residual.dtype, residual.device,
                                        residual.data_ptr() & 15),
                   out is None or (out.shape, out.stride(), out.dtype, out.device, out.data_ptr() & 15))
        except AttributeError:
            raise ValueError("x, residual and out must be tensors") from None
        desc, need, shape = self._calls.get(key) or self._describe(key, x, residual, out)
        if out is None:
            out = torch.empty(shape, dtype=self.out_dtype, device=dev)
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None  # held until the launch is in the stream
        scale, bias = self.scale, self.bias
        st = self._lib.aep_linear(desc, at, w_at, None if scale is None else scale.data_ptr(),
                                  None if bias is None else bias.data_ptr(),
                                  None if residual is None else residual.data_ptr(), out.data_ptr(),
                                  None if ws is None else ws.data_ptr(), need, L.raw_stream(dev.index))
        if st:
            L.check(st, "aep_linear")
        return out

    def _describe(self, key, x, residual, out):
        """(description, bytes of scratch, shape of the result) of a checked call, kept for the next ones like it."""
        n, k, x_dtype, w_dtype, y_dtype, bias_dtype = self._fixed
        dev = self.device
        _rows(x, "x", (self.x_dtype,), (None, k), dev)
        m = x.shape[0]
        _int32(m, 1 << 30, "rows", "aep_linear")
        if residual is not None:
            _rows(residual, "residual", (torch.float32, torch.bfloat16), (m, n), dev)
        if out is not None:
            _rows(out, "out", (self.out_dtype,), (m, n), dev)
        d = L.LinearDesc(m, n, k, x_dtype, w_dtype, y_dtype, bias_dtype,
                         y_dtype if residual is None else _CODE[residual.dtype], self._fn, _ld(x), self._ldw,
                         n if out is None else _ld(out), n if residual is None else _ld(residual))
        b = ctypes.c_size_t()
        # (an output that torch allocates is aligned)
        L.check(self._lib.aep_linear_workspace_at(ctypes.byref(d), x.data_ptr(), self.weight.data_ptr(),
                                                  None if residual is None else residual.data_ptr(),
                                                  16 if out is None else out.data_ptr(), ctypes.byref(b)),
                "aep_linear_workspace_at")
        if len(self._calls) >= 1024:
            self._calls.clear()
        call = self._calls[key] = (ctypes.byref(d), b.value, (m, n))
        return call


def linear(x: torch.Tensor, weight: torch.Tensor, *, scale: Optional[torch.Tensor] = None,
           bias: Optional[torch.Tensor] = None, activation: str = "none", residual: Optional[torch.Tensor] = None,
           out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``Linear`` for one call."""
    return Linear(weight, scale=scale, bias=bias, activation=activation, out_dtype=out_dtype)(x, residual, out)


class Router(_Fixed):
    """How a layer picks its experts (``aep_router``): softmax or sigmoid
    scores; experts in n_groups groups of consecutive ids, of which the
    top_groups best stay, each worth the sum of its group_top (1 or 2) best
    choices; the top_k best choices (score + bias); weights from the scores,
    renormalised over the chosen or not, times scale."""

    def __init__(self, n_experts: int, top_k: int, *, score: str = "softmax", n_groups: int = 1, top_groups: int = 1,
                 group_top: int = 1, renorm: bool = True, scale: float = 1.0):
        if score not in _SCORE:
            raise ValueError(f"score {score!r}, expected one of {', '.join(_SCORE)}")
        n_experts, top_k, n_groups, top_groups, group_top = (
            arg32(n, what, "aep_route_topk") for n, what in
            ((n_experts, "n_experts"), (top_k, "top_k"), (n_groups, "n_groups"), (top_groups, "top_groups"),
             (group_top, "group_top")))
        self.n_experts, self.top_k, self.score = n_experts, top_k, score
        self.n_groups, self.top_groups, self.group_top = n_groups, top_groups, group_top
        self.renorm, self.scale = bool(renorm), float(scale)
        self.desc = L.RouterDesc(n_experts, top_k, _SCORE[score], n_groups, top_groups, group_top, int(self.renorm),
                                 self.scale)
        self._at = ctypes.byref(self.desc)
        self._lib = L.lib()
        self._seen = set()  # what was checked of logits and biases
        # the library checks the values; routing no tokens does nothing else
        L.check(self._lib.aep_route_topk(self._at, None, max(n_experts, 0), None, 0, None, None, None, None),
                "aep_route_topk")


def route(router: Router, logits: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
          idx: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None,
          flag: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Expert ids [T, k] int32 and gate weights [T, k] float32 of logits [T, E]
    float32 (``aep_route_topk``).  bias [E] float32 is added to the scores for
    the choice only.  flag: int32 [1], set to 1 where a logit is NaN or +inf
    (-inf masks an expert) or a bias is not finite."""
    try:
        dev = logits.device
        key = (logits.shape, logits.stride(), logits.dtype, dev,
               bias is None or (bias.shape, bias.stride(), bias.dtype, bias.device))
    except AttributeError:
        raise ValueError("logits and bias must be tensors") from None
    if not logits.is_cuda:
        raise ValueError("logits must be a CUDA (HIP) tensor")
    if dev.index != L.current_device():
        with torch.cuda.device(dev):
            return route(router, logits, bias, idx=idx, weights=weights, flag=flag)
    # logits and bias like ones before, in all that is checked, need no checks
    if key not in router._seen:
        _rows(logits, "logits", (torch.float32,), (None, router.n_experts), dev)
        _int32(logits.shape[0], (1 << 31) - 1, "tokens", "aep_route_topk")
        if bias is not None:
            _rows(bias, "bias", (torch.float32,), (router.n_experts,), dev)
        if len(router._seen) >= 1024:
            router._seen.clear()
        router._seen.add(key)
    T, k = key[0][0], router.top_k
    if idx is not None or weights is not None or flag is not None:
        for t, name, dtype, shape in ((idx, "idx", torch.int32, (T, k)), (weights, "weights", torch.float32, (T, k)),
                                      (flag, "flag", torch.int32, (1,))):
            if t is not None:
                _rows(t, name, (dtype,), shape, dev)
                if not t.is_contiguous():
                    raise ValueError(f"{name} must be contiguous")
    if idx is None:
        idx = torch.empty((T, k), dtype=torch.int32, device=dev)
    if weights is None:
        weights = torch.empty_like(idx, dtype=torch.float32)  # (quicker than empty())
    st = router._lib.aep_route_topk(
        router._at, logits.data_ptr(), _ld(logits), None if bias is None else bias.data_ptr(), T, idx.data_ptr(),
        weights.data_ptr(), None if flag is None else flag.data_ptr(), L.raw_stream(dev.index))
    if st:
        L.check(st, "aep_route_topk")
    return idx, weights
