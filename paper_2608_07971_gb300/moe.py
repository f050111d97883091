"""Price-routed expert layer on torch CUDA tensors: the binding of include/esp_moe.h.

Argument marshalling only: every step runs in the library's CUDA kernels (there is no CPU fallback). ``Moe``
holds one handle. Its calls are queued on the stream given at creation or to ``set_stream``, or without one on the
caller's current torch stream at every call; they return without waiting. Every call takes ``out`` to reuse the
tensors of an earlier one (a serving loop, a CUDA graph), else allocates its results. A graph that captured calls
uses the handle's work space, so the handle is kept as long as the graph is replayed.

    m = Moe()
    r = m.route(logits, k, gate=Gate("softmax"), prices=prices)      # choice, weights, demand, plan
    h = m.linear(x, w1, offsets=r.offsets, rows=r.rows)              # rows by expert, 8-bit products
    y = m.linear(act(h), w2, offsets=r.offsets)
    out = m.combine(y, r.pos, r.weight)
    m.step_prices(prices, r.counts, eta=0.02)

or, with 16-bit weights and a gated block for each expert, and for a training step:

    w = m.gated_weight(inner, outer, "silu")                         # (E, 2 F, H) and (E, H, F)
    kept = m.keep(r.rows.shape[0], w)
    y = m.feed_forward(x, w, offsets=r.offsets, rows=r.rows, keep=kept)
    dx, dinner, douter = m.feed_forward_backward(dy, x, w, kept, offsets=r.offsets, rows=r.rows)
    norm = m.clip([dinner, douter, drouter], max_norm=1.0)           # in place
"""

from __future__ import annotations

import contextlib
import ctypes
import dataclasses
import math
from typing import Optional, Tuple

import torch

from . import esp

BLOCK = 128
MAX_EXPERTS, MAX_CHOICES = 1024, 32

EXPORTED = [
    "esp_moe_create", "esp_moe_set_stream", "esp_moe_route", "esp_moe_balance", "esp_moe_route_backward",
    "esp_moe_step_prices", "esp_moe_quantize_weight", "esp_moe_linear", "esp_moe_linear_backward", "esp_moe_combine",
    "esp_moe_combine_backward", "esp_moe_synchronize", "esp_moe_last_launch_count", "esp_moe_destroy",
    "esp_moe_debug_set_wait_limit", "esp_moe_debug_hold_load", "esp_moe_feed_forward", "esp_moe_feed_forward_backward",
    "esp_moe_clip",
]

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_KINDS = {"softmax": 0, "sigmoid": 1}
_ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3}


class _CGate(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("renorm", ctypes.c_int32), ("scale", ctypes.c_float)]


class _CWeight(ctypes.Structure):
    _fields_ = [("E", ctypes.c_int32), ("N", ctypes.c_int32), ("K", ctypes.c_int32), ("ld", ctypes.c_int64),
                ("ldt", ctypes.c_int64), ("q", ctypes.c_void_p), ("qt", ctypes.c_void_p), ("scale", ctypes.c_void_p)]


class _CGated(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("activation", ctypes.c_int32), ("E", ctypes.c_int32), ("F", ctypes.c_int32),
                ("H", ctypes.c_int32), ("ld_inner", ctypes.c_int64), ("ld_outer", ctypes.c_int64),
                ("inner", ctypes.c_void_p), ("outer", ctypes.c_void_p)]


class _CKept(ctypes.Structure):
    _fields_ = [("pre", ctypes.c_void_p), ("hidden", ctypes.c_void_p), ("rows", ctypes.c_void_p), ("copied", ctypes.c_int32)]


class _CTensor(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32)]


_bound = None


def load_library():
    """libesp.so with the argument types of esp_moe.h; raises if the library is missing."""
    global _bound
    lib = esp.load_library()
    if _bound is lib:
        return lib
    vp, i32, i64, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
    st, gate, weight = ctypes.c_int, ctypes.POINTER(_CGate), ctypes.POINTER(_CWeight)
    gated, kept = ctypes.POINTER(_CGated), ctypes.POINTER(_CKept)
    sig = {
        "esp_moe_create": ([ctypes.POINTER(vp), ctypes.c_int, vp], st),
        "esp_moe_set_stream": ([vp, vp], st),
        "esp_moe_route": ([vp, gate, i32, i64, i32, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp], st),
        "esp_moe_balance": ([vp, gate, i32, i64, i32, i32, i64, vp, vp, i32, vp, vp, vp, vp, vp], st),
        "esp_moe_route_backward": ([vp, gate, i32, i64, i32, i32, i64, vp, vp, vp, i32, vp, vp, vp, vp, i64, vp], st),
        "esp_moe_step_prices": ([vp, i32, vp, f64, f64, vp], st),
        "esp_moe_quantize_weight": ([vp, i32, vp, i64, weight], st),
        "esp_moe_linear": ([vp, i32, i64, i64, vp, i64, vp, weight, vp, i64, vp], st),
        "esp_moe_linear_backward": ([vp, i32, i64, i64, vp, i64, vp, weight, vp, i64, vp, i64, vp, i64, vp], st),
        "esp_moe_combine": ([vp, i32, i64, i32, i32, i64, i64, vp, vp, vp, i64, vp], st),
        "esp_moe_combine_backward": ([vp, i32, i64, i32, i32, i64, i64, vp, i64, vp, vp, vp, i64, vp, vp], st),
        "esp_moe_feed_forward": ([vp, gated, i64, i64, vp, i64, vp, vp, i64, vp, kept], st),
        "esp_moe_feed_forward_backward": ([vp, gated, i64, i64, vp, i64, vp, vp, kept, i64, vp, i64, vp, i32, vp, vp], st),
        "esp_moe_clip": ([vp, i32, ctypes.POINTER(_CTensor), f64, f64, vp], st),
        "esp_moe_synchronize": ([vp], st),
        "esp_moe_last_launch_count": ([vp, ctypes.POINTER(i64)], st),
        "esp_moe_destroy": ([vp], None),
        "esp_moe_debug_set_wait_limit": ([vp, ctypes.c_uint32], st),
        "esp_moe_debug_hold_load": ([vp], st),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    _bound = lib
    return lib


def _from_fields(self):
    """Copies and pickles are made of the fields: C arguments and marks of checked tensors belong to one object."""
    return type(self), tuple(getattr(self, f.name) for f in dataclasses.fields(self) if f.init)


@dataclasses.dataclass(frozen=True)
class Gate:
    """How a chosen expert's weight follows from the logits (esp_moe_gate)."""

    kind: str = "softmax"
    renorm: bool = True
    scale: float = 1.0

    def __post_init__(self):
        if self.kind not in _KINDS:
            raise ValueError(f"unknown gate {self.kind!r}")
        object.__setattr__(self, "_c", _CGate(_KINDS[self.kind], int(self.renorm), self.scale))
        object.__setattr__(self, "_ref", ctypes.byref(self._c))

    __reduce__ = _from_fields


@dataclasses.dataclass(frozen=True)
class Routing:
    """Results of ``Moe.route``: idx, weight (T, k); counts (E,); rows (T * k,), pos (T, k), offsets (E + 1,)
    or None without a plan. `checked` holds (device index, T, E, k) where ``Moe.routing`` made the tensors; a copy with
    other tensors (``dataclasses.replace``) starts without it."""

    idx: torch.Tensor
    weight: torch.Tensor
    counts: torch.Tensor
    rows: Optional[torch.Tensor] = None
    pos: Optional[torch.Tensor] = None
    offsets: Optional[torch.Tensor] = None
    checked: Optional[tuple] = dataclasses.field(default=None, init=False, repr=False, compare=False)

    __reduce__ = _from_fields


@dataclasses.dataclass(frozen=True)
class Balance:
    """Results of ``Moe.balance``: loss (2,) = balance, logit; counts (B, E), share (B, E), tokens (B,). `checked`
    holds (device index, B, E) where ``Moe.balancing`` made the tensors; a copy with other tensors starts without it."""

    loss: torch.Tensor
    counts: torch.Tensor
    share: torch.Tensor
    tokens: torch.Tensor
    checked: Optional[tuple] = dataclasses.field(default=None, init=False, repr=False, compare=False)

    __reduce__ = _from_fields


@dataclasses.dataclass
class Weight:
    """8-bit weights of E experts (N x K each): codes q (E, N, ld), scale (E, N / 128, K / 128) and, for
    gradients, the transposed codes qt (E, K, ldt)."""

    E: int
    N: int
    K: int
    q: torch.Tensor
    scale: torch.Tensor
    qt: Optional[torch.Tensor] = None

    def __post_init__(self):
        E, N, K, q, qt, scale = self.E, self.N, self.K, self.q, self.qt, self.scale

        def codes(t, rows, cols):
            return t.dtype is torch.uint8 and t.dim() == 3 and t.shape[:2] == (E, rows) and t.shape[2] >= cols and \
                t.is_contiguous() and t.device == scale.device

        if not codes(q, N, K) or (qt is not None and not codes(qt, K, N)) or scale.dtype is not torch.float32 or \
                scale.shape != (E, -(-N // BLOCK), -(-K // BLOCK)) or not scale.is_contiguous():
            raise ValueError("8-bit weights: contiguous uint8 codes (E, N, >= K), fp32 scales (E, N / 128, K / 128)")
        self._c = _CWeight(E, N, K, q.shape[2], qt.shape[2] if qt is not None else 0, q.data_ptr(), _ptr(qt), scale.data_ptr())
        self._ref = ctypes.byref(self._c)
        self._made_at = self._places()

    __reduce__ = _from_fields

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        if name[0] != "_":
            self._ref = None   # checked and made anew by the next call

    def _places(self):
        return _place(self.q), None if self.qt is None else _place(self.qt), _place(self.scale)

    def _arg(self):
        """The C argument for the fields as they are, whether assigned since or given other memory, another shape or type
        in place (``.data``)."""
        if self._ref is None or self._places() != self._made_at:
            self.__post_init__()
        return self._ref

    def codes(self) -> torch.Tensor:
        """The codes as float8_e4m3fn, (E, N, K)."""
        return self.q.view(torch.float8_e4m3fn)[:, :, :self.K]


@dataclasses.dataclass
class GatedWeight:
    """16-bit weights of E gated feed-forward blocks: inner (E, 2 F, H), gate rows before up rows, and outer (E, H, F),
    whose rows start at multiples of 16 bytes (``Moe.gated_weight`` lays out others). Both may be written to between calls."""

    inner: torch.Tensor
    outer: torch.Tensor
    activation: str = "silu"

    def __post_init__(self):
        a, b = self.inner, self.outer
        if self.activation not in _ACTIVATIONS:
            raise ValueError(f"unknown activation {self.activation!r}")
        if a.dim() != 3 or b.dim() != 3 or a.dtype not in (torch.bfloat16, torch.float16) or b.dtype is not a.dtype or \
                a.device != b.device or a.shape[1] % 2 or b.shape != (a.shape[0], a.shape[2], a.shape[1] // 2) or \
                a.numel() == 0 or not (_rows16(a) and _rows16(b)):
            raise ValueError("gated weights: bf16 or fp16, inner (E, 2 F, H) and outer (E, H, F), rows on multiples of 16 bytes")
        self.E, self.F, self.H = a.shape[0], b.shape[2], a.shape[2]
        self._c = _CGated(_DTYPES[a.dtype], _ACTIVATIONS[self.activation], self.E, self.F, self.H, a.stride(1), b.stride(1),
                          a.data_ptr(), b.data_ptr())
        self._ref = ctypes.byref(self._c)
        self._made_at = self._places()

    __reduce__ = _from_fields

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        if name in ("inner", "outer", "activation"):
            self._ref = None   # checked and made anew by the next call

    def _places(self):
        return _place(self.inner), _place(self.outer)

    def _arg(self):
        """As ``Weight._arg``; E, F and H follow the fields, so that it comes before what is checked against them."""
        if self._ref is None or self._places() != self._made_at:
            self.__post_init__()
        return self._ref


@dataclasses.dataclass
class Kept:
    """What ``Moe.feed_forward`` keeps for its gradients (esp_moe_kept): pre (M, 2, F64) fp32, hidden (M, F64), rows
    (M, H64), with F and H rounded up to multiples of 64. Made by ``Moe.keep``."""

    pre: torch.Tensor
    hidden: torch.Tensor
    rows: torch.Tensor
    copied: bool = False

    def _arg(self):
        return _CKept(self.pre.data_ptr(), self.hidden.data_ptr(), self.rows.data_ptr(), int(self.copied))


class Gradients:
    """A list of gradient tensors laid out for ``Moe.clip``: made once by ``Moe.gradients`` where the tensors stay the same
    from step to step."""

    def __init__(self, tensors, out, index: int):
        self.tensors, self.out = list(tensors), None if out is None else list(out)
        if self.out is not None and len(self.out) != len(self.tensors):
            raise ValueError("out: one tensor for each gradient expected")
        outs = self.tensors if self.out is None else self.out
        for t, o in zip(self.tensors, outs):
            for v in (t, o):
                if v.get_device() != index:
                    raise ValueError(f"a gradient is on {v.device}, the handle on cuda:{index}")
                if v.dtype not in _DTYPES or v.dtype is not t.dtype:
                    raise ValueError(f"gradients: type {v.dtype} not taken here")
                if v.shape != t.shape or not v.is_contiguous():
                    raise ValueError("gradients: contiguous tensors expected, out of the same shapes")
        self.index = index
        self._c = (_CTensor * len(self.tensors))(*(
            (t.data_ptr(), o.data_ptr(), t.numel(), _DTYPES[t.dtype]) for t, o in zip(self.tensors, outs)))
        all_of = self._all()
        self._made_at = list(map(_data_ptr, all_of))
        self._made_of = _TensorGuards(*all_of, dynamic_dims_sizes=None, dynamic_dims_strides=None)

    def _all(self):
        return self.tensors if self.out is None else self.tensors + self.out

    def _arg(self):
        all_of = self._all()
        # other memory, sizes, strides or types (``.data``)
        if list(map(_data_ptr, all_of)) != self._made_at or not self._made_of.check(*all_of):
            self.__init__(self.tensors, self.out, self.index)
        return self._c


_data_ptr = torch.Tensor.data_ptr
# whether each of many tensors has the sizes, strides and type that it had: 0.05 us a tensor, its attributes one by one 0.2
_TensorGuards = torch._C._dynamo.guards.TensorGuards

# the current stream's handle without a Stream object around it (0.1 instead of 2 us per call)
_raw_stream = torch._C._cuda_getCurrentRawStream


def _pad16(n: int) -> int:
    return (n + 15) // 16 * 16


def _pad64(n: int) -> int:
    return (n + 63) // 64 * 64


def _rows16(t) -> bool:
    """Whether the rows of a 3-D 16-bit tensor start at multiples of 16 bytes, planes following one another."""
    return t.stride(2) == 1 and t.stride(1) % 8 == 0 and t.stride(1) >= t.shape[2] and t.data_ptr() % 16 == 0 and \
        (t.shape[0] == 1 or t.stride(0) == t.shape[1] * t.stride(1))


def _place(t):
    """What a C argument made from a tensor depends on."""
    return t.data_ptr(), t.shape, t.stride(), t.dtype


def _ptr(t):
    return None if t is None else t.data_ptr()


class Moe:
    """One esp_moe handle.

    With a ``stream`` of its own all of a call's work is queued there: kernels, fills, copies, and the allocation of
    results, which belong to that stream in torch's sense. As with any side stream the program orders its inputs before
    the call and its use of the results after it (``synchronize``, or events), and calls ``record_stream`` where a
    tensor is freed on one stream while the other still uses it.
    """

    def __init__(self, device=None, stream: Optional[int] = None):
        self.h = None
        self._lib = load_library()
        if device is None:
            device = torch.cuda.current_device()
        device = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
        if device.type != "cuda":
            raise ValueError(f"a CUDA device expected, not {device}")
        self.device = torch.device("cuda", torch.cuda.current_device() if device.index is None else device.index)
        self._index = self.device.index
        self._follow = stream is None
        self._stream = torch.cuda.current_stream(self.device).cuda_stream if stream is None else int(stream)
        h = ctypes.c_void_p()
        esp._check(self._lib.esp_moe_create(ctypes.byref(h), self.device.index, self._stream or None), "esp_moe_create")
        self.h = h.value
        self._side = None   # torch's view of a stream of the handle's own
        if not self._follow:
            self._side = self._torch_stream(self._stream)

    # -- helpers

    def _torch_stream(self, stream: int):
        if stream == 0:
            return torch.cuda.default_stream(self.device)
        return torch.cuda.ExternalStream(stream, device=self.device)

    def _queue(self):
        """Context in which torch allocates and queues on the handle's stream."""
        return contextlib.nullcontext() if self._side is None else torch.cuda.stream(self._side)

    def _on_stream(self):
        if self.h is None:
            raise ValueError("the handle is closed")
        if self._follow:
            s = _raw_stream(self._index)
            if s != self._stream:
                self._move(s)

    def _move(self, stream: int) -> None:
        esp._check(self._lib.esp_moe_set_stream(self.h, stream or None), "esp_moe_set_stream")
        self._stream = stream

    def set_stream(self, stream: int) -> None:
        """Later calls run on the cudaStream_t `stream`, after what was queued before; the handle no longer follows
        the current stream."""
        self._move(stream)
        self._side = self._torch_stream(stream)
        self._follow = False

    def _need(self, t, name: str, dtype=None, shape=None, optional: bool = False):
        """Checks a dense argument: its device, type, shape."""
        if t is None:
            if optional:
                return
            raise ValueError(f"{name} is missing")
        if t.dtype is dtype and t.shape == shape and t.get_device() == self._index and t.is_contiguous():
            return
        if t.get_device() != self._index:
            raise ValueError(f"{name} is on {t.device}, the handle on {self.device}")
        if dtype is not None and t.dtype is not dtype:
            raise ValueError(f"{name}: {dtype} expected, not {t.dtype}")
        if shape is not None:
            if t.shape != shape:
                raise ValueError(f"{name}: shape {shape} expected, not {tuple(t.shape)}")
            if not t.is_contiguous():
                raise ValueError(f"{name} is not contiguous")

    def _matrix(self, t, name: str, rows=None, cols=None, dtype=None) -> Tuple[int, int]:
        """Checks a matrix of a floating-point type; returns its type code and leading dimension."""
        if t is None:
            raise ValueError(f"{name} is missing")
        if t.get_device() != self._index:
            raise ValueError(f"{name} is on {t.device}, the handle on {self.device}")
        code = _DTYPES.get(t.dtype)
        if code is None or (dtype is not None and t.dtype is not dtype):
            raise ValueError(f"{name}: type {t.dtype} not taken here")
        shape = t.shape
        if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
            raise ValueError(f"{name}: shape ({rows}, {cols}) expected, not {tuple(shape)}")
        n, m = shape
        if t.is_contiguous():
            return code, m
        step, unit = t.stride()
        if unit != 1 and m > 1 and n > 0:
            raise ValueError(f"{name}: a matrix with contiguous rows expected")
        return code, step if n > 1 else m

    def _new(self, shape, dtype):
        if self._side is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with self._queue():
            return torch.empty(shape, dtype=dtype, device=self.device)

    # -- router

    def routing(self, T: int, E: int, k: int, plan: bool = True) -> Routing:
        """Empty results of ``route``, to pass as its ``out``."""
        i32, plan_of = torch.int32, (None, None, None)
        if plan:
            plan_of = (self._new((T * k,), i32), self._new((T, k), i32), self._new((E + 1,), i32))
        r = Routing(self._new((T, k), i32), self._new((T, k), torch.float32), self._new((E,), torch.int64), *plan_of)
        object.__setattr__(r, "checked", (self._index, T, E, k))
        return r

    def route(self, logits, k: int, gate: Gate = Gate(), prices=None, valid=None, plan: bool = True,
              out: Optional[Routing] = None) -> Routing:
        """The k experts of greatest logit minus price of every token, their gate weights, the demand for each
        expert and (plan) the rows sorted by expert (esp_moe_route). valid: (T,) bool, False for padding."""
        code, ld = self._matrix(logits, "logits")
        T, E = logits.shape
        self._need(prices, "prices", torch.float32, (E,), optional=True)
        self._need(valid, "valid", torch.bool, (T,), optional=True)
        if out is None:
            out = self.routing(T, E, k, plan)
        elif out.checked != (self._index, T, E, k):
            self._need(out.idx, "out.idx", torch.int32, (T, k))
            self._need(out.weight, "out.weight", torch.float32, (T, k))
            self._need(out.counts, "out.counts", torch.int64, (E,))
            if out.rows is not None or out.pos is not None or out.offsets is not None:
                self._need(out.rows, "out.rows", torch.int32, (T * k,))
                self._need(out.pos, "out.pos", torch.int32, (T, k))
                self._need(out.offsets, "out.offsets", torch.int32, (E + 1,))
        self._on_stream()
        esp._check(self._lib.esp_moe_route(
            self.h, gate._ref, code, T, E, k, ld, logits.data_ptr(), _ptr(prices), _ptr(valid), out.idx.data_ptr(),
            out.weight.data_ptr(), out.counts.data_ptr(), _ptr(out.rows), _ptr(out.pos), _ptr(out.offsets)),
            "esp_moe_route")
        return out

    def balancing(self, B: int, E: int) -> Balance:
        """Empty results of ``balance``, to pass as its ``out``."""
        b = Balance(self._new((2,), torch.float32), self._new((B, E), torch.int64), self._new((B, E), torch.float32),
                    self._new((B,), torch.int64))
        object.__setattr__(b, "checked", (self._index, B, E))
        return b

    def balance(self, logits, idx, gate: Gate = Gate(), seq_offsets=None, out: Optional[Balance] = None) -> Balance:
        """Balance and logit losses of the choices idx, over the sequences that seq_offsets (B + 1,) int32 bounds
        (esp_moe_balance)."""
        code, ld = self._matrix(logits, "logits")
        T, E = logits.shape
        self._need(idx, "idx", torch.int32, (T, idx.shape[-1]))
        B = 1 if seq_offsets is None else seq_offsets.shape[0] - 1
        self._need(seq_offsets, "seq_offsets", torch.int32, (B + 1,), optional=True)
        if out is None:
            out = self.balancing(B, E)
        elif out.checked != (self._index, B, E):
            self._need(out.loss, "out.loss", torch.float32, (2,))
            self._need(out.counts, "out.counts", torch.int64, (B, E))
            self._need(out.share, "out.share", torch.float32, (B, E))
            self._need(out.tokens, "out.tokens", torch.int64, (B,))
        self._on_stream()
        esp._check(self._lib.esp_moe_balance(
            self.h, gate._ref, code, T, E, idx.shape[1], ld, logits.data_ptr(), idx.data_ptr(), B, _ptr(seq_offsets),
            out.loss.data_ptr(), out.counts.data_ptr(), out.share.data_ptr(), out.tokens.data_ptr()),
            "esp_moe_balance")
        return out

    def route_backward(self, logits, idx, gate: Gate = Gate(), dweight=None, balance: Optional[Balance] = None,
                       seq_offsets=None, dloss=None, out=None):
        """Gradient of the logits from the gate weights' gradient dweight (T, k), from the losses' gradients dloss
        (2,) with ``balance``'s results, or from both (esp_moe_route_backward)."""
        code, ld = self._matrix(logits, "logits")
        T, E = logits.shape
        self._need(idx, "idx", torch.int32, (T, idx.shape[-1]))
        k = idx.shape[1]
        self._need(dweight, "dweight", torch.float32, (T, k), optional=True)
        if (dloss is None) != (balance is None):
            raise ValueError("dloss and balance belong together")
        B = 1 if seq_offsets is None else seq_offsets.shape[0] - 1
        counts = tokens = None
        if balance is not None:
            self._need(dloss, "dloss", torch.float32, (2,))
            self._need(seq_offsets, "seq_offsets", torch.int32, (B + 1,), optional=True)
            counts, tokens = balance.counts, balance.tokens
            if balance.checked != (self._index, B, E):
                self._need(counts, "balance.counts", torch.int64, (B, E))
                self._need(tokens, "balance.tokens", torch.int64, (B,))
        if out is None:
            out = self._new((T, E), logits.dtype)
        _, ldo = self._matrix(out, "out", T, E, logits.dtype)
        self._on_stream()
        esp._check(self._lib.esp_moe_route_backward(
            self.h, gate._ref, code, T, E, k, ld, logits.data_ptr(), idx.data_ptr(), _ptr(dweight), B,
            _ptr(seq_offsets), _ptr(counts), _ptr(tokens), _ptr(dloss), ldo, out.data_ptr()),
            "esp_moe_route_backward")
        return out

    def step_prices(self, prices, counts, eta: float, slack: float = 1.0):
        """One price update in place from the demand `counts` (esp_moe_step_prices); slack: an expert's capacity
        in units of the mean demand."""
        E = prices.shape[0]
        self._need(prices, "prices", torch.float32, (E,))
        self._need(counts, "counts", torch.int64, (E,))
        self._on_stream()
        esp._check(self._lib.esp_moe_step_prices(self.h, E, counts.data_ptr(), eta, slack, prices.data_ptr()),
                   "esp_moe_step_prices")
        return prices

    # -- products

    def empty_weight(self, E: int, N: int, K: int, transposed: bool = False) -> Weight:
        """Room for the codes and scales of E x N x K weights; transposed: for gradients of the rows too."""
        q = self._new((E, N, _pad16(K)), torch.uint8)
        qt = self._new((E, K, _pad16(N)), torch.uint8) if transposed else None
        return Weight(E, N, K, q, self._new((E, -(-N // BLOCK), -(-K // BLOCK)), torch.float32), qt)

    def quantize_weight(self, w, transposed: bool = False, out: Optional[Weight] = None) -> Weight:
        """8-bit weights of w, (E, N, K) or (N, K) (esp_moe_quantize_weight)."""
        w3 = w if w.dim() == 3 else w[None]
        if w3.dim() != 3 or not w3.is_contiguous():
            raise ValueError("w: a contiguous (E, N, K) or (N, K) tensor expected")
        E, N, K = w3.shape
        code, ld = self._matrix(w3.view(E * N, K), "w")
        if out is None:
            out = self.empty_weight(E, N, K, transposed)
        elif (out.E, out.N, out.K) != (E, N, K):
            raise ValueError(f"out: weights of {(E, N, K)} expected")
        self._need(out.scale, "out")
        self._on_stream()
        esp._check(self._lib.esp_moe_quantize_weight(self.h, code, w3.data_ptr(), ld, out._arg()),
                   "esp_moe_quantize_weight")
        return out

    def load_weight(self, codes, scale, transposed: bool = False) -> Weight:
        """Weights that are stored as codes, (E, N, K) float8_e4m3fn, and scales, (E, N / 128, K / 128) fp32,
        laid out for the products (their memory is used as it is where the layout allows)."""
        E, N, K = codes.shape
        self._need(codes, "codes", torch.float8_e4m3fn)
        self._need(scale, "scale", torch.float32, (E, -(-N // BLOCK), -(-K // BLOCK)))
        with self._queue():
            if K % 16 == 0 and codes.is_contiguous() and codes.data_ptr() % 16 == 0:
                q = codes.view(torch.uint8)
            else:
                q = torch.zeros((E, N, _pad16(K)), dtype=torch.uint8, device=self.device)
                q[:, :, :K] = codes.view(torch.uint8)
            qt = None
            if transposed:
                qt = torch.zeros((E, K, _pad16(N)), dtype=torch.uint8, device=self.device)
                qt[:, :, :N] = q[:, :, :K].transpose(1, 2)
        return Weight(E, N, K, q, scale, qt)

    def _rows(self, x, weight: Weight, offsets, rows):
        self._need(weight.scale, "weight")
        if offsets is not None:
            self._need(offsets, "offsets", torch.int32, (weight.E + 1,))
        elif weight.E != 1:
            raise ValueError("offsets: needed for more than one expert")
        M = x.shape[0]
        if rows is not None:
            M = rows.shape[0]
            self._need(rows, "rows", torch.int32, (M,))
        return M

    def linear(self, x, weight: Weight, offsets=None, rows=None, out=None):
        """y (M, N): row i of expert e, offsets[e] <= i < offsets[e + 1], is x[rows[i]] W_e^T, or x[i] W_e^T
        without rows (esp_moe_linear). Rows outside every expert are left as they are."""
        code, ldx = self._matrix(x, "x", cols=weight.K)
        M = self._rows(x, weight, offsets, rows)
        if out is None:
            out = self._new((M, weight.N), x.dtype)
        _, ldy = self._matrix(out, "out", M, weight.N, x.dtype)
        self._on_stream()
        esp._check(self._lib.esp_moe_linear(self.h, code, x.shape[0], ldx, x.data_ptr(), M, _ptr(rows), weight._arg(),
                                            _ptr(offsets), ldy, out.data_ptr()), "esp_moe_linear")
        return out

    def linear_backward(self, dy, x, weight: Weight, offsets=None, rows=None, need=(True, True), out=(None, None)):
        """(dx, dw) of ``linear`` at dy (M, N): dx (M, K) in dy's type, dw (E, N, K) fp32; need: which of
        them (esp_moe_linear_backward). dx needs weights with transposed codes."""
        code, lddy = self._matrix(dy, "dy", cols=weight.N)
        _, ldx = self._matrix(x, "x", cols=weight.K, dtype=dy.dtype)
        M = self._rows(x, weight, offsets, rows)
        if dy.shape[0] != M:
            raise ValueError(f"dy: {M} rows expected")
        dx, dw = out
        lddx = 0
        if need[0]:
            if weight.qt is None:
                raise ValueError("the rows' gradient needs weights with transposed codes")
            if dx is None:
                dx = self._new((M, weight.K), dy.dtype)
            _, lddx = self._matrix(dx, "dx", M, weight.K, dy.dtype)
        if need[1]:
            if dw is None:
                dw = self._new((weight.E, weight.N, weight.K), torch.float32)
            self._need(dw, "dw", torch.float32, (weight.E, weight.N, weight.K))
        self._on_stream()
        esp._check(self._lib.esp_moe_linear_backward(
            self.h, code, x.shape[0], ldx, x.data_ptr(), M, _ptr(rows), weight._arg(), _ptr(offsets), lddy,
            dy.data_ptr(), lddx, _ptr(dx) if need[0] else None, weight.K, _ptr(dw) if need[1] else None),
            "esp_moe_linear_backward")
        return dx, dw

    # -- gated feed-forward blocks

    def gated_weight(self, inner, outer, activation: str = "silu") -> GatedWeight:
        """16-bit weights of gated blocks, inner (E, 2 F, H) and outer (E, H, F), or of one block without E. Tensors whose
        rows start at multiples of 16 bytes are used as they are, others are laid out anew (new values then go to the
        result's ``inner`` and ``outer``). Activations: silu, gelu, gelu_tanh, relu."""
        with self._queue():
            a, b = (self._laid_out(t, name) for t, name in ((inner, "inner"), (outer, "outer")))
        return GatedWeight(a, b, activation)

    def _laid_out(self, w, name: str):
        self._need(w, name)
        w = w if w.dim() == 3 else w[None]
        if w.dim() != 3:
            raise ValueError(f"{name}: a matrix for each expert expected")
        if w.dtype not in (torch.bfloat16, torch.float16):
            raise ValueError(f"{name}: type {w.dtype} not taken here")
        E, n, k = w.shape
        if _rows16(w):
            return w
        room = torch.zeros((E, n, _pad64(k)), dtype=w.dtype, device=self.device)[:, :, :k]
        room.copy_(w)
        return room

    def keep(self, M: int, weight: GatedWeight) -> Kept:
        """Room for what ``feed_forward`` keeps of M rows for their gradients."""
        weight._arg()
        F64, dt = _pad64(weight.F), weight.inner.dtype
        return Kept(self._new((M, 2, F64), torch.float32), self._new((M, F64), dt), self._new((M, _pad64(weight.H)), dt))

    def _need_kept(self, kept: Kept, M: int, weight: GatedWeight):
        F64, dt = _pad64(weight.F), weight.inner.dtype
        self._need(kept.pre, "pre", torch.float32, (M, 2, F64))
        self._need(kept.hidden, "hidden", dt, (M, F64))
        self._need(kept.rows, "rows", dt, (M, _pad64(weight.H)))

    def _block_rows(self, x, weight: GatedWeight, offsets, rows):
        weight._arg()
        self._need(weight.inner, "weight")
        code, ldx = self._matrix(x, "x", cols=weight.H, dtype=weight.inner.dtype)
        if offsets is not None:
            self._need(offsets, "offsets", torch.int32, (weight.E + 1,))
        elif weight.E != 1:
            raise ValueError("offsets: needed for more than one expert")
        M = x.shape[0]
        if rows is not None:
            M = rows.shape[0]
            self._need(rows, "rows", torch.int32, (M,))
        return M, ldx

    def feed_forward(self, x, weight: GatedWeight, offsets=None, rows=None, keep: Optional[Kept] = None, out=None):
        """y (M, H): row i of expert e is O_e (act(G_e v) * (U_e v)), v = x[rows[i]] or x[i] (esp_moe_feed_forward). Rows
        outside every expert are left as they are. keep: room that takes what the gradients need."""
        M, ldx = self._block_rows(x, weight, offsets, rows)
        if out is None:
            out = self._new((M, weight.H), x.dtype)
        _, ldy = self._matrix(out, "out", M, weight.H, x.dtype)
        kept = None
        if keep is not None:
            self._need_kept(keep, M, weight)
            kept = keep._arg()
        self._on_stream()
        esp._check(self._lib.esp_moe_feed_forward(
            self.h, weight._ref, x.shape[0], ldx, x.data_ptr(), M, _ptr(rows), _ptr(offsets), ldy, out.data_ptr(),
            None if kept is None else ctypes.byref(kept)), "esp_moe_feed_forward")
        if keep is not None:
            keep.copied = bool(kept.copied)
        return out

    def feed_forward_backward(self, dy, x, weight: GatedWeight, kept: Kept, offsets=None, rows=None,
                              need=(True, True, True), out=(None, None, None), dtype=None):
        """(dx, dinner, douter) of ``feed_forward`` at dy (M, H), called with the same arguments before: dx (M, H), dinner
        (E, 2 F, H), douter (E, H, F); need: which of them (esp_moe_feed_forward_backward). dtype: the weights' gradients'
        type where they are allocated here, the rows' or fp32."""
        M, ldx = self._block_rows(x, weight, offsets, rows)
        _, lddy = self._matrix(dy, "dy", M, weight.H, x.dtype)
        self._need_kept(kept, M, weight)
        dx, dinner, douter = (t if n else None for t, n in zip(out, need))
        dt = dtype or next((t.dtype for t in (dinner, douter) if t is not None), x.dtype)
        if dt is not x.dtype and dt is not torch.float32:
            raise ValueError(f"the weights' gradients: {x.dtype} or fp32 expected, not {dt}")
        E, F, H = weight.E, weight.F, weight.H
        lddx = H
        if need[0]:
            dx = self._new((M, H), x.dtype) if dx is None else dx
            _, lddx = self._matrix(dx, "dx", M, H, x.dtype)
        if need[1]:
            dinner = self._new((E, 2 * F, H), dt) if dinner is None else dinner
            self._need(dinner, "dinner", dt, (E, 2 * F, H))
        if need[2]:
            douter = self._new((E, H, F), dt) if douter is None else douter
            self._need(douter, "douter", dt, (E, H, F))
        self._on_stream()
        esp._check(self._lib.esp_moe_feed_forward_backward(
            self.h, weight._ref, x.shape[0], ldx, x.data_ptr(), M, _ptr(rows), _ptr(offsets), ctypes.byref(kept._arg()),
            lddy, dy.data_ptr(), lddx, _ptr(dx), _DTYPES[dt], _ptr(dinner), _ptr(douter)),
            "esp_moe_feed_forward_backward")
        return dx, dinner, douter

    # -- gradients together

    def gradients(self, tensors, out=None) -> Gradients:
        """A list of gradients for ``clip``; out: tensors of the same shapes and types that take the results."""
        return Gradients(tensors, out, self._index)

    def clip(self, gradients, max_norm: float = math.inf, scale: float = 1.0, norm=None):
        """The norm (fp32, on the device) of scale times all the gradients together, which become, in place or in their
        list's ``out``, gradient * scale * min(1, max_norm / norm) (esp_moe_clip). Where the norm is not finite they are
        scaled only. gradients: contiguous tensors, or what ``Moe.gradients`` made of them."""
        g = gradients if isinstance(gradients, Gradients) else Gradients(gradients, None, self._index)
        if g.index != self._index:
            raise ValueError(f"the gradients are on cuda:{g.index}, the handle on {self.device}")
        if norm is None:
            norm = self._new((), torch.float32)
        elif norm.numel() != 1:
            raise ValueError("norm: one element expected")
        self._need(norm, "norm", torch.float32, norm.shape)
        c = g._arg()
        self._on_stream()
        esp._check(self._lib.esp_moe_clip(self.h, len(c), c, max_norm, scale, norm.data_ptr()), "esp_moe_clip")
        return norm

    # -- return of the rows

    def combine(self, y, pos, weight=None, out=None):
        """out (T, H): the rows y[pos[t, j]] (those with pos >= 0) times weight[t, j], summed (esp_moe_combine)."""
        code, ldy = self._matrix(y, "y")
        M, H = y.shape
        self._need(pos, "pos", torch.int32, (pos.shape[0], pos.shape[-1]))
        T, k = pos.shape
        self._need(weight, "weight", torch.float32, (T, k), optional=True)
        if out is None:
            out = self._new((T, H), y.dtype)
        _, ldo = self._matrix(out, "out", T, H, y.dtype)
        self._on_stream()
        esp._check(self._lib.esp_moe_combine(self.h, code, T, k, H, M, ldy, y.data_ptr(), pos.data_ptr(), _ptr(weight),
                                             ldo, out.data_ptr()), "esp_moe_combine")
        return out

    def combine_backward(self, dout, y, pos, weight=None, out=(None, None)):
        """(dy, dweight) of ``combine`` at dout (T, H) (esp_moe_combine_backward). Rows that no pos names are
        left as they are in dy; a new dy holds zeros there."""
        code, lddo = self._matrix(dout, "dout")
        T, H = dout.shape
        _, ldy = self._matrix(y, "y", cols=H, dtype=dout.dtype)
        self._need(pos, "pos", torch.int32, (T, pos.shape[-1]))
        k = pos.shape[1]
        self._need(weight, "weight", torch.float32, (T, k), optional=True)
        dy, dweight = out
        if dy is None:
            with self._queue():
                dy = torch.zeros(y.shape, dtype=y.dtype, device=self.device)
        _, lddy = self._matrix(dy, "dy", y.shape[0], H, y.dtype)
        if dweight is None:
            dweight = self._new((T, k), torch.float32)
        self._need(dweight, "dweight", torch.float32, (T, k))
        self._on_stream()
        esp._check(self._lib.esp_moe_combine_backward(
            self.h, code, T, k, H, y.shape[0], lddo, dout.data_ptr(), ldy, y.data_ptr(), pos.data_ptr(), _ptr(weight),
            lddy, dy.data_ptr(), dweight.data_ptr()), "esp_moe_combine_backward")
        return dy, dweight

    # -- handle

    def synchronize(self) -> None:
        """Waits for the queued calls; raises if a product kernel gave up a bounded wait (any later call that finds
        that raises too, but does not wait)."""
        esp._check(self._lib.esp_moe_synchronize(self.h), "esp_moe_synchronize")

    def last_launch_count(self) -> int:
        n = ctypes.c_int64()
        esp._check(self._lib.esp_moe_last_launch_count(self.h, ctypes.byref(n)), "esp_moe_last_launch_count")
        return n.value

    def close(self) -> None:
        if self.h:
            self._lib.esp_moe_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
