"""Operators of a mixture-of-experts training step on the gfx950 kernels of libhapmoe.so.

The planner's inputs -- router statistics, router and expert times, optimizer time per
parameter -- are quantities of these operators:

  route, route_backward            a token's experts, weights and counts, and the rows' order
  expert_matmul, .._grad_x, .._w   products grouped by expert, with both gradients
  combine, combine_backward        a token's expert outputs put together
  AdamW                            the optimizer step, moments in 32 or 8 bits

and what stands around the layer in a training step:

  embed, embed_backward            the first stage's table, its gradient summed by token
  layer_norm, .._backward          rows' norm with or without the mean, the weight's gradient over rows
  route_balanced, .._backward      a router of scores, a bias for the choice and groups of experts
  dropout, dropout_backward        by a counter-based generator, without a mask, onto a residual

Thin calls of the C functions in include/hapmoe.h, which states each formula.  Tensors are on
the current device; work is enqueued on its current stream and outputs are allocated there
unless they are given.  A tensor, size or number that an operator cannot take raises ValueError
before anything is launched.  No call records a graph for automatic differentiation: gradients
are calls of their own.  There is no fallback path: without the library the first call raises.
"""
from __future__ import annotations

import array
import ctypes as C
import operator

import torch

from . import binding

F32, BF16, F16 = 0, 1, 2
INVAL = -1
MAX_EXPERTS = 1024
MAX_TOP_K = 32
BLOCK = 256   # elements that share an exponent in an 8-bit moment

_POINTER = torch.Tensor.data_ptr
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_LIB = None


class _Tensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("copy", C.c_void_p), ("m", C.c_void_p),
                ("v", C.c_void_p), ("m_exp", C.c_void_p), ("v_exp", C.c_void_p), ("n", C.c_int64),
                ("weight_decay", C.c_float), ("reserved", C.c_int32)]


class _Args(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("grad_scale", C.c_double), ("step", C.c_int64), ("seed", C.c_uint64), ("d_skip", C.c_void_p),
                ("grad_type", C.c_int32), ("copy_type", C.c_int32), ("state_bits", C.c_int32),
                ("reserved", C.c_int32)]


def _lib():
    global _LIB
    if _LIB is None:
        L = binding.lib()
        i32, i64, vp, f32 = C.c_int32, C.c_int64, C.c_void_p, C.c_float
        for name, args in {
                "hapmoe_route_ws_bytes": [i64, i32, i32, C.POINTER(i64)],
                "hapmoe_route": [vp, i32, i64, i64, i32, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, i64, vp],
                "hapmoe_route_backward": [vp, i32, i64, i64, i32, i32, vp, i32, vp, vp, vp, vp, vp],
                "hapmoe_combine": [vp, i32, i64, i64, i32, i64, vp, vp, vp, vp],
                "hapmoe_combine_backward": [vp, vp, i32, i64, i32, i64, vp, vp, vp, vp, vp, vp],
                "hapmoe_expert_matmul": [vp, i64, i64, vp, i32, i64, i32, i64, i64, vp, vp, i32, vp, vp],
                "hapmoe_expert_matmul_grad_x": [vp, i64, vp, i32, i64, i32, i64, i64, vp, vp, vp],
                "hapmoe_expert_matmul_grad_w": [vp, i64, vp, i64, i64, i32, i64, i32, i64, i64, vp, vp, i32, i32, vp,
                                                vp],
                "hapmoe_route_balanced": [vp, i32, i64, i64, i32, i32, vp, i32, i32, i32, i32, vp, i32, f32, vp, vp, vp, vp,
                                          vp, vp, vp, i64, vp],
                "hapmoe_route_balanced_backward": [vp, i32, i64, i64, i32, i32, i32, vp, i32, f32, vp, vp, vp, vp, vp],
                "hapmoe_layer_norm": [vp, i32, i64, i64, i64, vp, vp, i32, f32, vp, vp, vp, vp],
                "hapmoe_layer_norm_ws_bytes": [i64, i64, C.POINTER(i64)],
                "hapmoe_layer_norm_backward": [vp, i64, vp, i32, i64, i64, i64, vp, i32, vp, vp, vp, i64, vp, vp, vp, vp,
                                               i64, vp],
                "hapmoe_embed": [vp, i32, i64, vp, i32, i64, i64, i64, f32, vp, vp],
                "hapmoe_embed_ws_bytes": [i64, i64, C.POINTER(i64)],
                "hapmoe_embed_backward": [vp, i32, i64, i64, i64, vp, i32, i64, f32, i32, vp, vp, i64, vp],
                "hapmoe_dropout": [vp, i32, i64, i64, i64, vp, i64, C.c_double, C.c_uint64, C.c_uint64, vp, vp, vp],
                "hapmoe_adamw": [C.POINTER(_Tensor), vp, i32, C.POINTER(_Args), vp],
                "hapmoe_adamw_moments": [C.POINTER(_Tensor), vp, vp, i32, i32, vp]}.items():
            f = getattr(L, name)
            f.argtypes, f.restype = args, i32
        _LIB = L
    return _LIB


class InvalidArgument(binding.HapmoeError, ValueError):
    """A size or number that the C call refuses."""


def _check(code, what):
    if code != 0:
        raise (InvalidArgument if code == INVAL else binding.HapmoeError)(code, what)


try:   # the current stream's address without an object for it: 0.1 us of a call, where the object takes 2
    from torch._C import _cuda_getCurrentRawStream as _stream_of, _cuda_getDevice as _device
except ImportError:
    _device = torch.cuda.current_device

    def _stream_of(index):
        return torch.cuda.current_stream(index).cuda_stream


def _stream(t):
    return _stream_of(t.get_device())


def _need(ok, what):
    if not ok:
        raise ValueError(what)


# A call looks at a number's class itself before it asks these, which takes 0.1 us less.
def _whole(name, x):
    """A whole number, of Python or of what stands for one."""
    try:
        return operator.index(x)
    except Exception as e:   # a tensor of several elements has errors of its own
        raise ValueError(f"{name}: a whole number, not {x!r}") from e


def _real(name, x):
    """A number that 64 bits hold."""
    try:
        return C.c_double(x).value
    except Exception as e:
        raise ValueError(f"{name}: a number, not {x!r}") from e


def _on_device(name, t):
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise ValueError(f"{name}: a tensor on the GPU")
    if t.get_device() != _device():
        raise ValueError(f"{name}: on {t.device}, which is not the current device")


# The checks below run on every call, which a decoding step waits for: one expression where all is well, and only where it
# is not the tests one by one, with their messages.
def _array(name, t, dtype, *shape):
    """A contiguous tensor of this type and shape (None in the shape: any)."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.shape == shape \
            and t.is_contiguous() and t.get_device() == _device():
        return
    _on_device(name, t)
    if t.dtype != dtype:
        raise ValueError(f"{name}: {dtype}, not {t.dtype}")
    if t.dim() != len(shape) or any(want is not None and have != want for have, want in zip(t.shape, shape)):
        raise ValueError(f"{name}: shape {shape}, not {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: contiguous")


def _matrix(name, t, types):
    """A matrix of one of the types whose rows are contiguous; the distance of its rows in elements."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in types and t.dim() == 2 and t.is_contiguous() \
            and t.get_device() == _device() and t.shape[1]:
        return t.shape[1]
    _on_device(name, t)
    if t.dtype not in types:
        raise ValueError(f"{name}: one of {', '.join(str(x) for x in types)}, not {t.dtype}")
    if t.dim() != 2 or t.shape[1] == 0:
        raise ValueError(f"{name}: a matrix with columns, not {tuple(t.shape)}")
    rows, columns = t.shape
    step, unit = t.stride()
    if unit != 1 and columns > 1:
        raise ValueError(f"{name}: its rows have to be contiguous")
    if rows <= 1:
        return columns
    if step < columns:
        raise ValueError(f"{name}: its rows overlap")
    return step


# ---------------------------------------------------------------- the router
class Routing:
    """What ``route`` returns, and the buffers it writes: kept by a caller, they serve call after call of
    the same sizes (on one stream at a time).

    expert [tokens, top_k] int32 (-1: none), weight [tokens, top_k] fp32, count [experts] int32,
    offset [experts + 1] int32, slot [tokens * top_k] int32 and place [tokens, top_k] int32 as in
    include/hapmoe.h.  A Routing whose tensors were replaced is refused.
    """

    def __init__(self, tokens: int, experts: int, top_k: int, device="cuda"):
        need = C.c_int64(0)
        tokens, experts, top_k = _whole("tokens", tokens), _whole("experts", experts), _whole("top_k", top_k)
        _need(0 <= tokens and 1 <= experts <= MAX_EXPERTS and 1 <= top_k <= min(experts, MAX_TOP_K)
              and tokens * top_k < 2**31, f"no routing of {tokens} tokens to {top_k} of {experts} experts")
        _check(_lib().hapmoe_route_ws_bytes(tokens, experts, top_k, C.byref(need)), "hapmoe_route_ws_bytes")
        self.tokens, self.experts, self.top_k = tokens, experts, top_k
        i32 = {"dtype": torch.int32, "device": device}
        self.expert = torch.empty((tokens, top_k), **i32)
        self.weight = torch.empty((tokens, top_k), dtype=torch.float32, device=device)
        self.count = torch.empty(experts, **i32)
        self.offset = torch.empty(experts + 1, **i32)
        self.slot = torch.empty(tokens * top_k, **i32)
        self.place = torch.empty((tokens, top_k), **i32)
        self._ws = torch.empty(need.value, dtype=torch.uint8, device=device)
        self._outputs = self._addresses()
        self._ws_bytes = need.value

    def _addresses(self):
        return tuple(map(_POINTER, (self.weight, self.expert, self.count, self.offset, self.slot, self.place, self._ws)))


def _keep(keep, tokens):
    if keep is None:
        return None
    _on_device("keep", keep)
    _array("keep", keep, torch.uint8 if keep.dtype == torch.uint8 else torch.bool, tokens)
    return keep.data_ptr()


def route(logits, top_k: int, keep=None, renormalize=True, out: Routing = None) -> Routing:
    """The top_k experts of every row of ``logits`` [tokens, experts] and their softmax weights
    (``hapmoe_route``).  keep [tokens] bool: tokens with False take none.  renormalize: weights of the
    chosen add up to 1.  out: a ``Routing`` of these sizes to write to."""
    stride = _matrix("logits", logits, _TYPES)
    top_k = top_k if top_k.__class__ is int else _whole("top_k", top_k)
    tokens, experts = logits.shape
    if out is None:
        out = Routing(tokens, experts, top_k, logits.device)
    else:
        _need((out.tokens, out.experts, out.top_k) == (tokens, experts, top_k) and
              out.expert.device == logits.device, "out: made for other sizes or another device")
        # the call writes to these addresses, whatever the attributes name by now
        _need(out._addresses() == out._outputs, "out: a buffer was replaced")
    _check(_lib().hapmoe_route(logits.data_ptr(), _TYPES[logits.dtype], stride, tokens, experts, top_k,
                               _keep(keep, tokens), 1 if renormalize else 0, *out._outputs, out._ws_bytes, _stream(logits)),
           "hapmoe_route")
    return out


def route_backward(logits, routing: Routing, d_weight, keep=None, renormalize=True):
    """The gradient of the logits from that of the weights [tokens, top_k] fp32
    (``hapmoe_route_backward``), with the forward call's routing, keep and renormalize."""
    stride = _matrix("logits", logits, _TYPES)
    tokens, experts = logits.shape
    _need((routing.tokens, routing.experts) == (tokens, experts), "routing: made for other sizes")
    k = routing.top_k
    _array("routing.expert", routing.expert, torch.int32, tokens, k)
    _array("routing.weight", routing.weight, torch.float32, tokens, k)
    _array("d_weight", d_weight, torch.float32, tokens, k)
    d_logits = logits.new_empty((tokens, experts))
    _check(_lib().hapmoe_route_backward(logits.data_ptr(), _TYPES[logits.dtype], stride, tokens, experts, k,
                                        _keep(keep, tokens), 1 if renormalize else 0, routing.expert.data_ptr(),
                                        routing.weight.data_ptr(), d_weight.data_ptr(), d_logits.data_ptr(),
                                        _stream(logits)), "hapmoe_route_backward")
    return d_logits


SCORES = {"softmax": 0, "sigmoid": 1}
MAX_GROUPS = 64


def route_balanced(logits, top_k: int, bias=None, scores="sigmoid", groups=1, top_groups=None, group_best=2, keep=None,
                   renormalize=True, scale=1.0, out: Routing = None) -> Routing:
    """The top_k experts of every row of ``logits`` [tokens, experts] by their score ("sigmoid" or "softmax") plus
    ``bias`` [experts] fp32, out of the ``top_groups`` of ``groups`` equal groups of experts whose ``group_best`` (1 or
    2) best add up to most; weights are the scores without the bias, times ``scale`` (``hapmoe_route_balanced``).
    top_groups: None: all groups.  keep, renormalize and out as in ``route``."""
    stride = _matrix("logits", logits, _TYPES)
    tokens, experts = logits.shape
    kind = _scores(scores)
    top_groups = groups if top_groups is None else top_groups
    if not (top_k.__class__ is groups.__class__ is top_groups.__class__ is group_best.__class__ is int):
        top_k, groups = _whole("top_k", top_k), _whole("groups", groups)
        top_groups, group_best = _whole("top_groups", top_groups), _whole("group_best", group_best)
    scale = scale if scale.__class__ is float else _real("scale", scale)
    if not 1 <= groups <= MAX_GROUPS or experts % groups or not 1 <= top_groups <= groups or group_best not in (1, 2):
        raise ValueError(f"no choice of {group_best} of {top_groups} of {groups} groups of {experts} experts")
    if bias is not None:
        _array("bias", bias, torch.float32, experts)
    if out is None:
        out = Routing(tokens, experts, top_k, logits.device)
    else:
        _need((out.tokens, out.experts, out.top_k) == (tokens, experts, top_k) and
              out.expert.device == logits.device, "out: made for other sizes or another device")
        _need(out._addresses() == out._outputs, "out: a buffer was replaced")
    _check(_lib().hapmoe_route_balanced(logits.data_ptr(), _TYPES[logits.dtype], stride, tokens, experts, top_k,
                                        None if bias is None else bias.data_ptr(), kind, groups, top_groups, group_best,
                                        _keep(keep, tokens), 1 if renormalize else 0, scale, *out._outputs,
                                        out._ws_bytes, _stream(logits)), "hapmoe_route_balanced")
    return out


def _scores(scores):
    kind = SCORES.get(scores) if isinstance(scores, str) else None
    if kind is None:
        raise ValueError(f"scores: one of {', '.join(SCORES)}, not {scores}")
    return kind


def route_balanced_backward(logits, routing: Routing, d_weight, scores="sigmoid", keep=None, renormalize=True, scale=1.0):
    """The gradient of the logits from that of the weights [tokens, top_k] fp32
    (``hapmoe_route_balanced_backward``), with the forward call's routing, scores, keep, renormalize and scale."""
    stride = _matrix("logits", logits, _TYPES)
    tokens, experts = logits.shape
    kind = _scores(scores)
    scale = scale if scale.__class__ is float else _real("scale", scale)
    _need((routing.tokens, routing.experts) == (tokens, experts), "routing: made for other sizes")
    k = routing.top_k
    _array("routing.expert", routing.expert, torch.int32, tokens, k)
    _array("routing.weight", routing.weight, torch.float32, tokens, k)
    _array("d_weight", d_weight, torch.float32, tokens, k)
    d_logits = logits.new_empty((tokens, experts))
    _check(_lib().hapmoe_route_balanced_backward(
        logits.data_ptr(), _TYPES[logits.dtype], stride, tokens, experts, k, kind, _keep(keep, tokens),
        1 if renormalize else 0, scale, routing.expert.data_ptr(), routing.weight.data_ptr(), d_weight.data_ptr(),
        d_logits.data_ptr(), _stream(logits)), "hapmoe_route_balanced_backward")
    return d_logits


# --------------------------------------------------- a token's expert outputs
def _rows(name, t):
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in _TYPES and t.dim() == 2 and t.shape[1] \
            and t.is_contiguous() and t.get_device() == _device():
        return
    if _matrix(name, t, _TYPES) != t.shape[1]:
        raise ValueError(f"{name}: contiguous")


def _choices_of(place):
    shape = getattr(place, "shape", ())
    _array("place", place, torch.int32, *(shape if len(shape) == 2 else (None, None)))
    tokens, top_k = place.shape
    if not 1 <= top_k <= MAX_TOP_K:
        raise ValueError(f"place: 1 to {MAX_TOP_K} choices, not {top_k}")
    return tokens, top_k


def combine(y, place, weight=None):
    """out[t] = sum over j of weight[t, j] * y[place[t, j]] (``hapmoe_combine``); without weights, the sum:
    the gradient of the rows that ``expert_matmul`` gathers through slot."""
    _rows("y", y)
    tokens, top_k = _choices_of(place)
    if weight is not None:
        _array("weight", weight, torch.float32, tokens, top_k)
    rows, hidden = y.shape
    out = y.new_empty((tokens, hidden))
    _check(_lib().hapmoe_combine(y.data_ptr(), _TYPES[y.dtype], rows, tokens, top_k, hidden,
                                 place.data_ptr(), None if weight is None else weight.data_ptr(), out.data_ptr(),
                                 _stream(y)), "hapmoe_combine")
    return out


def combine_backward(d_out, y, slot, place, weight):
    """The gradients (d_y [rows, hidden], d_weight [tokens, top_k] fp32) of ``combine`` from that of its result
    (``hapmoe_combine_backward``); rows = tokens * top_k."""
    _rows("y", y)
    tokens, top_k = _choices_of(place)
    _array("y", y, y.dtype, tokens * top_k, None)
    hidden = y.shape[1]
    _array("d_out", d_out, y.dtype, tokens, hidden)
    _array("slot", slot, torch.int32, tokens * top_k)
    _array("weight", weight, torch.float32, tokens, top_k)
    d_y = torch.empty_like(y)
    d_weight = torch.empty_like(weight)
    _check(_lib().hapmoe_combine_backward(d_out.data_ptr(), y.data_ptr(), _TYPES[y.dtype], tokens, top_k, hidden,
                                          slot.data_ptr(), place.data_ptr(), weight.data_ptr(), d_y.data_ptr(),
                                          d_weight.data_ptr(), _stream(y)), "hapmoe_combine_backward")
    return d_y, d_weight


# ------------------------------------------------- products grouped by expert
_HALF = (torch.bfloat16, torch.float16)


def _rows_of(x, slot, top_k):
    top_k.__class__ is int or _whole("top_k", top_k)
    if slot is None:
        return x.shape[0]
    _array("slot", slot, torch.int32, None)
    if not -2**31 <= top_k < 2**31:   # the call's 32 bits; it refuses those below 1
        raise ValueError(f"top_k: at least 1 and below 2^31, not {top_k}")
    return slot.shape[0]


def _experts_of(offset):
    _array("offset", offset, torch.int32, None)
    experts = offset.shape[0] - 1
    if not 1 <= experts <= MAX_EXPERTS:
        raise ValueError(f"offset: 2 to {MAX_EXPERTS + 1} entries, not {experts + 1}")
    return experts


def expert_matmul(x, w, offset, slot=None, top_k=1):
    """y[i] = w[e] x[i] for the rows offset[e] .. offset[e + 1] of every expert e (``hapmoe_expert_matmul``).
    x [rows, inputs] and w [experts, outputs, inputs] bf16 or fp16; with slot [rows], row i is
    x[slot[i] // top_k], as ``route`` orders them."""
    stride = _matrix("x", x, _HALF)
    experts = _experts_of(offset)
    _array("w", w, x.dtype, experts, None, x.shape[1])
    _need(w.shape[1] > 0, "w: no outputs")
    rows = _rows_of(x, slot, top_k)
    y = x.new_empty((rows, w.shape[1]))
    _check(_lib().hapmoe_expert_matmul(x.data_ptr(), x.shape[0], stride, w.data_ptr(), _TYPES[x.dtype], rows, experts,
                                       w.shape[1], w.shape[2], offset.data_ptr(),
                                       None if slot is None else slot.data_ptr(), top_k, y.data_ptr(), _stream(x)),
           "hapmoe_expert_matmul")
    return y


def expert_matmul_grad_x(d_y, w, offset):
    """The gradient of the rows, w[e]^T d_y[i] (``hapmoe_expert_matmul_grad_x``).  Of rows that were gathered
    through slot, ``combine(d_x, place)`` adds up those of each token."""
    stride = _matrix("d_y", d_y, _HALF)
    experts = _experts_of(offset)
    _array("w", w, d_y.dtype, experts, d_y.shape[1], None)
    _need(w.shape[2] > 0, "w: no inputs")
    d_x = d_y.new_empty((d_y.shape[0], w.shape[2]))
    _check(_lib().hapmoe_expert_matmul_grad_x(d_y.data_ptr(), stride, w.data_ptr(), _TYPES[d_y.dtype], d_y.shape[0],
                                              experts, w.shape[1], w.shape[2], offset.data_ptr(), d_x.data_ptr(),
                                              _stream(d_y)), "hapmoe_expert_matmul_grad_x")
    return d_x


def expert_matmul_grad_w(d_y, x, offset, slot=None, top_k=1, dtype=torch.float32):
    """The gradient of the weights [experts, outputs, inputs], in fp32 or the inputs' type
    (``hapmoe_expert_matmul_grad_w``); x, slot and top_k as in ``expert_matmul``."""
    step = _matrix("d_y", d_y, _HALF)
    stride = _matrix("x", x, (d_y.dtype,))
    experts = _experts_of(offset)
    rows = _rows_of(x, slot, top_k)
    if dtype not in (torch.float32, d_y.dtype):
        raise ValueError(f"dtype: torch.float32 or {d_y.dtype}, not {dtype}")
    if rows != d_y.shape[0]:
        raise ValueError(f"d_y: {rows} rows, not {d_y.shape[0]}")
    d_w = torch.empty((experts, d_y.shape[1], x.shape[1]), dtype=dtype, device=x.device)
    _check(_lib().hapmoe_expert_matmul_grad_w(d_y.data_ptr(), step, x.data_ptr(), x.shape[0], stride,
                                              _TYPES[x.dtype], rows, experts,
                                              d_y.shape[1], x.shape[1], offset.data_ptr(),
                                              None if slot is None else slot.data_ptr(), top_k, _TYPES[dtype],
                                              d_w.data_ptr(), _stream(x)), "hapmoe_expert_matmul_grad_w")
    return d_w


# ----------------------------------------------------------- around the layer
def _vector(name, t, types, n):
    """A contiguous vector of n elements (None: any) of one of the types."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in types and t.dim() == 1 and (n is None or t.shape[0] == n) \
            and t.is_contiguous() and t.get_device() == _device():
        return
    _on_device(name, t)
    if t.dtype not in types:
        raise ValueError(f"{name}: one of {', '.join(str(x) for x in types)}, not {t.dtype}")
    _array(name, t, t.dtype, n)


def layer_norm(x, weight, bias=None, eps=1e-5, center=True):
    """y = (x - mean) * rstd * weight + bias of the rows of ``x`` [rows, hidden] (``hapmoe_layer_norm``), and mean and
    rstd [rows] fp32, which ``layer_norm_backward`` takes.  center False: mean counts as 0 (root mean square norm) and
    is None.  weight and bias [hidden]: fp32 or x's type, both the same."""
    stride = _matrix("x", x, _TYPES)
    eps = eps if eps.__class__ is float else _real("eps", eps)
    rows, hidden = x.shape
    _vector("weight", weight, (torch.float32, x.dtype), hidden)
    if bias is not None:
        _array("bias", bias, weight.dtype, hidden)
    y = x.new_empty((rows, hidden))
    rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    mean = torch.empty_like(rstd) if center else None
    _check(_lib().hapmoe_layer_norm(x.data_ptr(), _TYPES[x.dtype], stride, rows, hidden, weight.data_ptr(),
                                    None if bias is None else bias.data_ptr(), _TYPES[weight.dtype], eps,
                                    None if mean is None else mean.data_ptr(), rstd.data_ptr(), y.data_ptr(),
                                    _stream(x)), "hapmoe_layer_norm")
    return y, mean, rstd


def layer_norm_backward(d_y, x, weight, mean, rstd, add=None, bias=True):
    """The gradients (d_x, d_weight [hidden] fp32, d_bias [hidden] fp32) of ``layer_norm`` from that of y
    (``hapmoe_layer_norm_backward``); mean None: of the form that is not centred.  add [rows, hidden]: a gradient
    that reaches x another way, added to d_x.  bias False: d_bias is None."""
    stride = _matrix("x", x, _TYPES)
    rows, hidden = x.shape
    steps = []
    for name, t in (("d_y", d_y), ("add", add)):
        if t is None and name == "add":
            steps.append(hidden)
            continue
        steps.append(_matrix(name, t, (x.dtype,)))
        if t.shape != x.shape:
            raise ValueError(f"{name}: shape {tuple(x.shape)}, not {tuple(t.shape)}")
    _vector("weight", weight, (torch.float32, x.dtype), hidden)
    _array("rstd", rstd, torch.float32, rows)
    if mean is not None:
        _array("mean", mean, torch.float32, rows)
    need = C.c_int64(0)
    _check(_lib().hapmoe_layer_norm_ws_bytes(rows, hidden, C.byref(need)), "hapmoe_layer_norm_ws_bytes")
    d_x = x.new_empty((rows, hidden))
    d_weight = torch.empty(hidden, dtype=torch.float32, device=x.device)
    d_bias = torch.empty_like(d_weight) if bias else None
    ws = torch.empty(need.value, dtype=torch.uint8, device=x.device)
    _check(_lib().hapmoe_layer_norm_backward(
        d_y.data_ptr(), steps[0], x.data_ptr(), _TYPES[x.dtype], stride, rows, hidden, weight.data_ptr(),
        _TYPES[weight.dtype], None if mean is None else mean.data_ptr(), rstd.data_ptr(),
        None if add is None else add.data_ptr(), steps[1], d_x.data_ptr(), d_weight.data_ptr(),
        None if d_bias is None else d_bias.data_ptr(), ws.data_ptr(), need.value, _stream(x)),
        "hapmoe_layer_norm_backward")
    return d_x, d_weight, d_bias


_TOKEN_BITS = {torch.int32: 32, torch.int64: 64}


def embed(token, table, scale=1.0):
    """out[t] = scale * table[token[t]] for ``token`` [tokens] int32 or int64 and ``table`` [vocab, hidden]
    (``hapmoe_embed``); a token out of the table gives a row of zeros."""
    stride = _matrix("table", table, _TYPES)
    scale = scale if scale.__class__ is float else _real("scale", scale)
    _vector("token", token, _TOKEN_BITS, None)
    vocab, hidden = table.shape
    out = table.new_empty((token.shape[0], hidden))
    _check(_lib().hapmoe_embed(token.data_ptr(), _TOKEN_BITS[token.dtype], token.shape[0], table.data_ptr(),
                               _TYPES[table.dtype], stride, vocab, hidden, scale, out.data_ptr(), _stream(table)),
           "hapmoe_embed")
    return out


def embed_backward(d_out, token, vocab: int, scale=1.0, into=None):
    """The gradient of ``embed``'s table [vocab, hidden] in fp32 from that of its result
    (``hapmoe_embed_backward``).  into: an fp32 gradient of that shape that it is added to, which is returned; rows
    without a token stay as they are.  Each row's sum has a fixed order."""
    stride = _matrix("d_out", d_out, _TYPES)
    scale, vocab = scale if scale.__class__ is float else _real("scale", scale), _whole("vocab", vocab)
    tokens, hidden = d_out.shape
    _vector("token", token, _TOKEN_BITS, tokens)
    if not 1 <= vocab < 2**31 - 1:
        raise ValueError(f"vocab: at least 1 and below 2^31 - 1, not {vocab}")
    if into is None:
        d_table = torch.empty((vocab, hidden), dtype=torch.float32, device=d_out.device)
    else:
        _array("into", into, torch.float32, vocab, hidden)
        d_table = into
    need = C.c_int64(0)
    _check(_lib().hapmoe_embed_ws_bytes(tokens, hidden, C.byref(need)), "hapmoe_embed_ws_bytes")
    ws = torch.empty(need.value, dtype=torch.uint8, device=d_out.device)
    _check(_lib().hapmoe_embed_backward(d_out.data_ptr(), _TYPES[d_out.dtype], stride, tokens, hidden, token.data_ptr(),
                                        _TOKEN_BITS[token.dtype], vocab, scale, 0 if into is None else 1,
                                        d_table.data_ptr(), ws.data_ptr(), need.value, _stream(d_out)),
           "hapmoe_embed_backward")
    return d_table


def dropout(x, p, seed, offset=0, residual=None, counter=None):
    """residual + x / (1 - p) where an element of ``x`` [rows, columns] is kept, residual (or 0) where it is dropped,
    with a chance of p rounded to a multiple of 2^-16 (``hapmoe_dropout``).  Which are dropped is a function of seed,
    offset and the element's index alone: give every dropout of a step another offset.  counter: an int64 tensor [1] on
    the device that is added to offset when the call runs, for captured calls."""
    stride = _matrix("x", x, _TYPES)
    p = p if p.__class__ is float else _real("p", p)
    if not (seed.__class__ is offset.__class__ is int):
        seed, offset = _whole("seed", seed), _whole("offset", offset)
    step = 0
    if residual is not None:
        step = _matrix("residual", residual, (x.dtype,))
        if residual.shape != x.shape:
            raise ValueError(f"residual: shape {tuple(x.shape)}, not {tuple(residual.shape)}")
    if counter is not None:
        _array("counter", counter, torch.int64, 1)
    rows, columns = x.shape
    out = x.new_empty((rows, columns))
    _check(_lib().hapmoe_dropout(x.data_ptr(), _TYPES[x.dtype], stride, rows, columns,
                                 None if residual is None else residual.data_ptr(), step, p, seed & (2**64 - 1),
                                 offset & (2**64 - 1), None if counter is None else counter.data_ptr(), out.data_ptr(),
                                 _stream(x)), "hapmoe_dropout")
    return out


def dropout_backward(d_out, p, seed, offset=0, counter=None):
    """The gradient of ``dropout``'s x from that of its result, with the forward call's numbers; that of residual is
    d_out."""
    return dropout(d_out, p, seed, offset, None, counter)


# -------------------------------------------------------------- the optimizer
_CONTIGUOUS, _NUMEL = torch.Tensor.is_contiguous, torch.Tensor.numel
_DEVICE, _DTYPE = torch.Tensor.get_device, operator.attrgetter("dtype")


class AdamW:
    """AdamW over the caller's tensors, in place (``hapmoe_adamw``).

    params: fp32 (the masters); m, v: fp32 of the same sizes, or uint8 codes with m_exp and v_exp
    (int8, one for every 256 elements, the last of a tensor fewer); copies: None, or a bf16 or fp16
    tensor for each parameter that gets its new value; weight_decay: one number, or one for each.
    All contiguous, and kept alive by this object, which holds nothing else: state that starts at
    zero is zeros of these tensors.  Their memory is that of the moment this object is made: after
    one was given other storage (``p.data = q``, ``set_``, a resize) make another AdamW of them.
    """

    def __init__(self, params, m, v, copies=None, m_exp=None, v_exp=None, weight_decay=0.0):
        params, m, v = list(params), list(m), list(v)
        n = len(params)
        self.state_bits = 8 if m_exp is not None else 32
        _need((m_exp is None) == (v_exp is None), "m_exp and v_exp: both or neither")
        m_exp, v_exp = (None, None) if m_exp is None else (list(m_exp), list(v_exp))
        copies = None if copies is None else list(copies)
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * n
        for name, x in (("m", m), ("v", v), ("copies", copies), ("m_exp", m_exp), ("v_exp", v_exp),
                        ("weight_decay", decay)):
            _need(x is None or len(x) == n, f"{name}: one for each of {n} parameters")
        self.copy_type = None
        state = torch.float32 if self.state_bits == 32 else torch.uint8
        for i, p in enumerate(params):
            _on_device(f"params[{i}]", p)
            shape = tuple(p.shape)
            _array(f"params[{i}]", p, torch.float32, *shape)
            for name, x in (("m", m), ("v", v)):
                _on_device(f"{name}[{i}]", x[i])
                _need(x[i].numel() == p.numel(), f"{name}[{i}]: {p.numel()} elements, not {x[i].numel()}")
                _array(f"{name}[{i}]", x[i], state, *x[i].shape)
            for name, x in (("m_exp", m_exp), ("v_exp", v_exp)):
                if x is not None:
                    _array(f"{name}[{i}]", x[i], torch.int8, -(-p.numel() // BLOCK))
            if copies is not None:
                _on_device(f"copies[{i}]", copies[i])
                _need(copies[i].dtype in _HALF and copies[i].dtype == copies[0].dtype,
                      f"copies[{i}]: all torch.bfloat16 or all torch.float16")
                _array(f"copies[{i}]", copies[i], copies[0].dtype, *shape)
            decay[i] = _real(f"weight_decay[{i}]", decay[i])
            _need(decay[i] >= 0, f"weight_decay[{i}]: at least 0")
        self._index = params[0].get_device() if n else None
        self._kept = (params, m, v)
        # what the table's addresses lie in: a tensor given other storage would let go of it
        self._memory = [t.detach() for x in (params, m, v, copies, m_exp, v_exp) if x is not None for t in x]
        self._sizes = [p.numel() for p in params]
        self._table = (_Tensor * max(n, 1))()
        self._pointers = C.c_void_p * max(n, 1)
        self._args = _Args(copy_type=_TYPES[copies[0].dtype] if copies else 0, state_bits=self.state_bits)
        self._args_at = C.byref(self._args)
        for i, t in enumerate(self._table[:n]):
            t.param, t.m, t.v, t.n = params[i].data_ptr(), m[i].data_ptr(), v[i].data_ptr(), params[i].numel()
            t.copy = copies[i].data_ptr() if copies else None
            t.m_exp, t.v_exp = (m_exp[i].data_ptr(), v_exp[i].data_ptr()) if m_exp else (None, None)
            t.weight_decay = decay[i]

    def step(self, grads, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, seed=0, skip=None):
        """One step from one gradient for each parameter (contiguous, all of one type).  step: 1 for the first.
        grad_scale multiplies the gradients.  seed: of the 8-bit moments' roundings, another for every step.
        skip: an int32 tensor [1] on the device; if it is not 0 nothing changes.
        A captured step replays with the numbers of its capture: only with moments in 32 bits, at one lr and step."""
        n = len(self._sizes)
        if len(grads) != n:
            raise ValueError(f"grads: {n}, not {len(grads)}")
        a = self._args
        if n:
            index = self._index
            if index != _device():
                raise ValueError(f"the parameters' device {index} is not the current device")
            # list by list: a step over many small tensors waits for these checks
            try:
                dtype = grads[0].dtype
                fine = (set(map(_DTYPE, grads)) == {dtype} and dtype in _TYPES and set(map(_DEVICE, grads)) == {index}
                        and list(map(_NUMEL, grads)) == self._sizes and all(map(_CONTIGUOUS, grads)))
            except (AttributeError, TypeError):   # not all of them are tensors
                fine = False
            if not fine:
                raise ValueError(f"grads: contiguous tensors on device {index}, of one floating type of 32 or 16 bits and "
                                 "the parameters' sizes")
            a.grad_type = _TYPES[dtype]
        if not (step.__class__ is seed.__class__ is int):
            step, seed = _whole("step", step), _whole("seed", seed)
        if not -2**63 <= step < 2**63:   # the call's 64 bits; it refuses those below 1
            raise ValueError(f"step: {step}")
        try:
            a.lr, a.beta1, a.beta2, a.eps, a.grad_scale, a.step = lr, beta1, beta2, eps, grad_scale, step
        except Exception:   # with the name of the one that is no number
            for name, x in (("lr", lr), ("beta1", beta1), ("beta2", beta2), ("eps", eps), ("grad_scale", grad_scale)):
                _real(name, x)
            raise
        a.seed = seed & (2**64 - 1)
        if skip is not None:
            _array("skip", skip, torch.int32, 1)
        a.d_skip = None if skip is None else skip.data_ptr()
        pointers = array.array("Q", map(_POINTER, grads))   # held until the call returns
        _check(_lib().hapmoe_adamw(self._table, pointers.buffer_info()[0], n, self._args_at,
                                   _stream_of(torch.cuda.current_device() if n == 0 else index)), "hapmoe_adamw")

    def moments(self, dtype=torch.float32):
        """The values of m and v: two lists of tensors shaped like the parameters.  Moments in 8 bits are decoded
        to fp32 or bf16 (``hapmoe_adamw_moments``); fp32 ones are the state's own tensors."""
        params, m, v = self._kept
        if self.state_bits == 32:
            _need(dtype == torch.float32, "moments in 32 bits are torch.float32")
            return list(m), list(v)
        _need(dtype in (torch.float32, torch.bfloat16), f"dtype: torch.float32 or torch.bfloat16, not {dtype}")
        if params and self._index != torch.cuda.current_device():
            raise ValueError(f"the parameters' device {self._index} is not the current device")
        # one allocation, cut at multiples of 8 elements
        starts, total = [], 0
        for n in self._sizes * 2:
            starts.append(total)
            total += -(-n // 8) * 8
        flat = torch.empty(total, dtype=dtype, device=f"cuda:{self._index or 0}")
        pieces = [flat.as_strided(p.shape, p.stride(), at) for p, at in zip(params + params, starts)]
        out = pieces[:len(params)], pieces[len(params):]
        _check(_lib().hapmoe_adamw_moments(self._table, *(self._pointers(*map(_POINTER, x)) for x in out), len(params),
                                           _TYPES[dtype], _stream_of(torch.cuda.current_device())),
               "hapmoe_adamw_moments")
        return out
