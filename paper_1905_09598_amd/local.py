"""Local models on a trained map: the gate's product, the routing of documents
to experts, the experts' products, their gradients and the optimizer.

Thin binding of ``include/som_local.h`` (which has every formula).  All
arithmetic runs in the library's HIP kernels; this module marshals arguments,
allocates results and work memory from torch, and orders the calls on torch's
current stream.  Nothing is kept between calls except by ``AdamW``, which holds
the tensors it was made with.

Tensors are fp32, bf16 or fp16, live on one GPU, and have their last dimension
contiguous; matrices of weights are contiguous altogether.

    scores = local.linear(x, w, bias)                  # the gate
    r = local.route(scores, k=2)                       # index, weight, order
    y, kept = local.experts(x, r, w1, b1, w2, b2, "gelu", keep=True)
    d = local.experts_backward(dy, x, r, w1, b1, w2, b2, kept, "gelu")
    ds = local.route_backward(d.weight, scores, r)
    dx, dw, dbias = local.linear_backward(ds, x, w)
    optimizer.step([dw, dbias, d.w1, d.b1, d.w2, d.b2])

``gate_from_map`` gives the gate whose scores are a trained map's.
"""
from __future__ import annotations

import ctypes as C
import dataclasses
from typing import Any, Optional

import torch

from . import SomError, _check, _current_stream, lib as _lib

__all__ = [
    "ACTIVATIONS", "GATES", "EXPORTED", "SomError", "Routing", "ExpertsGradient", "AdamW", "linear",
    "linear_backward", "route", "route_backward", "dispatch", "experts", "experts_backward",
    "combine", "combine_backward", "gate_from_map",
]

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
GATES = {"softmax": 0, "sigmoid": 1}
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
STATE_BLOCK = 256

# Every symbol include/som_local.h declares.
EXPORTED = (
    "som_linear_workspace", "som_linear", "som_linear_backward", "som_route",
    "som_route_backward", "som_dispatch_workspace", "som_dispatch", "som_combine",
    "som_combine_backward", "som_adamw_room", "som_adamw_create", "som_adamw_destroy",
    "som_adamw_step",
)


class _LinearCall(C.Structure):
    """``som_linear_call`` of include/som_local.h."""

    _fields_ = [("type", C.c_int32), ("activation", C.c_int32), ("n", C.c_int64),
                ("inner", C.c_int32), ("outer", C.c_int32), ("x", C.c_void_p),
                ("ldx", C.c_int64), ("w", C.c_void_p), ("bias", C.c_void_p),
                ("residual", C.c_void_p), ("ldr", C.c_int64), ("y", C.c_void_p),
                ("z", C.c_void_p), ("experts", C.c_int32), ("k", C.c_int32),
                ("gather", C.c_int32), ("offsets", C.c_void_p), ("order", C.c_void_p),
                ("dy", C.c_void_p), ("lddy", C.c_int64), ("dx", C.c_void_p),
                ("dw", C.c_void_p), ("dbias", C.c_void_p), ("slope_z", C.c_void_p),
                ("slope_activation", C.c_int32), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_uint64), ("stream", C.c_void_p)]


class _RouteCall(C.Structure):
    """``som_route_call`` of include/som_local.h."""

    _fields_ = [("type", C.c_int32), ("gate", C.c_int32), ("n", C.c_int64),
                ("experts", C.c_int32), ("k", C.c_int32), ("groups", C.c_int32),
                ("top_groups", C.c_int32), ("group_best", C.c_int32),
                ("renormalise", C.c_int32), ("scale", C.c_float), ("scores", C.c_void_p),
                ("lds", C.c_int64), ("bias", C.c_void_p), ("index", C.c_void_p),
                ("weight", C.c_void_p), ("dweight", C.c_void_p),
                ("dweight_type", C.c_int32), ("dscores", C.c_void_p),
                ("stream", C.c_void_p)]


class _AdamwTensor(C.Structure):
    """``som_adamw_tensor`` of include/som_local.h."""

    _fields_ = [("param", C.c_void_p), ("count", C.c_int64), ("type", C.c_int32)]


_bound = None


def lib():
    """The loaded libsom with this module's calls declared."""
    global _bound
    if _bound is not None:
        return _bound
    L = _lib()
    vp, i32, i64, u64, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_double
    sig = {
        "som_linear_workspace": [C.POINTER(_LinearCall), i32, C.POINTER(u64)],
        "som_linear": [C.POINTER(_LinearCall)],
        "som_linear_backward": [C.POINTER(_LinearCall)],
        "som_route": [C.POINTER(_RouteCall)],
        "som_route_backward": [C.POINTER(_RouteCall)],
        "som_dispatch_workspace": [i64, i32, i32, C.POINTER(u64)],
        "som_dispatch": [vp, i64, i32, i32, vp, vp, vp, vp, u64, vp],
        "som_combine": [i32, i64, i32, i32, vp, vp, vp, vp, i64, vp, vp],
        "som_combine_backward": [i32, i64, i32, i32, vp, i64, vp, vp, vp, vp, vp, vp],
        "som_adamw_create": [C.POINTER(_AdamwTensor), i32, i32, vp, vp, vp, vp, vp,
                             C.POINTER(vp)],
        "som_adamw_destroy": [vp],
        "som_adamw_step": [vp, vp, vp, i64, f64, f64, f64, f64, f64, vp],
    }
    for name, args in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = C.c_int
    L.som_adamw_room.argtypes = [C.POINTER(_AdamwTensor), i32]
    L.som_adamw_room.restype = i64
    _bound = L
    return L


# ---------------------------------------------------------------- arguments
def _type(t, what: str) -> int:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what} must be a torch tensor")
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what} must be float32, bfloat16 or float16, got {t.dtype}")
    if not t.is_cuda:
        raise TypeError(f"{what} must live on the GPU")
    return code


def _like(t, x, shape, what: str, packed: bool = True):
    """t has x's type and the given shape; packed: without gaps."""
    _type(t, what)
    if t.dtype != x.dtype:
        raise TypeError(f"{what} must be {x.dtype}, got {t.dtype}")
    _shaped(t, x, shape, what, packed)


def _shaped(t, x, shape, what: str, packed: bool = True):
    if t.device != x.device:
        raise ValueError(f"{what} must be on {x.device}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must be {tuple(shape)}, got {tuple(t.shape)}")
    if packed:
        if not t.is_contiguous():
            raise ValueError(f"{what} must be contiguous")
    else:
        _rows(t, what)


def _rows(t, what: str):
    """Row stride of a matrix whose rows are contiguous and do not overlap."""
    if t.dim() != 2:
        raise ValueError(f"{what} must have two dimensions")
    if t.shape[1] > 1 and t.stride(1) != 1 or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise ValueError(f"{what} must have contiguous rows")


def _ld(t) -> int:
    return t.stride(0) if t.shape[0] > 1 else max(1, t.shape[1])


def _of(table, name: str, what: str) -> int:
    try:
        return table[name]
    except KeyError:
        raise ValueError(f"{what} must be one of {', '.join(table)}, got {name!r}") from None


def _ptr(t):
    return None if t is None else t.data_ptr()


def _work(nbytes: int, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _run_linear(call: _LinearCall, backward: bool, device) -> None:
    L = lib()
    need = C.c_uint64()
    name = "som_linear_backward" if backward else "som_linear"
    _check(L.som_linear_workspace(C.byref(call), int(backward), C.byref(need)), name)
    work = _work(need.value, device)
    call.workspace = _ptr(work)
    call.workspace_bytes = need.value
    call.stream = _current_stream()
    _check(getattr(L, name)(C.byref(call)), name)


# ------------------------------------------------------------------ product
def _dense_call(x, w, activation: str):
    code = _type(x, "x")
    _rows(x, "x")
    if w.dim() != 2:
        raise ValueError("w must have two dimensions")
    _like(w, x, (w.shape[0], x.shape[1]), "w")
    if not w.numel():
        raise ValueError("w must not be empty")
    return _LinearCall(type=code, activation=_of(ACTIVATIONS, activation, "activation"),
                       n=x.shape[0], inner=x.shape[1], outer=w.shape[0], x=_ptr(x), ldx=_ld(x),
                       w=_ptr(w))


def linear(x, w, bias=None, activation: str = "none", residual=None, keep: bool = False):
    """y = act(x wᵀ + bias) + residual for x (n, inner) and w (outer, inner).

    With ``keep`` returns (y, z): z = x wᵀ + bias as the gradient needs it, or
    None where the activation needs none."""
    call = _dense_call(x, w, activation)
    n, outer = x.shape[0], w.shape[0]
    if bias is not None:
        _like(bias, x, (outer,), "bias")
        call.bias = _ptr(bias)
    if residual is not None:
        _like(residual, x, (n, outer), "residual", packed=False)
        call.residual, call.ldr = _ptr(residual), _ld(residual)
    y = torch.empty((n, outer), dtype=x.dtype, device=x.device)
    z = torch.empty_like(y) if keep and activation != "none" else None
    call.y, call.z = _ptr(y), _ptr(z)
    _run_linear(call, False, x.device)
    return (y, z) if keep else y


def linear_backward(dy, x, w, z=None, activation: str = "none", bias: bool = True):
    """(dx, dw, dbias) of ``linear`` from the gradient dy of its result; dbias is
    None without ``bias``.  The residual's gradient is dy."""
    call = _dense_call(x, w, activation)
    n, outer = x.shape[0], w.shape[0]
    _like(dy, x, (n, outer), "dy", packed=False)
    if activation != "none":
        if z is None:
            raise ValueError("the gradient of an activation needs z (linear with keep=True)")
        _like(z, x, (n, outer), "z")
        call.z = _ptr(z)
    call.dy, call.lddy = _ptr(dy), _ld(dy)
    dx = torch.empty((n, x.shape[1]), dtype=x.dtype, device=x.device)
    dw = torch.empty_like(w)
    dbias = torch.empty(outer, dtype=x.dtype, device=x.device) if bias else None
    call.dx, call.dw, call.dbias = _ptr(dx), _ptr(dw), _ptr(dbias)
    _run_linear(call, True, x.device)
    return dx, dw, dbias


# ------------------------------------------------------------------ routing
@dataclasses.dataclass
class Routing:
    """Which experts the documents go to: index (n, k) int32, -1 for none;
    weight (n, k) fp32; the slots i k + j in the order of their experts (order),
    each slot's row in it (place, -1 for none) and each expert's first row
    (offsets, experts + 1 entries); and how the choice was made."""

    index: torch.Tensor
    weight: torch.Tensor
    experts: int
    offsets: torch.Tensor
    order: torch.Tensor
    place: torch.Tensor
    gate: str = ""
    renormalise: bool = True
    scale: float = 1.0

    @property
    def load(self):
        """Documents of each expert, int32."""
        return self.offsets[1:] - self.offsets[:-1]


def dispatch(index, weight, experts: int, **how) -> Routing:
    """The Routing of a given assignment: index (n, k) int32 with entries in [0,
    experts) or -1, weight (n, k) fp32 (None: 1).  For example the best units of
    ``Map.bmu``."""
    if not isinstance(index, torch.Tensor) or index.dtype != torch.int32 or not index.is_cuda:
        raise TypeError("index must be an int32 tensor on the GPU")
    if index.dim() != 2 or not index.is_contiguous() or index.shape[1] < 1:
        raise ValueError("index must be (n, k) and contiguous")
    n, k = index.shape
    if weight is not None:
        if not isinstance(weight, torch.Tensor) or weight.dtype != torch.float32:
            raise TypeError("weight must be float32")
        _shaped(weight, index, (n, k), "weight")
    L, need = lib(), C.c_uint64()
    _check(L.som_dispatch_workspace(n, k, experts, C.byref(need)), "som_dispatch")
    ints = torch.empty(2 * n * k + experts + 1, dtype=torch.int32, device=index.device)
    order, place, offsets = ints[:n * k], ints[n * k:2 * n * k], ints[2 * n * k:]
    work = _work(need.value, index.device)
    _check(L.som_dispatch(_ptr(index), n, k, experts, _ptr(offsets), _ptr(order), _ptr(place),
                          _ptr(work), need.value, _current_stream()), "som_dispatch")
    return Routing(index, weight, experts, offsets, order, place, **how)


def _route_call(scores, k: int):
    code = _type(scores, "scores")
    _rows(scores, "scores")
    return _RouteCall(type=code, n=scores.shape[0], experts=scores.shape[1], k=k,
                      scores=_ptr(scores), lds=_ld(scores), groups=1, top_groups=1,
                      group_best=1, stream=_current_stream())


def route(scores, k: int, bias=None, gate: str = "softmax", groups: int = 1,
          top_groups: int = 1, group_best: int = 1, renormalise: bool = True,
          scale: float = 1.0) -> Routing:
    """The k experts of each document by its scores (n, experts), with their
    weights, and the slots in the order of their experts.

    bias (experts,) fp32 acts on the choice alone; with ``groups`` only the
    experts of the ``top_groups`` groups with the largest values (the sum of a
    group's ``group_best`` largest) are chosen from.  Scores of -infinity close
    an expert to a document."""
    call = _route_call(scores, k)
    n, experts = scores.shape
    call.gate = _of(GATES, gate, "gate")
    call.groups, call.top_groups, call.group_best = groups, top_groups, group_best
    call.renormalise, call.scale = int(renormalise), scale
    if bias is not None:
        if not isinstance(bias, torch.Tensor) or bias.dtype != torch.float32:
            raise TypeError("bias must be float32")
        _shaped(bias, scores, (experts,), "bias")
        call.bias = _ptr(bias)
    if k < 1:
        raise ValueError("k must be at least 1")
    index = torch.empty((n, k), dtype=torch.int32, device=scores.device)
    weight = torch.empty((n, k), dtype=torch.float32, device=scores.device)
    call.index, call.weight = _ptr(index), _ptr(weight)
    _check(lib().som_route(C.byref(call)), "som_route")
    return dispatch(index, weight, experts, gate=gate, renormalise=renormalise, scale=scale)


def route_backward(dweight, scores, routing: Routing):
    """Gradient of the scores from that of ``routing.weight`` (fp32 or 16 bits)."""
    if routing.gate not in GATES:
        raise ValueError("the routing was not made by route()")
    n, k = routing.index.shape
    call = _route_call(scores, k)
    _shaped(scores, routing.index, (n, routing.experts), "scores", packed=False)
    call.gate = GATES[routing.gate]
    call.renormalise, call.scale = int(routing.renormalise), routing.scale
    call.index, call.weight = _ptr(routing.index), _ptr(routing.weight)
    call.dweight_type = _type(dweight, "dweight")
    _shaped(dweight, scores, (n, k), "dweight")
    call.dweight = _ptr(dweight)
    dscores = torch.empty((n, routing.experts), dtype=scores.dtype, device=scores.device)
    call.dscores = _ptr(dscores)
    _check(lib().som_route_backward(C.byref(call)), "som_route_backward")
    return dscores


# ------------------------------------------------------------------ experts
def _expert_call(x, routing: Routing, w, activation: str, gather: bool):
    code = _type(x, "x")
    _rows(x, "x")
    n, k = routing.index.shape
    if w.dim() != 3:
        raise ValueError("the experts' matrices must be (experts, outer, inner)")
    _like(w, x, (routing.experts, w.shape[1], x.shape[1]), "the experts' matrices")
    if not w.numel():
        raise ValueError("the experts' matrices must not be empty")
    rows = n if gather else n * k
    if x.shape[0] != rows:
        raise ValueError(f"x must have {rows} rows")
    if routing.index.device != x.device:
        raise ValueError(f"the routing must be on {x.device}")
    return _LinearCall(type=code, activation=_of(ACTIVATIONS, activation, "activation"), n=n,
                       inner=x.shape[1], outer=w.shape[1], x=_ptr(x), ldx=_ld(x), w=_ptr(w),
                       experts=routing.experts, k=k, gather=int(gather),
                       offsets=_ptr(routing.offsets), order=_ptr(routing.order))


def _expert_linear(x, routing, w, bias, activation, gather, keep):
    call = _expert_call(x, routing, w, activation, gather)
    rows, outer = routing.index.numel(), w.shape[1]
    if bias is not None:
        _like(bias, x, (routing.experts, outer), "the experts' bias")
        call.bias = _ptr(bias)
    y = torch.empty((rows, outer), dtype=x.dtype, device=x.device)
    z = torch.empty_like(y) if keep and activation != "none" else None
    call.y, call.z = _ptr(y), _ptr(z)
    _run_linear(call, False, x.device)
    return y, z


def _expert_linear_backward(dy, x, routing, w, has_bias, gather, slope_z=None,
                            slope_activation="none"):
    """(dx, dw, dbias) from the gradient dy of the product itself."""
    call = _expert_call(x, routing, w, "none", gather)
    rows = routing.index.numel()
    call.dy, call.lddy = _ptr(dy), _ld(dy)
    dx = torch.empty((rows, x.shape[1]), dtype=x.dtype, device=x.device)
    dw = torch.empty_like(w)
    dbias = torch.empty(w.shape[:2], dtype=x.dtype, device=x.device) if has_bias else None
    call.dx, call.dw, call.dbias = _ptr(dx), _ptr(dw), _ptr(dbias)
    if slope_z is not None:
        call.slope_z, call.slope_activation = _ptr(slope_z), ACTIVATIONS[slope_activation]
    _run_linear(call, True, x.device)
    return dx, dw, dbias


def combine(y, routing: Routing, residual=None, weighted: bool = True):
    """residual + the sum of each document's rows of y (one per slot, in the
    experts' order), times ``routing.weight`` if ``weighted``."""
    n, k = routing.index.shape
    code = _type(y, "y")
    _like(y, y, (n * k, y.shape[-1]), "y")
    if residual is not None:
        _like(residual, y, (n, y.shape[1]), "residual", packed=False)
    out = torch.empty((n, y.shape[1]), dtype=y.dtype, device=y.device)
    _check(lib().som_combine(code, n, k, y.shape[1], _ptr(y),
                             _ptr(routing.weight) if weighted else None, _ptr(routing.place),
                             _ptr(residual), _ld(residual) if residual is not None else 0,
                             _ptr(out), _current_stream()), "som_combine")
    return out


def combine_backward(dout, y, routing: Routing):
    """(dy, dweight) of ``combine`` from the gradient of its result."""
    n, k = routing.index.shape
    code = _type(y, "y")
    _like(y, y, (n * k, y.shape[-1]), "y")
    _like(dout, y, (n, y.shape[1]), "dout", packed=False)
    dy = torch.empty_like(y)
    dweight = torch.empty((n, k), dtype=y.dtype, device=y.device)
    _check(lib().som_combine_backward(code, n, k, y.shape[1], _ptr(dout), _ld(dout), _ptr(y),
                                      _ptr(routing.weight), _ptr(routing.place), _ptr(dy),
                                      _ptr(dweight), _current_stream()),
           "som_combine_backward")
    return dy, dweight


@dataclasses.dataclass
class ExpertsGradient:
    """Gradients of ``experts``; those of absent arguments are None."""

    x: torch.Tensor
    weight: torch.Tensor
    w1: torch.Tensor
    b1: Optional[torch.Tensor]
    w2: Optional[torch.Tensor]
    b2: Optional[torch.Tensor]


def experts(x, routing: Routing, w1, b1=None, w2=None, b2=None, activation: str = "gelu",
            residual=None, keep: bool = False):
    """The routed experts' answers to the documents x (n, inner), joined:

        residual + sum over j of weight[:, j] (w2_e act(w1_e x + b1_e) + b2_e)

    with e = index[:, j], w1 (experts, hidden, inner), w2 (experts, outer,
    hidden); without w2 the local linear maps w1_e x + b1_e.  With ``keep``
    returns (y, kept), kept being what ``experts_backward`` needs."""
    if w2 is None:
        if b2 is not None:
            raise ValueError("b2 without w2")
        answer, _ = _expert_linear(x, routing, w1, b1, "none", True, False)
        kept = (None, None, answer)
    else:
        h, z = _expert_linear(x, routing, w1, b1, activation, True, keep)
        answer, _ = _expert_linear(h, routing, w2, b2, "none", False, False)
        kept = (h, z, answer)
    y = combine(answer, routing, residual)
    return (y, kept) if keep else y


def experts_backward(dy, x, routing: Routing, w1, b1, w2, b2, kept: Any,
                     activation: str = "gelu") -> ExpertsGradient:
    """Gradients of ``experts`` from that of its result; the residual's is dy."""
    h, z, answer = kept
    danswer, dweight = combine_backward(dy, answer, routing)
    dw2 = db2 = None
    if w2 is not None:
        danswer, dw2, db2 = _expert_linear_backward(danswer, h, routing, w2, b2 is not None,
                                                    False, z, activation)
    dslots, dw1, db1 = _expert_linear_backward(danswer, x, routing, w1, b1 is not None, True)
    dx = combine(dslots, routing, weighted=False)
    return ExpertsGradient(dx, dweight, dw1, db1, dw2, db2)


def gate_from_map(weights, tau: float, dtype=torch.float32):
    """(w, bias) of the gate whose scores for a document x are, up to a constant
    per document, -|x - w_u|²/(2 tau) for the map's prototypes w_u (``Map.weights``):
    the larger, the nearer, so that the best score is the best-matching unit's."""
    if not tau > 0:
        raise ValueError("tau must be positive")
    w = (weights / tau).to(dtype).contiguous()
    return w, (-0.5 / tau * weights.square().sum(1)).to(dtype)


# ---------------------------------------------------------------- optimizer
class AdamW:
    """AdamW over a list of tensors (updated in place), states in 32 or 8 bits.

    The states of all tensors lie in one array each, every tensor from the next
    multiple of 256 elements on: ``mean`` and ``square`` (fp32, or
    float8_e4m3fn of m and of sqrt(v) with ``mean_scale`` and ``square_scale``,
    one fp32 per 256 elements), and with ``master`` the parameters in fp32.
    ``state`` takes such arrays over (a checkpoint's, with ``step`` steps done)."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 0.01, bits: int = 32, master: bool = False,
                 step: int = 0, state: Optional[dict] = None):
        self.handle = None
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        table = (_AdamwTensor * len(self.params))()
        device = self.params[0].device
        for i, p in enumerate(self.params):
            table[i] = _AdamwTensor(_ptr(p), p.numel(), _type(p, f"parameter {i}"))
            if p.device != device or not p.is_contiguous():
                raise ValueError(f"parameter {i} must be contiguous and on {device}")
        self.lr, self.betas, self.eps, self.weight_decay = lr, tuple(betas), eps, weight_decay
        self.bits, self.steps = bits, step
        L = lib()
        room = L.som_adamw_room(table, len(self.params))
        held = torch.float8_e4m3fn if bits == 8 else torch.float32
        names = {"mean": (room, held), "square": (room, held)}
        if bits == 8:
            names["mean_scale"] = names["square_scale"] = (room // STATE_BLOCK, torch.float32)
        if master or (state or {}).get("master") is not None:
            names["master"] = (room, torch.float32)
        self.master = self.mean_scale = self.square_scale = None
        for name, (count, dtype) in names.items():
            if state is None:
                t = torch.zeros(count * dtype.itemsize, dtype=torch.uint8,
                                device=device).view(dtype)
            else:
                t = state[name]
                if t.dtype != dtype or tuple(t.shape) != (count,) or t.device != device \
                        or not t.is_contiguous():
                    raise ValueError(f"state {name} must be {count} contiguous {dtype}")
            setattr(self, name, t)
        if state is None and self.master is not None:
            at = 0
            for p in self.params:
                self.master[at:at + p.numel()].copy_(p.reshape(-1))
                at += -(-p.numel() // STATE_BLOCK) * STATE_BLOCK
        handle = C.c_void_p()
        with torch.cuda.device(device):
            _check(L.som_adamw_create(table, len(self.params), bits, _ptr(self.mean),
                                      _ptr(self.square), _ptr(self.mean_scale),
                                      _ptr(self.square_scale), _ptr(self.master),
                                      C.byref(handle)), "som_adamw_create")
        self.handle = handle.value
        self._counts = [p.numel() for p in self.params]
        self._ptrs = (C.c_void_p * len(self.params))()
        self._codes = (C.c_int32 * len(self.params))()

    def step(self, grads, lr: Optional[float] = None) -> None:
        """One step with the gradients (contiguous, each of its parameter's
        size, of any of the three types) and, if given, another learning rate."""
        if len(grads) != len(self.params):
            raise ValueError(f"{len(self.params)} gradients are wanted, got {len(grads)}")
        for i, (g, count) in enumerate(zip(grads, self._counts)):
            self._codes[i] = _type(g, f"gradient {i}")
            if g.numel() != count or not g.is_contiguous():
                raise ValueError(f"gradient {i} must be contiguous with {count} elements")
            self._ptrs[i] = g.data_ptr() or None
        _check(lib().som_adamw_step(self.handle, self._ptrs, self._codes, self.steps + 1,
                                    self.lr if lr is None else lr, *self.betas, self.eps,
                                    self.weight_decay, _current_stream()), "som_adamw_step")
        self.steps += 1

    def close(self) -> None:
        """Release the table on the device (its memory may still be in use by
        enqueued steps: the release waits for them)."""
        if getattr(self, "handle", None):
            handle, self.handle = self.handle, None
            _check(lib().som_adamw_destroy(handle), "som_adamw_destroy")

    def __del__(self):  # pragma: no cover - best effort
        try:
            self.close()
        except Exception:
            pass
