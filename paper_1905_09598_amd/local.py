"""Local models on a trained map: the gate's product, the routing of documents
to experts, the experts' products, their gradients and the optimizer.

Thin binding of ``include/som_local.h`` (which has every formula).  All
arithmetic runs in the library's HIP kernels; this module marshals arguments,
allocates results and work memory from torch, and orders the calls on torch's
current stream.  Nothing is kept between calls except by ``AdamW``, which holds
the tensors it was made with.

Tensors are fp32, bf16 or fp16, live on one GPU, and have their last dimension
contiguous; matrices of weights are contiguous altogether.  The calls record no
graph: outside ``torch.no_grad()`` they refuse tensors that require a gradient.

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
from typing import Optional

import torch

from . import SomError, _check, lib as _lib

__all__ = [
    "ACTIVATIONS", "GATES", "EXPORTED", "SomError", "Routing", "ExpertsGradient", "AdamW", "linear",
    "linear_backward", "route", "route_backward", "dispatch", "experts", "experts_backward",
    "gate_from_map",
]

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
GATES = {"softmax": 0, "sigmoid": 1}
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
STATE_BLOCK = 256

# Every symbol include/som_local.h declares.
EXPORTED = (
    "som_linear_workspace", "som_linear_route", "som_linear", "som_linear_backward",
    "som_experts_workspace", "som_experts_route", "som_experts", "som_experts_backward",
    "som_route", "som_route_backward",
    "som_dispatch_workspace", "som_dispatch", "som_adamw_room", "som_adamw_create",
    "som_adamw_destroy", "som_adamw_step",
)


class _LinearCall(C.Structure):
    """``som_linear_call`` of include/som_local.h."""

    _fields_ = [("type", C.c_int32), ("activation", C.c_int32), ("n", C.c_int64),
                ("inner", C.c_int32), ("outer", C.c_int32), ("x", C.c_void_p),
                ("ldx", C.c_int64), ("w", C.c_void_p), ("bias", C.c_void_p),
                ("residual", C.c_void_p), ("ldr", C.c_int64), ("y", C.c_void_p),
                ("z", C.c_void_p), ("dy", C.c_void_p), ("lddy", C.c_int64),
                ("dx", C.c_void_p), ("dw", C.c_void_p), ("dbias", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64),
                ("stream", C.c_void_p)]


class _ExpertsCall(C.Structure):
    """``som_experts_call`` of include/som_local.h."""

    _fields_ = [("type", C.c_int32), ("activation", C.c_int32), ("n", C.c_int64),
                ("k", C.c_int32), ("experts", C.c_int32), ("inner", C.c_int32),
                ("hidden", C.c_int32), ("outer", C.c_int32), ("x", C.c_void_p),
                ("ldx", C.c_int64), ("w1", C.c_void_p), ("b1", C.c_void_p),
                ("w2", C.c_void_p), ("b2", C.c_void_p), ("residual", C.c_void_p),
                ("ldr", C.c_int64), ("weight", C.c_void_p), ("offsets", C.c_void_p),
                ("order", C.c_void_p), ("place", C.c_void_p), ("y", C.c_void_p),
                ("z", C.c_void_p), ("scaled", C.c_void_p), ("dy", C.c_void_p),
                ("lddy", C.c_int64), ("dx", C.c_void_p), ("dweight", C.c_void_p),
                ("dw1", C.c_void_p), ("db1", C.c_void_p), ("dw2", C.c_void_p),
                ("db2", C.c_void_p), ("workspace", C.c_void_p),
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
                ("offsets", C.c_void_p), ("order", C.c_void_p), ("place", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64),
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
        "som_linear_route": [C.POINTER(_LinearCall), i32, C.POINTER(i32)],
        "som_linear": [C.POINTER(_LinearCall)],
        "som_linear_backward": [C.POINTER(_LinearCall)],
        "som_experts_workspace": [C.POINTER(_ExpertsCall), i32, C.POINTER(u64)],
        "som_experts_route": [C.POINTER(_ExpertsCall), i32, C.POINTER(i32)],
        "som_experts": [C.POINTER(_ExpertsCall)],
        "som_experts_backward": [C.POINTER(_ExpertsCall)],
        "som_route": [C.POINTER(_RouteCall)],
        "som_route_backward": [C.POINTER(_RouteCall)],
        "som_dispatch_workspace": [i64, i32, i32, C.POINTER(u64)],
        "som_dispatch": [vp, i64, i32, i32, vp, vp, vp, vp, u64, vp],
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
def _no_graph(t, what: str) -> None:
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient, which these calls do not record: call "
                         "them under torch.no_grad() and form gradients by the _backward calls")


def _type(t, what: str) -> int:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what} must be a torch tensor")
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what} must be float32, bfloat16 or float16, got {t.dtype}")
    if not t.is_cuda:
        raise TypeError(f"{what} must live on the GPU")
    _no_graph(t, what)
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


def _stream(t) -> int:
    """The current stream of t's device, which has to be the current one."""
    index = t.device.index
    if index != torch._C._cuda_getDevice():
        raise ValueError(f"tensors must be on the current device, not {t.device}")
    return torch._C._cuda_getCurrentRawStream(index)


def _run(name: str, call, backward: bool, x) -> None:
    """A call that takes work memory, on x's device."""
    L = lib()
    need = C.c_uint64()
    call.stream = _stream(x)
    at = C.byref(call)
    run = f"som_{name}_backward" if backward else f"som_{name}"
    _check(getattr(L, f"som_{name}_workspace")(at, backward, C.byref(need)), run)
    if need.value:
        work = torch.empty(need.value, dtype=torch.uint8, device=x.device)
        call.workspace = work.data_ptr()
        call.workspace_bytes = need.value
    _check(getattr(L, run)(at), run)


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
    _run("linear", call, False, x)
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
    _run("linear", call, True, x)
    return dx, dw, dbias


# ------------------------------------------------------------------ routing
class Routing:
    """Which experts the documents go to: index (n, k) int32, -1 for none;
    weight (n, k) fp32, or None for 1; the slots i k + j in the order of their
    experts (``order``), each slot's row in it (``place``, -1 for none) and each
    expert's first row (``offsets``, experts + 1 entries), all int32; and how the
    choice was made (gate, renormalise, scale), for its gradient."""

    __slots__ = ("index", "weight", "experts", "gate", "renormalise", "scale", "_ints")

    def __init__(self, index, weight, experts: int, ints, gate: str = "",
                 renormalise: bool = True, scale: float = 1.0):
        self.index, self.weight, self.experts, self._ints = index, weight, experts, ints
        self.gate, self.renormalise, self.scale = gate, renormalise, scale

    # one allocation: order, place, offsets
    @property
    def order(self):
        return self._ints[:self.index.numel()]

    @property
    def place(self):
        slots = self.index.numel()
        return self._ints[slots:2 * slots]

    @property
    def offsets(self):
        return self._ints[2 * self.index.numel():]

    @property
    def load(self):
        """Documents of each expert, int32."""
        return self.offsets[1:] - self.offsets[:-1]

    def _pointers(self):
        """Addresses of offsets, order and place."""
        at, slots = self._ints.data_ptr(), self.index.numel()
        return at + 8 * slots, at, at + 4 * slots


def _order_of(index, weight, experts: int, device, **how):
    """A Routing with room for its order, and the work memory the sort takes."""
    n, k = index.shape
    need = C.c_uint64()
    _check(lib().som_dispatch_workspace(n, k, experts, C.byref(need)), "som_dispatch")
    ints = torch.empty(2 * n * k + experts + 1, dtype=torch.int32, device=device)
    work = torch.empty(need.value, dtype=torch.uint8, device=device) if need.value else None
    return Routing(index, weight, experts, ints, **how), work, need.value


def dispatch(index, weight, experts: int) -> Routing:
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
        _no_graph(weight, "weight")
        _shaped(weight, index, (n, k), "weight")
    r, work, need = _order_of(index, weight, experts, index.device)
    _check(lib().som_dispatch(index.data_ptr(), n, k, experts, *r._pointers(), _ptr(work), need,
                              _stream(index)), "som_dispatch")
    return r


def _route_call(scores, k: int):
    code = _type(scores, "scores")
    _rows(scores, "scores")
    n, experts = scores.shape
    return _RouteCall(code, 0, n, experts, k, 1, 1, 1, 1, 1.0, scores.data_ptr(), _ld(scores))


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
        _no_graph(bias, "bias")
        _shaped(bias, scores, (experts,), "bias")
        call.bias = bias.data_ptr()
    if k < 1:
        raise ValueError("k must be at least 1")
    device = scores.device
    index = torch.empty((n, k), dtype=torch.int32, device=device)
    weight = torch.empty((n, k), dtype=torch.float32, device=device)
    r, work, need = _order_of(index, weight, experts, device, gate=gate,
                              renormalise=renormalise, scale=scale)
    call.index, call.weight = index.data_ptr(), weight.data_ptr()
    call.offsets, call.order, call.place = r._pointers()
    call.workspace, call.workspace_bytes = _ptr(work), need
    call.stream = _stream(scores)
    _check(lib().som_route(C.byref(call)), "som_route")
    return r


def route_backward(dweight, scores, routing: Routing):
    """Gradient of the scores from that of ``routing.weight`` (fp32 or 16 bits)."""
    if routing.gate not in GATES:
        raise ValueError("the routing was not made by route()")
    n, k = routing.index.shape
    call = _route_call(scores, k)
    _shaped(scores, routing.index, (n, routing.experts), "scores", packed=False)
    call.gate = GATES[routing.gate]
    call.renormalise, call.scale = int(routing.renormalise), routing.scale
    call.index, call.weight = routing.index.data_ptr(), routing.weight.data_ptr()
    call.dweight_type = _type(dweight, "dweight")
    _shaped(dweight, scores, (n, k), "dweight")
    call.dweight = dweight.data_ptr()
    dscores = torch.empty((n, routing.experts), dtype=scores.dtype, device=scores.device)
    call.dscores = dscores.data_ptr()
    call.stream = _stream(scores)
    _check(lib().som_route_backward(C.byref(call)), "som_route_backward")
    return dscores


# ------------------------------------------------------------------ experts
@dataclasses.dataclass
class ExpertsGradient:
    """Gradients of ``experts``; those of absent arguments are None."""

    x: torch.Tensor
    weight: torch.Tensor
    w1: torch.Tensor
    b1: Optional[torch.Tensor]
    w2: Optional[torch.Tensor]
    b2: Optional[torch.Tensor]


def _experts_call(x, routing: Routing, w1, b1, w2, b2, activation: str):
    code = _type(x, "x")
    _rows(x, "x")
    n, k = routing.index.shape
    e = routing.experts
    if x.shape[0] != n:
        raise ValueError(f"x must have {n} rows")
    if w1.dim() != 3 or not w1.numel():
        raise ValueError("w1 must be (experts, hidden, inner)")
    hidden, inner = w1.shape[1], x.shape[1]
    _like(w1, x, (e, hidden, inner), "w1")
    if b1 is not None:
        _like(b1, x, (e, hidden), "b1")
    outer, act = hidden, 0
    if w2 is not None:
        act = _of(ACTIVATIONS, activation, "activation")
        if w2.dim() != 3 or not w2.numel():
            raise ValueError("w2 must be (experts, outer, hidden)")
        outer = w2.shape[1]
        _like(w2, x, (e, outer, hidden), "w2")
        if b2 is not None:
            _like(b2, x, (e, outer), "b2")
    elif b2 is not None:
        raise ValueError("b2 without w2")
    if routing.index.device != x.device:
        raise ValueError(f"the routing must be on {x.device}")
    return _ExpertsCall(code, act, n, k, e, inner, hidden, outer, x.data_ptr(), _ld(x),
                        w1.data_ptr(), _ptr(b1), _ptr(w2), _ptr(b2), None, 0,
                        _ptr(routing.weight), *routing._pointers())


def experts(x, routing: Routing, w1, b1=None, w2=None, b2=None, activation: str = "gelu",
            residual=None, keep: bool = False):
    """The routed experts' answers to the documents x (n, inner), joined:

        residual + sum over j of weight[:, j] (w2_e act(w1_e x + b1_e) + b2_e)

    with e = index[:, j], w1 (experts, hidden, inner), w2 (experts, outer,
    hidden); without w2 the local linear maps w1_e x + b1_e.  With ``keep``
    returns (y, kept), kept being what ``experts_backward`` needs."""
    call = _experts_call(x, routing, w1, b1, w2, b2, activation)
    n = x.shape[0]
    if residual is not None:
        _like(residual, x, (n, call.outer), "residual", packed=False)
        call.residual, call.ldr = residual.data_ptr(), _ld(residual)
    y = torch.empty((n, call.outer), dtype=x.dtype, device=x.device)
    call.y = y.data_ptr()
    kept = None
    if keep and w2 is not None:
        kept = torch.empty((2, routing.index.numel(), call.hidden), dtype=x.dtype,
                           device=x.device)
        call.z, call.scaled = kept[0].data_ptr(), kept[1].data_ptr()
    _run("experts", call, False, x)
    return (y, kept) if keep else y


def experts_backward(dy, x, routing: Routing, w1, b1, w2, b2, kept,
                     activation: str = "gelu") -> ExpertsGradient:
    """Gradients of ``experts`` from that of its result; the residual's is dy."""
    call = _experts_call(x, routing, w1, b1, w2, b2, activation)
    n, k = routing.index.shape
    _like(dy, x, (n, call.outer), "dy", packed=False)
    call.dy, call.lddy = dy.data_ptr(), _ld(dy)
    if w2 is not None:
        if kept is None:
            raise ValueError("the gradient needs what experts(keep=True) kept")
        _like(kept, x, (2, n * k, call.hidden), "kept")
        call.z, call.scaled = kept[0].data_ptr(), kept[1].data_ptr()

    def like(t):
        return None if t is None else torch.empty_like(t)

    d = ExpertsGradient(torch.empty((n, x.shape[1]), dtype=x.dtype, device=x.device),
                        torch.empty((n, k), dtype=x.dtype, device=x.device),
                        like(w1), like(b1), like(w2), like(b2))
    call.dx, call.dweight = d.x.data_ptr(), d.weight.data_ptr()
    call.dw1, call.db1, call.dw2, call.db2 = _ptr(d.w1), _ptr(d.b1), _ptr(d.w2), _ptr(d.b2)
    _run("experts", call, True, x)
    return d


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
    ``state`` takes such arrays over (a checkpoint's, with ``step`` steps done).
    The parameters have to stay where they are: ``step`` refuses one that has moved
    or changed its size."""

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
            with torch.no_grad():        # a module's parameters are welcome
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
                self.master[at:at + p.numel()].copy_(p.detach().reshape(-1))
                at += -(-p.numel() // STATE_BLOCK) * STATE_BLOCK
        handle = C.c_void_p()
        with torch.cuda.device(device):
            _check(L.som_adamw_create(table, len(self.params), bits, _ptr(self.mean),
                                      _ptr(self.square), _ptr(self.mean_scale),
                                      _ptr(self.square_scale), _ptr(self.master),
                                      C.byref(handle)), "som_adamw_create")
        self.handle = handle.value
        self._counts = [p.numel() for p in self.params]
        self._device = device.index
        self._places = [p.data_ptr() for p in self.params]
        self._ptrs = (C.c_void_p * len(self.params))()
        self._codes = (C.c_int32 * len(self.params))()

    def step(self, grads, lr: Optional[float] = None) -> None:
        """One step with the gradients (contiguous, each of its parameter's
        size, of any of the three types) and, if given, another learning rate."""
        if len(grads) != len(self.params):
            raise ValueError(f"{len(self.params)} gradients are wanted, got {len(grads)}")
        for i, (g, count) in enumerate(zip(grads, self._counts)):
            code = _TYPES.get(getattr(g, "dtype", None))
            if code is None or g.get_device() != self._device:
                _type(g, f"gradient {i}")
                raise ValueError(f"gradient {i} must be on {self.params[0].device}")
            self._codes[i] = code
            if g.numel() != count or not g.is_contiguous():
                raise ValueError(f"gradient {i} must be contiguous with {count} elements")
            self._ptrs[i] = g.data_ptr() or None
        if ([p.data_ptr() for p in self.params] != self._places
                or [p.numel() for p in self.params] != self._counts):
            raise ValueError("a parameter is no longer in the memory the optimizer was made with")
        _check(lib().som_adamw_step(self.handle, self._ptrs, self._codes, self.steps + 1,
                                    self.lr if lr is None else lr, *self.betas, self.eps,
                                    self.weight_decay, _stream(self.params[0])), "som_adamw_step")
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
