"""The local models' C entries: exported, and refusing bad arguments on the host
before any device work (no GPU needed)."""
import ctypes as C
import os
import re

import pytest

import paper_1905_09598_amd as som
from paper_1905_09598_amd import local

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "som_local.h")


def status(code):
    return som.STATUS[code]


def test_library_exports_every_declared_symbol():
    text = open(HEADER).read()
    names = set(re.findall(r"^\s*(?:som_status|int64_t)\s+(som_\w+)\s*\(", text, flags=re.M))
    assert names == set(local.EXPORTED)
    for name in names:
        assert hasattr(local.lib(), name), name


@pytest.mark.parametrize("struct,binding", [("som_linear_call", local._LinearCall),
                                            ("som_experts_call", local._ExpertsCall),
                                            ("som_route_call", local._RouteCall),
                                            ("som_adamw_tensor", local._AdamwTensor)])
def test_structures_have_the_header_s_fields_in_order(struct, binding):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct %s \{(.*?)\}" % struct, text, flags=re.S).group(1)
    fields = []
    for line in body.split(";"):
        line = line.strip()
        if line:
            kind = re.match(r"(?:const\s+)?(\w+)", line).group(1)
            for part in re.sub(r"^(?:const\s+)?\w+", "", line, count=1).split(","):
                fields.append((part.strip().lstrip("*").strip(),
                               "pointer" if "*" in part else kind))
    size = {"int32_t": 4, "int64_t": 8, "uint64_t": 8, "float": 4, "pointer": 8}
    assert [f[0] for f in binding._fields_] == [f[0] for f in fields]
    assert [C.sizeof(f[1]) for f in binding._fields_] == [size[f[1]] for f in fields]


def _linear(**change):
    values = dict(type=0, n=4, inner=8, outer=8, ldx=8, lddy=8)
    values.update(change)
    return local._LinearCall(**values)


@pytest.mark.parametrize("change,want", [
    (dict(type=3), "SOM_E_ARG"), (dict(activation=-1), "SOM_E_ARG"),
    (dict(activation=4), "SOM_E_ARG"), (dict(n=-1), "SOM_E_ARG"), (dict(inner=0), "SOM_E_ARG"),
    (dict(outer=-2), "SOM_E_ARG"), (dict(ldx=7), "SOM_E_ARG"),
    (dict(inner=4000001, ldx=4000001), "SOM_E_UNSUPPORTED"),
    (dict(outer=4000001), "SOM_E_UNSUPPORTED"), (dict(n=1 << 41), "SOM_E_UNSUPPORTED"),
    ({}, "SOM_E_ARG")])
def test_linear_refuses(change, want):
    L = local.lib()
    call = _linear(**change)          # without arrays: even good sizes are refused
    assert status(L.som_linear(C.byref(call))) == want
    assert status(L.som_linear_backward(C.byref(call))) == want
    need = C.c_uint64()
    assert status(L.som_linear_workspace(C.byref(call), 0, C.byref(need))) == (
        want if change else "SOM_OK")


@pytest.mark.parametrize("change,want", [
    (dict(type=3), "SOM_E_ARG"), (dict(activation=9), "SOM_E_ARG"), (dict(n=-1), "SOM_E_ARG"),
    (dict(k=0), "SOM_E_ARG"), (dict(experts=0), "SOM_E_ARG"), (dict(inner=0), "SOM_E_ARG"),
    (dict(hidden=0), "SOM_E_ARG"), (dict(ldx=3), "SOM_E_ARG"),
    (dict(w2=None, activation=1), "SOM_E_ARG"), (dict(w2=None, b2=1), "SOM_E_ARG"),
    (dict(w2=None, outer=9), "SOM_E_ARG"), (dict(w2=None, z=1, scaled=1), "SOM_E_ARG"),
    (dict(n=1 << 31), "SOM_E_UNSUPPORTED"), (dict(hidden=4000001), "SOM_E_UNSUPPORTED"),
    (dict(experts=1 << 20, hidden=1 << 20), "SOM_E_UNSUPPORTED"), ({}, "SOM_E_ARG")])
def test_experts_refuses(change, want):
    values = dict(n=4, k=2, experts=3, inner=8, hidden=8, outer=8, ldx=8, lddy=8, w2=1)
    values.update(change)
    L, call, need = local.lib(), local._ExpertsCall(**values), C.c_uint64()
    assert status(L.som_experts(C.byref(call))) == want
    assert status(L.som_experts_backward(C.byref(call))) == want
    assert status(L.som_experts_workspace(C.byref(call), 1, C.byref(need))) == (
        want if change else "SOM_OK")


def test_null_calls():
    L = local.lib()
    need = C.c_uint64()
    assert L.som_linear(None) == 1 and L.som_linear_backward(None) == 1
    assert L.som_linear_workspace(None, 0, C.byref(need)) == 1
    assert L.som_linear_workspace(C.byref(_linear()), 0, None) == 1
    assert L.som_route(None) == 1 and L.som_route_backward(None) == 1
    assert L.som_dispatch(None, 4, 2, 8, None, None, None, None, 0, None) == 1
    assert L.som_dispatch_workspace(4, 2, 8, None) == 1
    assert L.som_experts(None) == 1 and L.som_experts_backward(None) == 1
    assert L.som_experts_workspace(None, 0, C.byref(need)) == 1
    assert L.som_adamw_destroy(None) == 0
    assert L.som_adamw_step(None, None, None, 1, 0.1, 0.9, 0.9, 1e-8, 0.0, None) == 1
    assert L.som_adamw_create(None, 1, 32, None, None, None, None, None, None) == 1


@pytest.mark.parametrize("change", [
    dict(type=5), dict(gate=2), dict(n=-1), dict(experts=0), dict(experts=16385, lds=16385),
    dict(k=0), dict(k=9), dict(groups=3), dict(groups=0), dict(top_groups=2), dict(group_best=0),
    dict(group_best=3), dict(scale=float("inf")), dict(lds=7), {}])
def test_route_refuses(change):
    values = dict(n=3, experts=8, k=2, groups=1, top_groups=1, group_best=1, scale=1.0, lds=8)
    values.update(change)
    call = local._RouteCall(**values)
    assert status(local.lib().som_route(C.byref(call))) == "SOM_E_ARG"
    assert status(local.lib().som_route_backward(C.byref(call))) == "SOM_E_ARG"


def test_slots_beyond_32_bits():
    L, need = local.lib(), C.c_uint64()
    assert status(L.som_dispatch_workspace(1 << 30, 4, 8, C.byref(need))) == "SOM_E_UNSUPPORTED"
    assert status(L.som_dispatch_workspace(1 << 20, 4, 0, C.byref(need))) == "SOM_E_ARG"
    call = local._RouteCall(n=1 << 31, experts=8, k=2, groups=1, top_groups=1, group_best=1,
                            scale=1.0, lds=8)
    assert status(L.som_route(C.byref(call))) == "SOM_E_UNSUPPORTED"


def test_workspace_grows_with_what_a_call_needs():
    L, need = local.lib(), C.c_uint64()

    def bytes_of(backward=0, **change):
        call = _linear(**change)
        assert L.som_linear_workspace(C.byref(call), backward, C.byref(need)) == 0
        return need.value

    whole = dict(n=4096, inner=512, outer=4096, ldx=512, type=1)
    assert bytes_of(**whole) == 0                      # aligned, enough tiles
    odd = bytes_of(**dict(whole, inner=511, ldx=511))
    assert odd >= (4096 + 4096) * 512 * 2              # both operands in whole pieces
    assert bytes_of(n=0) == 0


def test_adamw_room_and_refusals():
    L = local.lib()
    table = (local._AdamwTensor * 3)(local._AdamwTensor(None, 1, 0),
                                     local._AdamwTensor(None, 256, 0),
                                     local._AdamwTensor(None, 257, 0))
    assert L.som_adamw_room(table, 3) == 256 + 256 + 512
    assert L.som_adamw_room(None, 3) == -1
    out = C.c_void_p()
    for bits in (16, 0):
        assert L.som_adamw_create(table, 3, bits, 1, 1, None, None, None, C.byref(out)) == 1
    assert L.som_adamw_create(table, 3, 8, 1, 1, None, None, None, C.byref(out)) == 1
    assert L.som_adamw_create(table, 0, 32, 1, 1, None, None, None, C.byref(out)) == 1
    assert L.som_adamw_create(table, 3, 32, None, None, None, None, None, C.byref(out)) == 1
    assert not out.value
    table[1].count = -1
    assert L.som_adamw_room(table, 3) == -1


def test_experts_beyond_what_a_routing_holds():
    L, need = local.lib(), C.c_uint64()
    call = local._ExpertsCall(n=4, k=2, experts=16385, inner=8, hidden=8, outer=8, ldx=8,
                              lddy=8, w2=1)
    assert status(L.som_experts(C.byref(call))) == "SOM_E_UNSUPPORTED"
    assert status(L.som_experts_backward(C.byref(call))) == "SOM_E_UNSUPPORTED"
    call.experts = 16384
    assert status(L.som_experts_workspace(C.byref(call), 1, C.byref(need))) == "SOM_OK"


def test_experts_workspace_counts_each_array_once():
    # local linear maps: dx's parts and dweight alone take the same array
    L, need = local.lib(), C.c_uint64()

    def bytes_of(**wanted):
        call = local._ExpertsCall(n=4096, k=2, experts=16, inner=2048, hidden=512, outer=512,
                                  ldx=2048, lddy=512, **wanted)
        assert status(L.som_experts_workspace(C.byref(call), 1, C.byref(need))) == "SOM_OK"
        return need.value

    assert bytes_of(dx=256) == bytes_of(dweight=256) == bytes_of(dx=256, dweight=256)


def test_experts_copy_their_inner_gradient_once():
    # rows of 2041: both products of the first layer's gradient read dz from a copy in whole
    # pieces, and from the same one
    L, need = local.lib(), C.c_uint64()

    def bytes_of(**wanted):
        call = local._ExpertsCall(type=2, activation=1, n=20000, k=2, experts=16, inner=2000,
                                  hidden=2041, outer=2000, ldx=2000, lddy=2000, w2=256, **wanted)
        assert status(L.som_experts_workspace(C.byref(call), 1, C.byref(need))) == "SOM_OK"
        return need.value

    gate = bytes_of(dweight=256)      # dz itself and what its product takes
    copy = 40000 * 2048 * 2
    assert bytes_of(dx=256) >= gate + copy and bytes_of(dw1=256) >= gate + copy
    assert bytes_of(dx=256) + bytes_of(dw1=256) - bytes_of(dx=256, dw1=256) == gate + copy


def test_the_optimizer_refuses_gradients_of_another_device():
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode

    opt = local.AdamW.__new__(local.AdamW)     # as on the first of two GPUs
    opt.handle, opt.params, opt._counts, opt._device = None, [torch.zeros(4)], [4], 0
    opt._places, opt._codes, opt._ptrs = [opt.params[0].data_ptr()], [0], [0]
    with FakeTensorMode():
        other = torch.empty(4, device="cuda:1")
    with pytest.raises(ValueError, match="gradient 0 must be on"):
        opt.step([other])
    with pytest.raises(TypeError, match="gradient 0"):
        opt.step([torch.zeros(4)])
    with pytest.raises(TypeError, match="gradient 0"):
        opt.step([1.0])


def test_how_products_run_is_told():
    L, tiles = local.lib(), (C.c_int32 * 4)()
    call = _linear(n=16001, inner=2048, outer=2048, ldx=2048, lddy=2048, type=1)
    assert status(L.som_linear_route(C.byref(call), 0, tiles)) == "SOM_OK"
    assert tiles[0] in (64, 128, 256) and tiles[1] == 0
    assert status(L.som_linear_route(C.byref(call), 1, tiles)) == "SOM_OK"
    assert list(tiles[:2]) == [0, 0]                    # no gradient is wanted
    call.dw = 256
    assert status(L.som_linear_route(C.byref(call), 1, tiles)) == "SOM_OK"
    assert tiles[0] == 0 and tiles[1] in (64, 128, 256)
    for n, want in ((0, 0), (3, 16)):
        call.n = n
        assert status(L.som_linear_route(C.byref(call), 0, tiles)) == "SOM_OK"
        assert tiles[0] == want
    assert status(L.som_linear_route(C.byref(call), 0, None)) == "SOM_E_ARG"
    assert status(L.som_linear_route(None, 0, tiles)) == "SOM_E_ARG"
    call = local._ExpertsCall(n=4000, k=2, experts=3, inner=333, hidden=777, outer=333, ldx=333,
                              lddy=333, w2=256, dweight=256)
    assert status(L.som_experts_route(C.byref(call), 0, tiles)) == "SOM_OK"
    assert tiles[0] and tiles[1] and not tiles[2] and not tiles[3]
    assert status(L.som_experts_route(C.byref(call), 1, tiles)) == "SOM_OK"
    assert tiles[0] and not any(tiles[1:])
    assert status(L.som_experts_route(C.byref(call), 1, None)) == "SOM_E_ARG"
    call.k = 0
    assert status(L.som_experts_route(C.byref(call), 1, tiles)) == "SOM_E_ARG"


def test_experts_workspace_before_the_routing_is_there():
    # the routing's arrays are always needed, so that asking without them asks the same
    L, need = local.lib(), C.c_uint64()
    for type_ in (0, 1, 2):
        for n, k, experts, inner, hidden in ((300, 2, 40, 64, 72), (5000, 1, 3, 501, 2001),
                                             (20000, 2, 16, 2000, 2041), (3, 2, 8, 128, 64)):
            call = local._ExpertsCall(type=type_, n=n, k=k, experts=experts, inner=inner,
                                      hidden=hidden, outer=inner, ldx=inner, lddy=inner, w2=256,
                                      b2=256, dx=256, dweight=256, dw1=256, db1=256, dw2=256,
                                      db2=256)
            for backward in (0, 1):
                got = []
                for array in (0, 256):
                    call.offsets = call.order = call.place = array
                    assert status(L.som_experts_workspace(C.byref(call), backward,
                                                          C.byref(need))) == "SOM_OK"
                    got.append(need.value)
                assert got[0] == got[1], (type_, n, k, experts, inner, hidden, backward)
