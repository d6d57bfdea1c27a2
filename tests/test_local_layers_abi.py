"""The C entries of layer norm, the gated layer, distillation and the products in 8
bits: refusing bad arguments on the host before any device work (no GPU needed)."""
import ctypes as C
import math
import os
import re

import pytest

import paper_1905_09598_amd as som
from paper_1905_09598_amd import local

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "som_local.h")


def status(code):
    return som.STATUS[code]


@pytest.mark.parametrize("struct,binding", [
    ("som_norm_call", local._NormCall), ("som_gated_call", local._GatedCall),
    ("som_distill_call", local._DistillCall), ("som_blocks_call", local._BlocksCall),
    ("som_linear8_call", local._Linear8Call)])
def test_structures_have_the_header_s_fields_in_order(struct, binding):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct %s \{(.*?)\}" % struct, text, flags=re.S).group(1)
    fields = []
    for line in body.split(";"):
        line = line.strip()
        if line:
            kind = re.match(r"(?:const\s+)?(\w+)", line).group(1)
            for part in re.sub(r"^(?:const\s+)?\w+", "", line, count=1).split(","):
                fields.append((part.strip().lstrip("*").strip(), "pointer" if "*" in part else kind))
    size = {"int32_t": 4, "int64_t": 8, "uint64_t": 8, "float": 4, "pointer": 8}
    assert [f[0] for f in binding._fields_] == [f[0] for f in fields]
    assert [C.sizeof(f[1]) for f in binding._fields_] == [size[f[1]] for f in fields]


@pytest.mark.parametrize("change,want", [
    (dict(type=3), "SOM_E_ARG"), (dict(n=-1), "SOM_E_ARG"), (dict(width=0), "SOM_E_ARG"),
    (dict(ldx=7), "SOM_E_ARG"), (dict(eps=-1e-5), "SOM_E_ARG"), (dict(eps=math.nan), "SOM_E_ARG"),
    (dict(eps=math.inf), "SOM_E_ARG"), (dict(width=4000001, ldx=4000001), "SOM_E_UNSUPPORTED"),
    (dict(n=1 << 41), "SOM_E_UNSUPPORTED"), ({}, "SOM_E_ARG")])
def test_norm_refuses(change, want):
    values = dict(type=0, width=8, n=4, ldx=8, lddy=8, eps=1e-5)
    values.update(change)
    L, call, need = local.lib(), local._NormCall(**values), C.c_uint64()
    assert status(L.som_norm(C.byref(call))) == want
    assert status(L.som_norm_backward(C.byref(call))) == want
    for backward in (0, 1):
        assert status(L.som_norm_workspace(C.byref(call), backward, C.byref(need))) == (
            want if change else "SOM_OK")


def test_norm_workspace():
    L, need = local.lib(), C.c_uint64()
    call = local._NormCall(type=1, width=2048, n=100, ldx=2048, eps=1e-5)
    for backward, dweight, some in ((0, 1, False), (1, 0, False), (1, 1, True)):
        call.dweight = dweight
        assert status(L.som_norm_workspace(C.byref(call), backward, C.byref(need))) == "SOM_OK"
        assert (need.value > 0) == some and need.value % 256 == 0


@pytest.mark.parametrize("change,want", [
    (dict(type=-1), "SOM_E_ARG"), (dict(activation=4), "SOM_E_ARG"), (dict(n=-1), "SOM_E_ARG"),
    (dict(inner=0), "SOM_E_ARG"), (dict(hidden=0), "SOM_E_ARG"), (dict(ldx=7), "SOM_E_ARG"),
    (dict(inner=4000001, ldx=4000001), "SOM_E_UNSUPPORTED"),
    (dict(hidden=2000001), "SOM_E_UNSUPPORTED"), (dict(n=1 << 41), "SOM_E_UNSUPPORTED"),
    ({}, "SOM_E_ARG")])
def test_gated_refuses(change, want):
    values = dict(type=1, activation=3, n=4, inner=8, hidden=8, ldx=8, lddy=8)
    values.update(change)
    L, call, need = local.lib(), local._GatedCall(**values), C.c_uint64()
    tiles = (C.c_int32 * 2)()
    assert status(L.som_gated(C.byref(call))) == want
    assert status(L.som_gated_backward(C.byref(call))) == want
    for backward in (0, 1):
        asked = want if change else "SOM_OK"
        assert status(L.som_gated_workspace(C.byref(call), backward, C.byref(need))) == asked
        assert status(L.som_gated_route(C.byref(call), backward, tiles)) == asked


@pytest.mark.parametrize("change,want", [
    (dict(type=3), "SOM_E_ARG"), (dict(teacher_type=7), "SOM_E_ARG"), (dict(n=-1), "SOM_E_ARG"),
    (dict(classes=0), "SOM_E_ARG"), (dict(lds=9), "SOM_E_ARG"), (dict(k=-1), "SOM_E_ARG"),
    (dict(k=65), "SOM_E_ARG"), (dict(k=0), "SOM_E_ARG"), (dict(k=0, mix=0.0, index=8), "SOM_E_ARG"),
    (dict(temperature=0.0), "SOM_E_ARG"), (dict(temperature=math.nan), "SOM_E_ARG"),
    (dict(temperature=2.0 ** 21), "SOM_E_ARG"), (dict(mix=-0.1), "SOM_E_ARG"),
    (dict(mix=1.1), "SOM_E_ARG"), (dict(mix=math.nan), "SOM_E_ARG"), (dict(mix=0.5), "SOM_E_ARG"),
    (dict(scale=math.nan), "SOM_E_ARG"),
    (dict(classes=(1 << 20) + 1, lds=1 << 21), "SOM_E_UNSUPPORTED"),
    (dict(n=1 << 41), "SOM_E_UNSUPPORTED"), ({}, "SOM_E_ARG")])
def test_distill_refuses(change, want):
    values = dict(type=0, n=4, classes=10, k=2, lds=10, temperature=1.0, mix=1.0, scale=1.0)
    values.update(change)
    call = local._DistillCall(**values)
    assert status(local.lib().som_distill(C.byref(call))) == want


@pytest.mark.parametrize("change,want", [
    (dict(type=3), "SOM_E_ARG"), (dict(n=-1), "SOM_E_ARG"), (dict(width=0), "SOM_E_ARG"),
    (dict(ldx=7), "SOM_E_ARG"), (dict(width=4000001, ldx=4000001), "SOM_E_UNSUPPORTED"),
    (dict(n=1 << 41), "SOM_E_UNSUPPORTED"), ({}, "SOM_E_ARG")])
def test_to_blocks_refuses(change, want):
    values = dict(type=0, width=8, n=4, ldx=8)
    values.update(change)
    call = local._BlocksCall(**values)
    assert status(local.lib().som_to_blocks(C.byref(call))) == want


@pytest.mark.parametrize("change,want", [
    (dict(type=0), "SOM_E_ARG"), (dict(type=3), "SOM_E_ARG"), (dict(activation=5), "SOM_E_ARG"),
    (dict(n=-1), "SOM_E_ARG"), (dict(inner=0), "SOM_E_ARG"), (dict(outer=0), "SOM_E_ARG"),
    (dict(ldx=7), "SOM_E_ARG"), (dict(inner=4000001, ldx=4000001), "SOM_E_UNSUPPORTED"),
    (dict(outer=4000001), "SOM_E_UNSUPPORTED"), (dict(n=1 << 41), "SOM_E_UNSUPPORTED"),
    ({}, "SOM_E_ARG")])
def test_linear8_refuses(change, want):
    values = dict(type=1, n=4, inner=8, outer=8, ldx=8)
    values.update(change)
    L, call, need = local.lib(), local._Linear8Call(**values), C.c_uint64()
    assert status(L.som_linear8(C.byref(call))) == want
    assert status(L.som_linear8_workspace(C.byref(call), C.byref(need))) == (
        want if change else "SOM_OK")


@pytest.mark.parametrize("n,inner,outer", [(0, 40, 24), (1, 8, 8), (16, 2048, 10000), (17, 1231, 8),
                                           (637, 128, 8192), (1601, 11700, 2707)])
def test_linear8_route_agrees_with_its_work_memory(n, inner, outer):
    """In 8 bits already, a product needs memory for the parts of its contraction alone."""
    L, need, route = local.lib(), C.c_uint64(), (C.c_int32 * 2)(-1, -1)
    call = local._Linear8Call(type=1, n=n, inner=inner, outer=outer, ldx=inner, x_codes=256)
    assert status(L.som_linear8_route(C.byref(call), route)) == "SOM_OK"
    assert status(L.som_linear8_workspace(C.byref(call), C.byref(need))) == "SOM_OK"
    tile, parts = route
    assert (tile, parts) == (0, 0) if n == 0 else tile in (16, 64, 128, 256) and parts >= 1
    assert (tile == 16) == (0 < n <= 16)
    wide = -(-outer // tile) * tile if n else 0
    assert need.value == (-(-parts * n * wide * 4 // 256) * 256 if parts > 1 else 0)
    assert L.som_linear8_route(C.byref(call), None) == 1 and L.som_linear8_route(None, route) == 1
    call.type = 0
    assert status(L.som_linear8_route(C.byref(call), route)) == "SOM_E_ARG"


def test_null_calls():
    L, need = local.lib(), C.c_uint64()
    for name in ("som_norm", "som_norm_backward", "som_gated", "som_gated_backward", "som_distill",
                 "som_to_blocks", "som_linear8"):
        assert getattr(L, name)(None) == 1, name
    assert L.som_norm_workspace(None, 0, C.byref(need)) == 1
    assert L.som_gated_workspace(None, 0, C.byref(need)) == 1
    assert L.som_linear8_workspace(None, C.byref(need)) == 1
    call = local._GatedCall(type=1, n=4, inner=8, hidden=8, ldx=8)
    assert L.som_gated_workspace(C.byref(call), 0, None) == 1
    assert L.som_gated_route(C.byref(call), 0, None) == 1


def test_no_rows_need_no_arrays():
    """Calls without rows pass without a device where they have nothing to write."""
    L = local.lib()
    call = local._DistillCall(type=0, n=0, classes=10, k=2, lds=10, temperature=1.0, mix=0.5, scale=1.0)
    assert status(L.som_distill(C.byref(call))) == "SOM_OK"
    blocks = local._BlocksCall(type=0, width=8, n=0, ldx=8)
    assert status(L.som_to_blocks(C.byref(blocks))) == "SOM_OK"
