"""The C calls of the operators around a layer refuse malformed arguments before any device work (no GPU needed: the
device addresses are never followed)."""
import ctypes as C
import math

import pytest

from paper_2609_39350_amd import operators as ops
from .test_operators_host import INVAL, NO_DEVICE, P, WORKSPACE, changed

NOT_THERE = 1 << 30


def refuses(f, good, wrong):
    assert f(*good) in NO_DEVICE
    for i, values in wrong.items():
        for v in values:
            assert f(*changed(good, **{f"a{i}": v})) == INVAL, (i, v)


def test_route_balanced():
    f = ops._lib().hapmoe_route_balanced
    good = [P, ops.F32, 64, 4096, 64, 8, P, 1, 8, 4, 2, None, 1, 2.5, P, P, P, P, P, P, P, NOT_THERE, None]
    refuses(f, good, {0: (None, P + 2), 1: (3, -1), 2: (63, 2**50), 3: (-1, 2**31), 4: (0, 2000), 5: (0, 65, 33), 6: (P + 2,),
                      7: (-1, 2), 8: (0, 65, 7, -8), 9: (0, 9), 10: (0, 3), 13: (0.0, -1.0, math.nan, math.inf),
                      14: (None,), 15: (None,), 16: (None,), 17: (None,), 18: (None,), 19: (None,), 20: (None, P + 2)})
    assert f(*changed(good, a6=None, a8=1, a9=1, a10=1)) in NO_DEVICE
    assert f(*changed(good, a21=16)) == WORKSPACE
    # no tokens: only the counts and offsets are there
    assert f(*changed(good, a0=None, a3=0, a14=None, a15=None, a18=None, a19=None, a20=None)) in NO_DEVICE


def test_route_balanced_backward():
    f = ops._lib().hapmoe_route_balanced_backward
    good = [P, ops.BF16, 64, 4096, 64, 8, 1, None, 0, 1.0, P, P, P, P, None]
    refuses(f, good, {0: (None, P + 1), 1: (-1, 3), 2: (1,), 3: (-1,), 5: (0, 65), 6: (-1, 2), 9: (0.0, math.nan),
                      10: (None,), 11: (None,), 12: (None,), 13: (None, P + 1)})


def test_layer_norm():
    L = ops._lib()
    good = [P, ops.BF16, 128, 64, 128, P, P, ops.F32, 1e-5, P, P, P, None]
    refuses(L.hapmoe_layer_norm, good, {
        0: (None, P + 1), 1: (-1, 3), 2: (127, 2**50), 3: (-1, 2**31), 4: (0, 2**25), 5: (None, P + 2), 6: (P + 2,),
        7: (ops.F16, 5, -1), 8: (-1.0, math.nan, math.inf), 9: (P + 2,), 10: (None, P + 2), 11: (None, P + 1)})
    for none in ({"a6": None}, {"a9": None}, {"a7": ops.BF16}, {"a8": 0.0}):
        assert L.hapmoe_layer_norm(*changed(good, **none)) in NO_DEVICE
    need = C.c_int64(-1)
    assert L.hapmoe_layer_norm_ws_bytes(0, 128, C.byref(need)) == 0 and need.value == 0
    assert L.hapmoe_layer_norm_ws_bytes(64, 128, C.byref(need)) == 0 and need.value > 0
    for long in (20000, 2**24):   # rows that no workgroup holds: the workspace stays small
        assert L.hapmoe_layer_norm_ws_bytes(4096, long, C.byref(need)) == 0 and 0 < need.value <= max(2**23, 8 * long)
    for bad in ((-1, 128), (64, 0), (64, 2**25), (2**31, 8)):
        assert L.hapmoe_layer_norm_ws_bytes(*bad, C.byref(need)) == INVAL
    assert L.hapmoe_layer_norm_ws_bytes(64, 128, None) == INVAL
    good = [P, 128, P, ops.F16, 128, 64, 128, P, ops.F16, P, P, P, 128, P, P, P, P, NOT_THERE, None]
    f = L.hapmoe_layer_norm_backward
    refuses(f, good, {
        0: (None, P + 1), 1: (127,), 2: (None, P + 1), 3: (-1, 3), 4: (100,), 5: (-1, 2**31), 6: (0, 2**25),
        7: (None, P + 1), 8: (ops.BF16,), 9: (P + 1,), 10: (None, P + 2), 11: (P + 1,), 12: (1,), 13: (None, P + 1),
        14: (None, P + 2), 15: (P + 2,), 16: (None, P + 8)})
    for none in ({"a9": None}, {"a11": None, "a12": 0}, {"a15": None}):
        assert f(*changed(good, **none)) in NO_DEVICE
    assert f(*changed(good, a17=16)) == WORKSPACE


def test_embed():
    L = ops._lib()
    good = [P, 32, 64, P, ops.BF16, 128, 1000, 128, 2.0, P, None]
    refuses(L.hapmoe_embed, good, {
        0: (None, P + 2), 1: (16, 0, -32), 2: (-1, 2**31), 3: (None, P + 1), 4: (-1, 3), 5: (127,), 6: (0, -1, 2**31),
        7: (0, 2**25), 8: (math.nan, math.inf), 9: (None, P + 1)})
    assert L.hapmoe_embed(*changed(good, a0=P + 4, a1=64)) == INVAL   # 64-bit tokens lie on multiples of 8
    need = C.c_int64(-1)
    assert L.hapmoe_embed_ws_bytes(0, 128, C.byref(need)) == 0 and need.value == 0
    assert L.hapmoe_embed_ws_bytes(64, 128, C.byref(need)) == 0 and need.value > 0
    for bad in ((-1, 128), (64, 0), (64, 2**25), (2**31, 8)):
        assert L.hapmoe_embed_ws_bytes(*bad, C.byref(need)) == INVAL
    good = [P, ops.F32, 128, 64, 128, P, 64, 1000, 1.0, 0, P, P, NOT_THERE, None]
    f = L.hapmoe_embed_backward
    refuses(f, good, {
        0: (None, P + 2), 1: (-1, 3), 2: (127,), 3: (-1, 2**31), 4: (0, 2**25), 5: (None, P + 4), 6: (8,),
        7: (0, 2**31, 2**31 - 1), 8: (math.nan,), 10: (None, P + 2), 11: (None, P + 8)})
    assert f(*changed(good, a12=16)) == WORKSPACE


def test_dropout():
    good = [P, ops.F16, 128, 64, 128, P, 128, 0.1, 1, 2, P, P, None]
    refuses(ops._lib().hapmoe_dropout, good, {
        0: (None, P + 1), 1: (-1, 3), 2: (127, 2**50), 3: (-1, 2**31), 4: (0, 2**25), 5: (P + 1,), 6: (127,),
        7: (-0.1, 1.1, math.nan), 10: (P + 4,), 11: (None, P + 1)})
    assert ops._lib().hapmoe_dropout(*changed(good, a5=None, a6=0, a10=None)) in NO_DEVICE


def test_wrong_tensors_raise_value_error():
    import torch
    x, v, i = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4, dtype=torch.int32)
    for f, args in ((ops.route_balanced, (x, 2)), (ops.layer_norm, (x, v)), (ops.layer_norm_backward, (x, x, v, v, v)),
                    (ops.embed, (i, x)), (ops.embed_backward, (x, i, 9)), (ops.dropout, (x, 0.1, 1)),
                    (ops.dropout_backward, (x, 0.1, 1))):
        with pytest.raises(ValueError):
            f(*args)
