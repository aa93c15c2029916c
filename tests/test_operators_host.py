"""The operators' C calls refuse malformed arguments before any device work (no GPU needed: the
device addresses are never followed)."""
import ctypes as C
import math

import pytest

from paper_2609_39350_amd import binding, operators as ops

INVAL, WORKSPACE = -1, -3
NO_DEVICE = (-4, -5)   # past the checks: no usable device here
P = 1 << 20            # an aligned address

if __import__("torch").cuda.is_available():
    pytest.skip("addresses here are made up", allow_module_level=True)


def changed(base, **by_index):
    args = list(base)
    for k, v in by_index.items():
        args[int(k[1:])] = v
    return args


def test_struct_sizes():
    assert C.sizeof(ops._Tensor) == 64 and C.sizeof(ops._Args) == 80


def test_route():
    L = ops._lib()
    need = C.c_int64(-1)
    assert L.hapmoe_route_ws_bytes(4096, 64, 8, C.byref(need)) == 0 and need.value > 0
    assert L.hapmoe_route_ws_bytes(4, 64, 8, C.byref(need)) == 0 and need.value == 0
    for bad in ((-1, 8, 2), (4, 0, 1), (4, 1025, 2), (4, 8, 9), (4, 8, 0), (4, 64, 33), (2**31, 8, 1), (2**30, 8, 2)):
        assert L.hapmoe_route_ws_bytes(*bad, C.byref(need)) == INVAL, bad
    assert L.hapmoe_route_ws_bytes(4, 8, 2, None) == INVAL
    good = [P, ops.F32, 64, 4096, 64, 8, None, 1, P, P, P, P, P, P, P, 1 << 30, None]
    assert L.hapmoe_route(*good) in NO_DEVICE
    for i, v in ((0, None), (0, P + 2), (1, 3), (2, 63), (3, -1), (4, 2000), (5, 65), (8, None), (9, None), (10, None),
                 (11, None), (12, None), (13, None), (14, None)):
        assert L.hapmoe_route(*changed(good, **{f"a{i}": v})) == INVAL, (i, v)
    assert L.hapmoe_route(*changed(good, a15=16)) == WORKSPACE
    good = [P, ops.BF16, 64, 4096, 64, 8, None, 0, P, P, P, P, None]
    assert L.hapmoe_route_backward(*good) in NO_DEVICE
    for i, v in ((0, None), (0, P + 1), (1, -1), (2, 1), (5, 0), (8, None), (9, None), (10, None), (11, None)):
        assert L.hapmoe_route_backward(*changed(good, **{f"a{i}": v})) == INVAL, (i, v)


def test_combine():
    L = ops._lib()
    good = [P, ops.F16, 64, 8, 8, 128, P, None, P, None]
    assert L.hapmoe_combine(*good) in NO_DEVICE
    for i, v in ((0, None), (0, P + 1), (1, 9), (2, -1), (2, 2**31), (3, -1), (4, 0), (4, 33), (5, 0), (5, 2**25),
                 (6, None), (8, None)):
        assert L.hapmoe_combine(*changed(good, **{f"a{i}": v})) == INVAL, (i, v)
    good = [P, P, ops.F32, 8, 8, 128, P, P, P, P, P, None]
    assert L.hapmoe_combine_backward(*good) in NO_DEVICE
    for i in (0, 1, 6, 7, 8, 9, 10):
        assert L.hapmoe_combine_backward(*changed(good, **{f"a{i}": None})) == INVAL, i


def test_expert_products():
    L = ops._lib()
    good = [P, 512, 128, P, ops.BF16, 1024, 8, 256, 128, P, P, 2, P, None]
    assert L.hapmoe_expert_matmul(*good) in NO_DEVICE
    for i, v in ((0, None), (0, P + 1), (1, -1), (2, 127), (3, None), (3, P + 1), (4, ops.F32), (5, -1), (5, 2**31),
                 (6, 0), (6, 1025), (7, 0), (8, 0), (8, 2**31), (9, None), (11, 0), (12, None), (12, P + 1)):
        assert L.hapmoe_expert_matmul(*changed(good, **{f"a{i}": v})) == INVAL, (i, v)
    assert L.hapmoe_expert_matmul(*changed(good, a10=None)) == INVAL   # without slot x needs a row each
    assert L.hapmoe_expert_matmul(*changed(good, a10=None, a1=1024, a11=0)) in NO_DEVICE
    good = [P, 256, P, ops.F16, 1024, 8, 256, 128, P, P, None]
    assert L.hapmoe_expert_matmul_grad_x(*good) in NO_DEVICE
    for i, v in ((0, None), (1, 255), (2, None), (3, 0), (4, -1), (8, None), (9, None)):
        assert L.hapmoe_expert_matmul_grad_x(*changed(good, **{f"a{i}": v})) == INVAL, (i, v)
    good = [P, 256, P, 512, 128, ops.F16, 1024, 8, 256, 128, P, P, 2, ops.F32, P, None]
    assert L.hapmoe_expert_matmul_grad_w(*good) in NO_DEVICE
    for i, v in ((0, None), (2, None), (4, 100), (13, ops.BF16), (13, 7), (14, None), (14, P + 2)):
        assert L.hapmoe_expert_matmul_grad_w(*changed(good, **{f"a{i}": v})) == INVAL, (i, v)


def adamw(tensor=(), grad=P, **args):
    t = (ops._Tensor * 2)()
    for x in t:
        x.param = x.m = x.v = P
        x.n = 100
    for k, v in dict(tensor).items():
        setattr(t[1], k, v)
    a = ops._Args(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, grad_scale=1.0, step=1, state_bits=32)
    for k, v in args.items():
        setattr(a, k, v)
    return ops._lib().hapmoe_adamw(t, (C.c_void_p * 2)(P, grad), 2, C.byref(a), None)


def test_adamw():
    assert adamw() in NO_DEVICE
    assert adamw({"n": 0, "param": None, "copy": P}) in NO_DEVICE
    for bad in ({"n": -1}, {"param": None}, {"m": None}, {"v": None}, {"param": P + 2}, {"m": P + 1},
                {"copy": P}, {"weight_decay": -0.1}, {"weight_decay": math.inf}, {"n": 2**60}):
        assert adamw(bad) == INVAL, bad
    for bad in ({"lr": -1.0}, {"lr": math.nan}, {"beta1": 1.0}, {"beta2": -0.1}, {"eps": -1.0}, {"step": 0},
                {"grad_scale": math.inf}, {"grad_type": 5}, {"state_bits": 16}, {"state_bits": 8}, {"d_skip": P + 1}):
        assert adamw(**bad) == INVAL, bad
    assert adamw(grad=None) == INVAL and adamw(grad=P + 1) == INVAL
    f = ops._lib().hapmoe_adamw
    assert f(None, None, 1, None, None) == INVAL and f(None, None, -1, C.byref(ops._Args()), None) == INVAL


def test_adamw_moments():
    f = ops._lib().hapmoe_adamw_moments

    def call(tensor=(), m=P, v=P, out_type=ops.BF16, n=2):
        t = (ops._Tensor * 2)()
        for x in t:
            x.m = x.v = x.m_exp = x.v_exp = P
            x.n = 100
        for k, value in dict(tensor).items():
            setattr(t[1], k, value)
        return f(t, (C.c_void_p * 2)(P, m), (C.c_void_p * 2)(P, v), n, out_type, None)

    assert call() in NO_DEVICE and call(m=None, v=None, tensor={"n": 0}) in NO_DEVICE
    for bad in ({"m": None}, {"v": None}, {"m": P + 1}, {"out_type": ops.F16}, {"n": -1}, {"tensor": {"n": -1}},
                {"tensor": {"m": None}}, {"tensor": {"v_exp": None}}, {"tensor": {"n": 2**60}}):
        assert call(**bad) == INVAL, bad
    assert f(None, None, None, 1, ops.F32, None) == INVAL


def test_wrong_tensors_raise_value_error():
    import torch
    x = torch.zeros(4, 8)
    for f, args in ((ops.route, (x, 2)), (ops.combine, (x, x.int())), (ops.expert_matmul, (x, x, x)),
                    (ops.AdamW, ([x], [x], [x]))):
        with pytest.raises(ValueError):
            f(*args)
    with pytest.raises(ValueError):
        ops.Routing(4, 8, 9, "cpu")
    assert binding.lib() is ops._lib()
