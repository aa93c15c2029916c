"""What an operator cannot take raises ValueError, whatever is wrong with it, and launches nothing."""
import math

import numpy as np
import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import binding, operators as ops   # noqa: E402
from .test_gpu_operators import normal, offsets   # noqa: E402

pytestmark = pytest.mark.gpu


def refused(f, *a, **k):
    with pytest.raises(ValueError):
        f(*a, **k)


@pytest.mark.parametrize("keep", [[True] * 5, np.ones(5, dtype=bool), 1, "all"])
def test_keep_that_is_no_tensor(keep):
    logits = normal(1, 5, 8)
    refused(ops.route, logits, 2, keep=keep)
    r = ops.route(logits, 2)
    refused(ops.route_backward, logits, r, torch.zeros(5, 2, device="cuda"), keep=keep)


@pytest.mark.parametrize("wrong", [None, 3, [1.0] * 8, np.zeros((8, 16), dtype=np.float32)])
def test_operands_that_are_no_tensors(wrong):
    x, w, off = normal(1, 8, 16, dtype=torch.bfloat16), normal(2, 2, 4, 16, dtype=torch.bfloat16), offsets([3, 5])
    d_y = normal(3, 8, 4, dtype=torch.bfloat16)
    y, place, weight = normal(4, 8, 16), torch.arange(8, dtype=torch.int32, device="cuda").view(4, 2), normal(5, 4, 2)
    slot = place.reshape(-1)
    for f, args in ((ops.route, (normal(6, 4, 8), 2)), (ops.combine, (y, place)),
                    (ops.combine_backward, (y[:4], y, slot, place, weight)), (ops.expert_matmul, (x, w, off)),
                    (ops.expert_matmul_grad_x, (d_y, w, off)), (ops.expert_matmul_grad_w, (d_y, x, off))):
        f(*args)
        for i, a in enumerate(args):
            if isinstance(a, torch.Tensor):
                refused(f, *args[:i], wrong, *args[i + 1:])
    if wrong is not None:   # None is none
        refused(ops.combine, y, place, wrong)
        refused(ops.expert_matmul, x, w, off, slot=wrong)
    p, m, v = (torch.zeros(300, device="cuda") for _ in range(3))
    for i in range(3):
        refused(ops.AdamW, *([wrong] if i == j else [t] for j, t in enumerate((p, m, v))))
    refused(ops.AdamW, [p], [m], [v], copies=[wrong])
    codes = [torch.zeros(300, dtype=torch.uint8, device="cuda") for _ in range(2)]
    exps = torch.zeros(2, dtype=torch.int8, device="cuda")
    refused(ops.AdamW, [p], codes[:1], codes[1:], m_exp=[wrong], v_exp=[exps])
    opt = ops.AdamW([p, p.clone()], [m, m.clone()], [v, v.clone()])
    for grads in ([wrong, p], [p, wrong], [wrong, wrong]):
        refused(opt.step, grads, lr=1e-3, step=1)
    if wrong is not None:
        refused(opt.step, [p, p], lr=1e-3, step=1, skip=wrong)
    assert all((t == 0).all() for t in (p, m, v))


def test_numbers():
    logits = normal(1, 5, 8)
    for k in (0, -1, 9, 33, 2**31, 2**32 + 2, -2**32 + 2):
        refused(ops.route, logits, k)
    x, w, off = normal(1, 8, 16, dtype=torch.bfloat16), normal(2, 2, 4, 16, dtype=torch.bfloat16), offsets([3, 5])
    d_y, slot = normal(3, 8, 4, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.int32, device="cuda")
    for k in (0, -1, 2**31, 2**32 + 1, -2**32 + 1):
        refused(ops.expert_matmul, x, w, off, slot=slot, top_k=k)
        refused(ops.expert_matmul_grad_w, d_y, x, off, slot=slot, top_k=k)
    p, m, v = (torch.zeros(300, device="cuda") for _ in range(3))
    opt = ops.AdamW([p], [m], [v])
    g = [torch.ones(300, device="cuda")]
    for bad in ({"lr": -1.0, "step": 1}, {"lr": math.inf, "step": 1}, {"lr": math.nan, "step": 1}, {"lr": 1e-3, "step": 0},
                {"lr": 1e-3, "step": -3}, {"lr": 1e-3, "step": 2**63}, {"lr": 1e-3, "step": 2**64 + 1},
                {"lr": 1e-3, "step": -2**64 + 1},
                {"lr": 1e-3, "step": 1, "beta1": 1.0}, {"lr": 1e-3, "step": 1, "beta2": -0.5},
                {"lr": 1e-3, "step": 1, "eps": math.nan}, {"lr": 1e-3, "step": 1, "grad_scale": math.inf}):
        refused(opt.step, g, **bad)
    assert all((t == 0).all() for t in (p, m, v))
    with pytest.raises(binding.HapmoeError):   # of the C call, as the planner's are
        opt.step(g, lr=-1.0, step=1)
