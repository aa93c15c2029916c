"""A number of the wrong kind raises ValueError, as one of the wrong size does, and launches nothing; whole numbers and
reals of other libraries are numbers."""
import numpy as np
import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_operator_refusals import refused   # noqa: E402
from .test_gpu_operators import normal, offsets   # noqa: E402

pytestmark = pytest.mark.gpu
NO_REAL = ["0.5", b"1", [0.5], (1.0,), 1j, 10**400, torch.zeros(2)]
NO_WHOLE = ["1", b"1", 1.0, 2.5, [1], 1j, np.float32(1.0), torch.zeros(2, dtype=torch.int64), torch.tensor(1.0)]


def test_around_the_layer():
    logits, x, w, token = normal(1, 6, 8), normal(2, 6, 16), normal(3, 16), torch.arange(6, device="cuda")
    r, d_weight = ops.route_balanced(logits, 2), normal(4, 6, 2)
    for bad in NO_REAL + [None]:
        refused(ops.route_balanced, logits, 2, scale=bad)
        refused(ops.route_balanced_backward, logits, r, d_weight, scale=bad)
        refused(ops.layer_norm, x, w, eps=bad)
        refused(ops.embed, token, x, scale=bad)
        refused(ops.embed_backward, x, token, 9, scale=bad)
        refused(ops.dropout, x, bad, 1)
        refused(ops.dropout_backward, x, bad, 1)
    for bad in NO_WHOLE + [None]:
        refused(ops.route_balanced, logits, bad)
        refused(ops.route_balanced, logits, bad, out=r)
        for name in ("groups", "top_groups", "group_best"):
            if not (bad is None and name == "top_groups"):   # None: all of them
                refused(ops.route_balanced, logits, 2, **{name: bad})
        refused(ops.embed_backward, x, token, bad)
        for name in ("seed", "offset"):
            for f in (ops.dropout, ops.dropout_backward):
                refused(f, x, 0.1, **{"seed": 1, name: bad})


def test_in_the_layer():
    logits, x = normal(1, 6, 8), normal(2, 6, 16, dtype=torch.bfloat16)
    w, off, slot = normal(3, 2, 4, 16, dtype=torch.bfloat16), offsets([2, 4]), torch.arange(6, dtype=torch.int32, device="cuda")
    d_y, r = normal(4, 6, 4, dtype=torch.bfloat16), ops.route(logits, 2)
    for bad in NO_WHOLE + [None]:
        refused(ops.route, logits, bad)
        refused(ops.route, logits, bad, out=r)
        for sizes in ((bad, 8, 2), (6, bad, 2), (6, 8, bad)):
            refused(ops.Routing, *sizes)
        for of in (slot, None):
            refused(ops.expert_matmul, x, w, off, slot=of, top_k=bad)
            refused(ops.expert_matmul_grad_w, d_y, x, off, slot=of, top_k=bad)
    p, m, v = (torch.zeros(300, device="cuda") for _ in range(3))
    step, good = ops.AdamW([p], [m], [v]).step, {"lr": 1e-3, "step": 1}
    for bad in NO_REAL + [None]:
        for name in ("lr", "beta1", "beta2", "eps", "grad_scale"):
            refused(step, [p], **dict(good, **{name: bad}))
        if not hasattr(bad, "__len__"):   # one for each
            refused(ops.AdamW, [p], [m], [v], weight_decay=bad)
    refused(ops.AdamW, [p], [m], [v], weight_decay=["0.1"])
    for bad in NO_WHOLE + [None]:
        for name in ("step", "seed"):
            refused(step, [p], **dict(good, **{name: bad}))
    assert all((t == 0).all() for t in (p, m, v))


def test_numbers_of_other_libraries():
    logits, x, w, token = normal(1, 6, 8), normal(2, 6, 16), normal(3, 16), torch.arange(6, device="cuda")
    whole, real = (np.int64, np.int32, torch.tensor), (np.float64, int, torch.tensor)
    for a, b in zip(whole, real):
        r = ops.route_balanced(logits, a(2), groups=a(4), top_groups=a(2), group_best=a(1), scale=b(2))
        assert torch.equal(r.weight, ops.route_balanced(logits, 2, groups=4, top_groups=2, group_best=1, scale=2.0).weight)
        assert torch.equal(ops.layer_norm(x, w, eps=b(0))[0], ops.layer_norm(x, w, eps=0.0)[0])
        assert torch.equal(ops.embed(token, x, scale=b(3)), ops.embed(token, x, scale=3.0))
        assert torch.equal(ops.embed_backward(x, token, a(9), scale=b(3)), ops.embed_backward(x, token, 9, scale=3.0))
        for n in (0, 3):
            assert torch.equal(ops.dropout(x, b(0), a(n), a(n)), ops.dropout(x, 0.0, n, n))
        assert torch.equal(ops.route(logits, a(3)).expert, ops.route(logits, 3).expert)

