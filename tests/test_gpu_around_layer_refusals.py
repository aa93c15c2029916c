"""What the operators around a layer cannot take raises ValueError, whatever is wrong with it, and launches nothing."""
import math

import numpy as np
import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_operator_refusals import refused   # noqa: E402
from .test_gpu_operators import normal   # noqa: E402

pytestmark = pytest.mark.gpu


def calls():
    x, w, r = normal(1, 6, 16), normal(2, 16), normal(3, 6)
    token = torch.arange(6, device="cuda")
    logits, d_weight = normal(4, 6, 8), normal(5, 6, 2)
    return {"route_balanced": (ops.route_balanced, (logits, 2), {"bias": normal(6, 8), "groups": 4, "top_groups": 2}),
            "route_balanced_backward": (ops.route_balanced_backward, (logits, ops.route_balanced(logits, 2), d_weight), {}),
            "layer_norm": (ops.layer_norm, (x, w, w), {}),
            "layer_norm_backward": (ops.layer_norm_backward, (x, x, w, r, r), {"add": x}),
            "embed": (ops.embed, (token, x), {}),
            "embed_backward": (ops.embed_backward, (x, token, 9), {"into": normal(7, 9, 16)}),
            "dropout": (ops.dropout, (x, 0.1, 1), {"residual": x, "counter": torch.zeros(1, dtype=torch.int64, device="cuda")}),
            "dropout_backward": (ops.dropout_backward, (x, 0.1, 1), {})}


@pytest.mark.parametrize("name", list(calls()) if torch.cuda.is_available() else [])
def test_operands(name):
    """No tensor, a tensor on the host, of another type, with one element fewer, not contiguous."""
    f, args, more = calls()[name]
    f(*args, **more)
    wrong = {3: lambda t: 3, "list": lambda t: t.tolist(), "numpy": lambda t: t.cpu().numpy(), "host": lambda t: t.cpu(),
             "complex": lambda t: t.to(torch.complex64), "short": lambda t: t[..., :-1] if t.numel() > 1 else t[:0],
             "flat": lambda t: t[None], "step": lambda t: t.repeat_interleave(2, -1)[..., ::2] if t.shape[-1] > 1 else t[:0]}
    # tensors that a call may have of any size or step by themselves
    free = {("route_balanced", 0, "short"), ("embed", 0, "short"), ("embed", 1, "short"), ("dropout_backward", 0, "short")}
    for what, change in wrong.items():
        for i, a in enumerate(args):
            if isinstance(a, torch.Tensor) and (name, i, what) not in free:
                refused(f, *args[:i], change(a), *args[i + 1:], **more)
        for key, a in more.items():
            if isinstance(a, torch.Tensor):
                refused(f, *args, **dict(more, **{key: change(a)}))


def test_sizes_and_numbers():
    logits = normal(1, 6, 8)
    for bad in ({"scores": "tanh"}, {"scores": None}, {"scores": 1}, {"groups": 3}, {"groups": 0}, {"groups": -2},
                {"groups": 2, "top_groups": 3}, {"groups": 2, "top_groups": 0}, {"group_best": 3}, {"group_best": 0},
                {"scale": 0.0}, {"scale": -1.0}, {"scale": math.nan}, {"scale": math.inf}, {"keep": [True] * 6},
                {"keep": np.ones(6, dtype=bool)}):
        refused(ops.route_balanced, logits, 2, **bad)
    for k in (0, -1, 9, 2**32 + 2):
        refused(ops.route_balanced, logits, k)
    refused(ops.route_balanced, logits, 2, out=ops.Routing(5, 8, 2))
    refused(ops.route_balanced, normal(1, 6, 130), 2, groups=65, top_groups=1)
    r = ops.Routing(6, 8, 2)
    r.weight = torch.empty_like(r.weight)
    refused(ops.route_balanced, logits, 2, out=r)
    x, w, s = normal(2, 6, 16), normal(3, 16), normal(4, 6)
    for eps in (-1e-5, math.nan, math.inf):
        refused(ops.layer_norm, x, w, eps=eps)
    refused(ops.layer_norm, x, w.bfloat16())
    refused(ops.layer_norm, x.bfloat16(), w.half())
    refused(ops.layer_norm, x.bfloat16(), w, w.bfloat16())
    refused(ops.layer_norm_backward, x.bfloat16(), x, w, s, s)
    refused(ops.layer_norm_backward, x, x, w, s, s, add=x.bfloat16())
    token = torch.arange(6, device="cuda")
    for scale in (math.nan, math.inf):
        refused(ops.embed, token, x, scale=scale)
        refused(ops.embed_backward, x, token, 9, scale=scale)
    refused(ops.embed, token.short(), x)
    for vocab in (0, -1, 2**31 - 1, 2**31, 2**32 + 9):
        refused(ops.embed_backward, x, token, vocab)
    refused(ops.embed_backward, x, token, 9, into=torch.zeros(9, 16, device="cuda", dtype=torch.bfloat16))
    for p in (-0.1, 1.5, math.nan):
        refused(ops.dropout, x, p, 1)
    refused(ops.dropout, x, 0.1, 1, residual=x.bfloat16())
    refused(ops.dropout, x, 0.1, 1, counter=torch.zeros(1, dtype=torch.int32, device="cuda"))
    refused(ops.layer_norm, x[:, :0], w[:0])
    refused(ops.dropout, x.T, 0.1, 1)
    refused(ops.dropout, x[:1].expand(6, 16), 0.1, 1)   # rows that overlap
