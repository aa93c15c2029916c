"""The balanced router's gradient of a token with one choice: renormalised, its weight is the scale whatever the logits are,
so the gradient is 0."""
import math

import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_operators import normal, say   # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [1.0, 2.5, 0.3, 1e-3, 7.77, 1e20])
def test_gradient_is_zero(scores, dtype, scale):
    say("one choice", scores, dtype, scale)
    for T, E, k in ((500, 64, 1), (3, 8, 1), (300, 256, 4)):
        logits = (normal(T, T, E) * 3).to(dtype)
        if k > 1:   # one expert left open to each
            one = torch.arange(T, device="cuda") * 7 % E
            logits[torch.arange(E, device="cuda")[None] != one[:, None]] = -math.inf
        how = {"scores": scores, "scale": scale}
        r = ops.route_balanced(logits, k, bias=normal(1, E) * 0.1, **how)
        assert (r.expert[:, 0] >= 0).all() and (r.expert[:, 1:] < 0).all()
        d = ops.route_balanced_backward(logits, r, normal(2, T, k), **how)
        assert (d == 0).all()
