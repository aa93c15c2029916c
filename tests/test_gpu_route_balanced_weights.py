"""The balanced router's weights by bounds of their own arithmetic, some units of 2^-24, whatever the number of experts."""
import math

import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_around_layer import balanced_ref   # noqa: E402
from .test_gpu_operators import U32, close, normal, say   # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def units(x, top, scores, renormalize, E):
    """Of the chosen logits x [T, k] and the row's largest, top [T, 1].

    An exponential is off by 3.5 units (2 of the instruction, 1.5 of what corrects its argument's rounding) and by one for
    each unit that its argument's difference is long.  Sums of the chosen take 5 additions, a quotient and the scale one
    each.  The total of a softmax that is not renormalised is of exponentials whose argument is rounded twice and
    multiplied by a constant that is off by 0.22: 2.22 units times the shares' mean difference, at most log E, then 2 of
    the instruction, a lane's additions and 4.  One more for the products of errors."""
    if scores == "sigmoid":
        if not renormalize:   # exponential, 1 + it, quotient, scale
            return torch.full_like(x, 3.5 + 1 + 1 + 1 + 1)
        low = x.clamp_max(0)
        d = low.amax(1, keepdim=True) - low
        one = 3.5 + 3.5 / 2 + 1 + 1   # over 1 + an exponential
        return d + one + d.amax(1, keepdim=True) + one + 5 + 2 + 1
    if renormalize:
        d = x.amax(1, keepdim=True) - x
        return d + 3.5 + d.amax(1, keepdim=True) + 3.5 + 5 + 2 + 1
    lane = next(n for n in (4, 8, 16, 32, 64) if E <= 16 * n)
    return top - x + 3.5 + 2.22 * math.log(E) + 2 + lane + 3 + 2 + 1


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T,E,k,G,TG", [(3000, 8, 2, 1, 1), (3000, 64, 6, 8, 4), (3000, 256, 8, 8, 4), (1500, 512, 32, 1, 1),
                                        (1500, 1024, 8, 32, 8), (1500, 1000, 20, 1, 1)])
def test_weights(T, E, k, G, TG, scores, renormalize, dtype):
    say("weights", T, E, k, G, TG, scores, renormalize, dtype)
    logits = (normal(E + k, T, E) * 2).to(dtype)
    for bias in (None, normal(3, E) * 0.1, torch.zeros(E, device="cuda")):
        how = {"bias": bias, "scores": scores, "groups": G, "top_groups": TG, "renormalize": renormalize, "scale": 2.5}
        r = ops.route_balanced(logits, k, **how)
        ref = balanced_ref(logits, k, **how)
        assert torch.equal(r.expert.cpu().long(), ref["expert"])
        x = logits.double().cpu()
        off = units(x.gather(1, ref["expert"]), x.amax(1, keepdim=True), scores, renormalize, E)
        close(r.weight.cpu(), ref["weight"], ref["weight"] * off * U32, "weight")
