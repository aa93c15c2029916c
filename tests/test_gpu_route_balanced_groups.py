"""The balanced router by groups whose sums leave fp32, against the formulas in 64 bits."""
import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_around_layer import balanced_ref, check_balanced   # noqa: E402
from .test_gpu_operators import normal, say   # noqa: E402

pytestmark = pytest.mark.gpu
F32 = torch.float32
LOW = torch.finfo(F32).min


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T,E,k,G,TG", [   # groups of whole lanes, and of others
    (70, 256, 8, 8, 4), (50, 16, 6, 8, 6), (40, 512, 20, 16, 5), (70, 60, 8, 6, 4), (50, 63, 12, 21, 9), (30, 1000, 4, 8, 2)])
@pytest.mark.parametrize("far", [LOW, -2.5e38, -1e9, 1e9, -LOW])
def test_groups_of_far_biases(T, E, k, G, TG, scores, far):
    """Biases that take groups out, or put them first, without an infinity: two of them add up to more than fp32 holds.  Their
    groups are open: where too few others are, they are chosen."""
    say("groups of far biases", T, E, k, G, TG, scores, far)
    logits, plain = normal(E, T, E), normal(5, E) * 0.1
    for n in (1, G - TG, G - TG + 1, G - 1, G):   # how many, the last ones and every other one
        for which in (range(G - n, G), range(G - 1, -1, -2)[:n]):
            bias = plain.clone()
            for g in which:
                bias[g * (E // G):(g + 1) * (E // G)] = far
            for best in (1, 2):
                how = {"bias": bias, "scores": scores, "groups": G, "top_groups": TG, "group_best": best}
                ref = balanced_ref(logits, k, **how)
                assert (ref["expert"] >= 0).all() or TG * (E // G) < k   # as meant: all experts are open
                check_balanced(ops.route_balanced(logits, k, **how), ref, E)
