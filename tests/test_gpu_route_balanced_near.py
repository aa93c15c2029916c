"""The balanced router where neighbours in the order are nearer to each other than fp32 resolves, against the formula in
64 bits, at every place that the choices lie in."""
import numpy as np
import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_around_layer import balanced_ref, check_balanced   # noqa: E402
from .test_gpu_operators import say   # noqa: E402

pytestmark = pytest.mark.gpu


def near_pairs(T, E, k, scores, pairs, seed):
    """Logits [T, E] and a bias for which the sums of the experts of ranks j and j + 1, j of pairs, are nearer to each other
    than fp32 resolves, in an order that changes from token to token, and all others 2^-12 apart."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(E).astype(np.float32)
    want = np.empty(E)   # the sums, by rank
    at = 1.75
    for j in range(E):
        want[j] = at
        at -= 0.0 if j in pairs else 2.0 ** -12
    rank = rng.permutation(E)
    of = np.argsort(rank)
    for j in pairs:
        x[of[j + 1]] = x[of[j]]
    logits = np.repeat(x[None], T, 0)
    # equal logits and biases but for a few units of a logit, which leave the other sums where they are
    for r in sorted({r for j in pairs for r in (j, j + 1)}):
        logits[:, of[r]] = (logits[:, of[r]].view(np.int32) + rng.integers(-3, 4, T, dtype=np.int32)).view(np.float32)
    s = scores_of(x[None].astype(np.float64), scores)[0]
    bias = (want[rank] - s).astype(np.float32)
    return logits, bias


def scores_of(x, scores):
    if scores == "sigmoid":
        return 1 / (1 + np.exp(-x))
    e = np.exp(x - x.max(1, keepdims=True))
    return e / e.sum(1, keepdims=True)


def near_as_meant(logits, bias, scores, pairs, E):
    """Sums of the pairs within 2^-22 and, where they differ, not within the 2^-46 that 64 bits could turn; others far."""
    c = -np.sort(-(scores_of(logits.astype(np.float64), scores) + bias.astype(np.float64)), axis=1)
    gap = c[:, :-1] - c[:, 1:]
    near = np.isin(np.arange(E - 1), pairs)
    return (gap[:, near] < 2.0 ** -22).all() and (gap[:, ~near] > 2.0 ** -13).all() and \
        ((gap == 0) | (gap > 2.0 ** -46)).all()


# ranks of the pairs: the last choice and the first that is not; choices 15 and 16, the last lane's and the first one's
# second; 14 and 15; the first two; three in a row over the border
NEAR = [(k, pairs) for k in (15, 16, 17, 32) for pairs in
        ((k - 1,), (14,), (15,), (0,), (k - 2, k - 1), (k - 1, k), (k,), tuple(range(k)))]


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,G,TG", [(64, 1, 1), (256, 8, 4), (1024, 1, 1), (60, 1, 1), (240, 6, 3)])
def test_near_neighbours_of_many_choices(E, G, TG, scores):
    """Only named neighbours of the order are near: each has to be found, at every place that the choices lie in."""
    T = 40
    for k, pairs in NEAR:
        say("near neighbours", E, G, TG, scores, k, pairs)
        logits, bias = near_pairs(T, E // G * TG, k, scores, pairs, 7 * k + len(pairs) + pairs[0])
        assert near_as_meant(logits, bias, scores, pairs, E // G * TG)
        if G > TG:   # the other groups far behind, so that the choice of groups is not near
            more = E - E // G * TG
            logits = np.concatenate([logits, np.full((T, more), -30.0, dtype=np.float32)], 1)
            bias = np.concatenate([bias, np.full(more, -4.0, dtype=np.float32)])
        logits, bias = torch.from_numpy(logits).cuda(), torch.from_numpy(bias).cuda()
        how = {"bias": bias, "scores": scores, "groups": G, "top_groups": TG}
        check_balanced(ops.route_balanced(logits, k, **how), balanced_ref(logits, k, **how), E)
