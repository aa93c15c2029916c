"""How many parts a layer that does not fit runs in (no GPU needed)."""
import pytest

from paper_2609_39350_amd import measure


def old(experts, top_k, tokens, fits):
    n = 1
    while not fits(experts // n) and experts % (2 * n) == 0 and experts // (2 * n) >= top_k and tokens % (2 * n) == 0:
        n *= 2
    return n


@pytest.mark.parametrize("experts,top_k,tokens", [(8, 2, 2048), (64, 8, 4096), (256, 8, 4096), (24, 2, 2048), (24, 2, 6),
                                                  (7, 1, 64), (256, 8, 100)])
def test_parts_without_groups(experts, top_k, tokens):
    for most in (0, 1, 3, 8, 20, 64, 1000):
        for balance in (None, {}, {"scores": "softmax"}, {"groups": 1, "top_groups": None}, {"groups": 1, "top_groups": 1}):
            assert measure.parts(experts, top_k, tokens, lambda n: n <= most, balance) == old(experts, top_k, tokens,
                                                                                              lambda n: n <= most)


@pytest.mark.parametrize("experts,groups,stay,top_k,want", [
    (24, 3, 1, 2, 4), (24, 8, 8, 2, 1), (24, 8, 1, 2, 1), (24, 2, 1, 2, 4), (24, 3, 3, 2, 8), (256, 8, 4, 8, 16),
    (256, 8, None, 8, 32), (256, 8, 1, 8, 4), (16, 8, 2, 8, 1), (64, 64, 8, 8, 1)])
def test_parts_leave_groups_whole_and_experts_enough(experts, groups, stay, top_k, want):
    got = measure.parts(experts, top_k, 4096, lambda n: False, {"scores": "sigmoid", "groups": groups, "top_groups": stay})
    assert got == want
    left = experts // got
    assert got == 1 or (left % groups == 0 and left // groups * (stay or groups) >= top_k)
