"""A layer that runs in parts with a router of groups: the parts leave groups whole, and experts enough in those kept."""
import pytest

from paper_2609_39350_amd import workloads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


def test_parts_leave_whole_groups(torch):
    """24 experts, two for a token: halved while the groups divide them and those kept have two experts."""
    from paper_2609_39350_amd import measure
    problem = workloads.config(1)
    m = problem["model"]
    m["n_experts"], m["hidden"], m["top_k"] = 24, 64, 2
    m["params_expert"][:] = 3 * 24 * 64 * 8
    for groups, top_groups, part in ((1, 1, 8), (3, 1, 4), (8, 8, 1), (8, 1, 1), (2, 1, 4), (3, 3, 8)):
        got = measure.measure(problem, steps=1, warmup=0, limit_bytes=1, state_bits=8,
                              balance={"scores": "sigmoid", "groups": groups, "top_groups": top_groups})
        assert got["part"] == part, (groups, top_groups, got["part"])
        assert got["expert_tokens"].sum() * part == got["tokens"] * 2
