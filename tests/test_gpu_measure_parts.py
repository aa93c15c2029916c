"""A layer that runs in parts: its experts' times count for the whole, its router runs whole."""
import pytest

from paper_2609_39350_amd import workloads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


@pytest.mark.parametrize("limit", [10**8, 10**12])
def test_the_router_is_timed_at_its_whole_size(torch, monkeypatch, limit):
    """A router's work is tokens times experts: of a part of both it is not a part of the whole."""
    from paper_2609_39350_amd import measure
    problem = workloads.config(1)
    m = problem["model"]
    seen = {"route": [], "route_backward": []}
    for name, shapes in seen.items():
        real = getattr(measure.operators, name)
        monkeypatch.setattr(measure.operators, name,
                            lambda logits, *a, real=real, shapes=shapes, **k: (shapes.append(tuple(logits.shape)),
                                                                              real(logits, *a, **k))[1])
    steps, warmup = 3, 1
    got = measure.measure(problem, steps=steps, warmup=warmup, limit_bytes=limit, state_bits=8)
    assert (got["part"] > 1) == (limit == 10**8)
    whole = (int(m["seq_len"]) * int(m["micro_batch_size"]), int(m["n_experts"]))
    for shapes in seen.values():
        assert shapes.count(whole) == steps + warmup
    assert got["route_ns"] > 0


def test_router_step_is_the_layers(torch):
    """The parts that are timed apart are those that the layer's step is made of."""
    from paper_2609_39350_amd import measure
    layer = measure.Layer(96, 64, 40, 6, 2, seed=3)
    got = measure.layer_step(layer.x, layer.router, layer.experts, layer.d_out, 2)
    logits, r = measure.router_forward(layer.x, layer.router, 2)
    for name in ("expert", "weight", "count", "offset", "slot", "place"):
        assert torch.equal(getattr(r, name), getattr(got["routing"], name))
    d_weight = torch.randn(96, 2, device="cuda")
    d_router, d_x = measure.router_backward(layer.x, layer.router, logits, r, d_weight)
    d_logits = measure.operators.route_backward(logits, r, d_weight)
    assert torch.equal(d_router, d_logits.T @ layer.x) and torch.equal(d_x, (d_logits @ layer.router).float())


def test_a_router_of_more_experts_than_one_call_takes(torch):
    from paper_2609_39350_amd import measure
    problem = workloads.config(1)
    m = problem["model"]
    m["n_experts"], m["hidden"], m["params_expert"][:] = 2048, 64, 3 * 2048 * 64 * 8
    got = measure.measure(problem, steps=1, warmup=0, limit_bytes=10**7)
    assert got["part"] >= 2 and got["experts"] == 2048 and got["route_ns"] > 0
