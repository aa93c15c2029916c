"""The measured layer: its step against automatic differentiation in 64 bits, and its figures in
a planner problem."""
import numpy as np
import pytest

from paper_2609_39350_amd import binding, workloads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


def test_layer_step_against_autograd(torch):
    """A layer's output and gradients; every bf16 rounding on the way costs up to 2^-8 of a value, and there are at
    most six between an input and a gradient."""
    from paper_2609_39350_amd import measure
    T, H, F, E, k = 96, 64, 40, 6, 2
    layer = measure.Layer(T, H, F, E, k, seed=3)
    got = measure.layer_step(layer.x, layer.router, layer.experts, layer.d_out, k)
    leaves = [t.double().cpu().requires_grad_() for t in (layer.x, layer.router, *layer.experts)]
    x, router, gate, up, down = leaves
    # the layer's own choices: logits in bf16 may order near ties otherwise
    expert = got["routing"].expert.long().cpu()
    p = torch.softmax(x @ router.T, 1).gather(1, expert)
    p = p / p.sum(1, keepdim=True)
    out = torch.zeros(T, H, dtype=torch.float64)
    for j in range(k):
        e = expert[:, j]
        g, u = (torch.bmm(w[e], x[:, :, None])[:, :, 0] for w in (gate, up))
        h = torch.nn.functional.silu(g) * u
        out = out + p[:, j, None] * torch.bmm(down[e], h[:, :, None])[:, :, 0]
    out.backward(layer.d_out.double().cpu())
    want = [out.detach()] + [t.grad for t in leaves]
    have = [got["out"], got["d_x"], got["d_router"], *got["d_experts"]]
    for name, a, b in zip(("out", "d_x", "d_router", "d_gate", "d_up", "d_down"), have, want):
        error = float((a.double().cpu() - b).norm() / b.norm())
        assert error < 6 * 2.0 ** -8, (name, error)


@pytest.mark.parametrize("bits", [32, 8])
def test_layer_learns(torch, bits):
    """Steps against the gradient of |out - target|^2 / 2 bring it down."""
    from paper_2609_39350_amd import measure
    layer = measure.Layer(256, 64, 48, 4, 2, state_bits=bits, seed=1)
    target = torch.zeros_like(layer.x)
    first = None
    for _ in range(30):
        out = layer.step()["out"].float()
        layer.d_out = (out - target).bfloat16()
        loss = float((out - target).square().mean())
        first = first or loss
        for g in layer.optimizer.moments()[1]:
            assert (g >= 0).all()
    assert loss < first


def test_measured_problem_plans(torch):
    from paper_2609_39350_amd import measure
    problem = workloads.config(1)
    got = measure.measure(problem, steps=2, warmup=1)
    assert got["part"] == 1 and got["expert_tokens"].sum() == 2048 * 2
    assert all(got[n] > 0 for n in ("route_ns", "combine_ns", "experts_ns", "opt_ns_per_param"))
    q = measure.apply(problem, 1, got)
    binding.validate(q)
    assert np.array_equal(q["cluster"]["t_dense"][0], problem["cluster"]["t_dense"][0])   # the other type's stay
    assert np.array_equal(q["cluster"]["t_dense"][1] - q["cluster"]["t_ffn"][1],
                          problem["cluster"]["t_dense"][1] - problem["cluster"]["t_ffn"][1])
    assert np.array_equal(q["model"]["expert_tokens"][got["layer"]], got["expert_tokens"])
    plan = binding.Planner(q, "cuda:0").run()
    assert sum(plan["layers"]) == 8
    with pytest.raises(ValueError):
        measure.apply(problem, 2, got)
    dense = workloads.random_tiny(4)
    dense["model"]["is_moe"][:] = 0
    with pytest.raises(ValueError):
        measure.measure(dense)


def test_part_of_the_experts(torch):
    from paper_2609_39350_amd import measure
    problem = workloads.config(1)
    got = measure.measure(problem, steps=1, warmup=0, limit_bytes=10**8, state_bits=8)
    assert got["part"] > 1 and 8 // got["part"] >= 2
    counts = measure.apply(problem, 0, got)["model"]["expert_tokens"]
    assert np.array_equal(counts, problem["model"]["expert_tokens"])
