"""The measured layer in its place: embedding, norm, a router whose choice is balanced, dropout onto the residual."""
import math

import pytest

from paper_2609_39350_amd import binding, workloads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


def test_block_step_against_autograd(torch):
    """Output and gradients; every bf16 rounding on the way costs up to 2^-8 of a value, and there are at most ten between
    an input and a gradient."""
    from paper_2609_39350_amd import measure, operators
    T, H, F, E, k, V, p = 96, 64, 40, 8, 2, 50, 0.25
    bias = torch.linspace(-0.1, 0.1, E, device="cuda")
    balance = {"scores": "sigmoid", "bias": bias, "groups": 4, "top_groups": 2, "scale": 1.5}
    block = measure.Block(T, H, F, E, k, seed=3, balance=balance, vocab=V, p=p)
    block.norm = tuple(torch.randn(H, device="cuda", generator=torch.Generator("cuda").manual_seed(i)) * 0.2 + 1 - i
                       for i in range(2))
    block.grad.fill_(0.5)
    got = block.forward_backward(lambda name: None)
    kept = (operators.dropout(torch.ones(T, H, device="cuda"), p, 3, 0) != 0).cpu()
    leaves = [t.double().cpu().requires_grad_() for t in (block.table, *block.norm, block.router, *block.experts)]
    table, weight, shift, router, gate, up, down = leaves
    x = table[block.token.cpu()]
    dev = x - x.mean(1, keepdim=True)
    n = dev / (dev.square().mean(1, keepdim=True) + 1e-5).sqrt() * weight + shift
    expert = got["routing"].expert.long().cpu()   # the layer's own choices
    assert (expert >= 0).all()
    s = torch.sigmoid(n @ router.T).gather(1, expert)
    s = 1.5 * s / s.sum(1, keepdim=True)
    layer = torch.zeros(T, H, dtype=torch.float64)
    for j in range(k):
        e = expert[:, j]
        g, u = (torch.bmm(w[e], n[:, :, None])[:, :, 0] for w in (gate, up))
        layer = layer + s[:, j, None] * torch.bmm(down[e], (torch.nn.functional.silu(g) * u)[:, :, None])[:, :, 0]
    cut = math.floor(p * 65536 + 0.5)
    out = x + torch.where(kept, layer * (65536 / (65536 - cut)), 0.0)
    out.backward(block.d_out.double().cpu())
    have = [got["out"], got["d_table"] - 0.5, *got["d_norm"], got["d_router"], *got["d_experts"]]
    names = ("out", "d_table", "d_norm", "d_norm_bias", "d_router", "d_gate", "d_up", "d_down")
    for name, a, b in zip(names, have, [out.detach()] + [t.grad for t in leaves]):
        error = float((a.double().cpu() - b).norm() / b.norm())
        # 0.5 was there before: the sums are rounded at that size
        assert error < 10 * 2.0 ** -8 + (name == "d_table") * 0.5 * 2.0 ** -24 * b.numel() ** 0.5 / float(b.norm()), (name, error)


def test_measure_with_block_and_balance(torch):
    from paper_2609_39350_amd import measure
    problem = workloads.config(1)
    plain = measure.measure(problem, steps=1, warmup=0)
    assert not {"embed_ns", "norm_ns", "dropout_ns"} & set(plain)
    got = measure.measure(problem, steps=2, warmup=1, balance={"scores": "softmax", "groups": 4, "top_groups": 2}, vocab=1000)
    assert all(got[n] > 0 for n in ("embed_ns", "norm_ns", "dropout_ns", "route_ns", "combine_ns", "experts_ns"))
    assert got["expert_tokens"].sum() == got["tokens"] * problem["model"]["top_k"]
    binding.validate(measure.apply(problem, 1, got))
    bias = torch.zeros(problem["model"]["n_experts"], device="cuda")
    parts = measure.measure(problem, steps=1, warmup=0, limit_bytes=10**8, state_bits=8, vocab=300,
                            balance={"scores": "sigmoid", "bias": bias})
    assert parts["part"] > 1 and parts["norm_ns"] > 0
