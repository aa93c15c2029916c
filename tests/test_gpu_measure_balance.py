"""The measured layer with a router whose choice is balanced: its gradients go by all that its weights were made with."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("kept", [False, True])
def test_router_backward_is_the_forward_pass_gradient(torch, scores, renormalize, kept):
    """Against differentiation in 64 bits of the weights that the forward pass gave.  The logits' gradient is the balanced
    router's own; the products with it are fp32 sums of 50 and 12 terms."""
    from paper_2609_39350_amd import measure
    T, H, E, k = 50, 32, 12, 3
    g = torch.Generator("cuda").manual_seed(1)
    x, router, d_weight = (torch.randn(s, generator=g, device="cuda") for s in ((T, H), (E, H), (T, k)))
    router *= H ** -0.5
    keep = torch.rand(T, generator=g, device="cuda") < 0.7 if kept else None
    balance = {"scores": scores, "groups": 4, "top_groups": 2, "scale": 1.5, "renormalize": renormalize}
    if kept:
        balance["keep"] = keep
    logits, r = measure.router_forward(x, router, k, balance)
    d_router, d_x = measure.router_backward(x, router, logits, r, d_weight, balance)
    leaves = [t.double().cpu().requires_grad_() for t in (x, router)]
    s = leaves[0] @ leaves[1].T
    s = torch.sigmoid(s) if scores == "sigmoid" else torch.softmax(s, 1)
    expert = r.expert.long().cpu()   # the router's own choices
    chosen = torch.where(expert >= 0, s.gather(1, expert.clamp_min(0)), 0.0)
    weight = 1.5 * chosen
    if renormalize:
        weight = weight / chosen.sum(1, keepdim=True).clamp_min(1e-30)
    (weight * d_weight.double().cpu()).sum().backward()
    for name, a, leaf in (("d_router", d_router, leaves[1]), ("d_x", d_x, leaves[0])):
        error = float((a.double().cpu() - leaf.grad).norm() / leaf.grad.norm())
        # logits of 32 products, scores of 12, sums of 50: less than 200 roundings of 2^-24, of terms that may cancel by 10
        assert error < 2000 * 2.0 ** -24, (name, error)


def test_a_layer_with_tokens_that_take_no_experts(torch):
    from paper_2609_39350_amd import measure
    keep = torch.arange(96, device="cuda") % 3 > 0
    balance = {"scores": "sigmoid", "groups": 4, "top_groups": 2, "keep": keep, "renormalize": False}
    layer = measure.Layer(96, 64, 40, 8, 2, seed=3, balance=balance)
    got = layer.forward_backward(lambda name: None)
    assert ((got["routing"].expert < 0).all(1) == ~keep).all()
    assert (got["out"][~keep] == 0).all() and (got["d_x"][~keep] == 0).all()
    assert got["d_router"].isfinite().all() and all(d.isfinite().all() for d in got["d_experts"])
