"""Layer norm of rows too long or too short to be held: sums of equal elements, whose roundings in 32 bits would add up, by
bounds that do not grow with the row."""
import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_operators import TINY, U32, UNIT, close, normal, say   # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H", [20001, (1 << 20) + 3, 1 << 24])
def test_rows_of_one_element(H, dtype):
    """All of a row's elements are the same: 64 bits hold their sum and the mean is the element itself."""
    say("layer_norm", H, dtype)
    values = torch.tensor([0.1, -1 / 3, 1000.3], device="cuda").to(dtype)
    x = values[:, None].expand(3, H).contiguous()
    w, b = normal(1, H), normal(2, H)
    y, mean, rstd = ops.layer_norm(x, w, b, eps=1e-5)
    assert torch.equal(mean, values.float())
    assert (y.float() == b.to(dtype).float()).all()   # no element differs from the mean
    y, mean, rstd = ops.layer_norm(x, w, b, eps=1e-5, center=False)
    v = values.double()[:, None]
    want = (v * v + 1e-5).rsqrt()
    # the mean of the squares and its sum with eps are rounded, then root and quotient, half a step each: (1 + 1) / 2 + 2,
    # and a fourth unit for eps, itself rounded
    close(rstd[:, None], want, want * 4 * U32, "rstd")
    # products of x, rstd and the weight, then the bias; y's own rounding
    out = v * want * w.double() + b.double()
    close(y, out, (v * want * w.double()).abs() * 7 * U32 + out.abs() * (U32 + UNIT[dtype]) + TINY[dtype], "y")


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("H", [20001, (1 << 20) + 3])
def test_gradient_of_long_rows(H, center):
    """Gradients and elements that take two values each: the means over a row are their formulas' to a few units."""
    say("layer_norm_backward", H, center)
    R = 3
    at = torch.arange(H, device="cuda")
    x = torch.where(at % 2 == 0, 0.7, 0.1).expand(R, H).contiguous()
    d_y = torch.where(at % 3 == 0, 0.3, 0.1).expand(R, H).contiguous()
    w = torch.ones(H, device="cuda")
    y, mean, rstd = ops.layer_norm(x, w, eps=1e-5, center=center)
    d_x, d_w, d_b = ops.layer_norm_backward(d_y, x, w, mean, rstd)
    # by the kernel's own mean and rstd, which are inputs of the gradient
    m = mean.double()[:, None] if center else 0.0
    rs, g = rstd.double()[:, None], d_y.double()
    hat = (x.double() - m) * rs
    a = g.mean(1, keepdim=True) if center else 0.0 * rs
    b = (g * hat).mean(1, keepdim=True)
    want = rs * (g - a - hat * b)
    # hat: 2 units of it, the means: rounded once and of products with hat 3 units of their terms, the differences and
    # products 5 more
    size = g.abs() + a.abs() + (hat * b).abs() + hat.abs() * (g * hat).abs().mean(1, keepdim=True)
    close(d_x, want, 8 * U32 * rs * size, "d_x")
    for name, got, terms in (("d_weight", d_w, g * hat), ("d_bias", d_b, g)):
        close(got, terms.sum(0), 16 * U32 * terms.abs().sum(0), name)


@pytest.mark.parametrize("H", [1, 5, 7])
def test_weight_gradient_of_many_short_rows(H):
    """Rows of less than eight elements, all with the same gradient: parts of 2,048 rows and more."""
    R = (1 << 20) + 5
    say("layer_norm_backward", R, H)
    x = normal(1, R, H)
    d_y = torch.full((R, H), 0.1, device="cuda")
    mean, rstd = torch.zeros(R, device="cuda"), torch.full((R,), 1.0, device="cuda")
    _, d_w, d_b = ops.layer_norm_backward(d_y, x, torch.ones(H, device="cuda"), mean, rstd)
    # of 512 parts a run of 32 is added up, then 16 runs, in 32 bits; 4 for the parts' rounding and xhat's
    for name, got, terms in (("d_weight", d_w, d_y.double() * x.double()), ("d_bias", d_b, d_y.double())):
        close(got, terms.sum(0), (32 + 16 + 4) * U32 * terms.abs().sum(0), name)
