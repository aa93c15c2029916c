"""The gradient of combine where slot and place do not agree: d_y goes by slot, d_weight by place, as the
header states, and every row of both is defined."""
import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_operators import TINY, U32, UNIT, close, gen, normal, say   # noqa: E402

pytestmark = pytest.mark.gpu


def reference(d_out, y, slot, place, weight):
    """d_y, d_weight and the sum of d_weight's products' sizes, in 64 bits on the host."""
    d, yd, w = d_out.double().cpu(), y.double().cpu(), weight.double().cpu().view(-1)
    rows, k = y.shape[0], place.shape[1]
    d_y = torch.zeros(yd.shape, dtype=torch.float64)
    d_weight, size = (torch.zeros(rows, dtype=torch.float64) for _ in range(2))
    for i, (s, p) in enumerate(zip(slot.tolist(), place.view(-1).tolist())):
        if 0 <= s < rows:
            d_y[i] = w[s] * d[s // k]
        if 0 <= p < rows:
            d_weight[i], size[i] = (d[i // k] * yd[p]).sum(), (d[i // k] * yd[p]).abs().sum()
    return d_y, d_weight.view(place.shape), size.view(place.shape)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("H", [7, 64, 1032])
@pytest.mark.parametrize("what", ["dropped place", "dropped slot", "both", "place twice", "slot twice", "out of range",
                                  "any"])
def test_gradient_where_slot_and_place_disagree(what, H, dtype):
    T, k = 21, 4
    rows = T * k
    say("combine", what, H, dtype)
    r = ops.route(normal(1, T, 10), k)
    slot, place = r.slot.clone(), r.place.clone()
    flat = place.view(-1)
    some = torch.randperm(rows, generator=gen(2), device="cuda")[:rows // 3]
    if what in ("dropped place", "both"):
        flat[some] = -1
    if what in ("dropped slot", "both"):
        slot[some if what == "dropped slot" else some.flip(0)[:9]] = -1
    if what == "place twice":
        flat[some] = flat[some.roll(1)[:1]].expand_as(some).clone()
    if what == "slot twice":
        slot[some] = slot[some[:1]].expand_as(some).clone()
    if what == "out of range":
        flat[some] = rows + some.int()
        slot[some.flip(0)[:11]] = torch.iinfo(torch.int32).max
        slot[some[:2]], flat[some[2:4]] = -5, torch.iinfo(torch.int32).min
    if what == "any":
        slot.copy_(torch.randint(-2, rows + 2, (rows,), generator=gen(3), device="cuda"))
        flat.copy_(torch.randint(-2, rows + 2, (rows,), generator=gen(4), device="cuda"))
    y, d_out, weight = normal(5, rows, H, dtype=dtype), normal(6, T, H, dtype=dtype), normal(7, T, k)
    # memory that a row without a writer would show
    torch.full((rows, H), 77.0, dtype=dtype, device="cuda")
    d_y, d_weight = ops.combine_backward(d_out, y, slot, place, weight)
    want_y, want_w, size = reference(d_out, y, slot, place, weight)
    close(d_y.cpu(), want_y, want_y.abs() * (UNIT[dtype] + U32) + TINY[dtype], "d_y")
    close(d_weight.cpu(), want_w, size * (H + 1) * U32 + 1e-38, "d_weight")
    assert (d_y[(slot < 0) | (slot >= rows)] == 0).all() and (d_weight[(place < 0) | (place >= rows)] == 0).all()
