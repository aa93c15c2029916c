"""Buffers whose addresses an object keeps: a Routing's outputs and an AdamW's tensors, replaced after it
was made."""
import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_operators import normal   # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["weight", "expert", "count", "offset", "slot", "place"])
@pytest.mark.parametrize("how", ["attribute", "data"])
def test_a_routing_with_a_replaced_buffer_is_refused(name, how):
    """Its call would write to memory that nothing holds any more."""
    logits = normal(1, 80, 16)
    r = ops.Routing(80, 16, 2)
    first = ops.route(logits, 2, out=r)
    want = {n: getattr(first, n).clone() for n in ("weight", "expert", "count", "offset", "slot", "place")}
    new = torch.full_like(getattr(r, name), 5)
    if how == "attribute":
        setattr(r, name, new)
    else:
        getattr(r, name).data = new
    with pytest.raises(ValueError):
        ops.route(logits, 2, out=r)
    torch.cuda.synchronize()
    assert (getattr(r, name) == 5).all()
    again = ops.route(logits, 2, out=ops.Routing(80, 16, 2))
    assert all(torch.equal(getattr(again, n), w) for n, w in want.items())
