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


@pytest.mark.parametrize("bits", [32, 8])
def test_an_optimizer_keeps_the_memory_that_it_was_made_on(bits):
    """A parameter, copy or moment given other storage afterwards: the step still works on what it was made on, which
    nothing else gets in the meantime; an optimizer made anew works on the new."""
    n = 4 << 20   # blocks of their own, which the allocator would give to the next tensor of the size
    p, c = normal(1, n), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = [normal(2, n)]
    if bits == 32:
        m, v, small = normal(3, n), normal(4, n).square(), {}
    else:
        m, v = (torch.full((n,), 40, dtype=torch.uint8, device="cuda") for _ in range(2))
        small = {k: [torch.full((n // 256,), -10, dtype=torch.int8, device="cuda")] for k in ("m_exp", "v_exp")}
    state = [p, c, m, v] + [x[0] for x in small.values()]
    before = [t.clone() for t in state]
    opt = ops.AdamW([p], [m], [v], copies=[c], **small)
    for t in state:
        t.data = t.data.clone()
    others = [torch.zeros_like(t) for t in state for _ in range(2)]   # takes freed memory, if there is any
    opt.step(g, lr=1e-2, step=5, seed=1)
    assert all((t == 0).all() for t in others)
    assert all(torch.equal(a, b) for a, b in zip(state, before))
    opt = ops.AdamW([p], [m], [v], copies=[c], **small)
    opt.step(g, lr=1e-2, step=5, seed=1)
    assert not torch.equal(p, before[0]) and torch.equal(c, p.bfloat16())


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_replays_with_the_numbers_of_its_capture(bits):
    """lr, step and seed are read by the call: every replay is the call with the same ones."""
    def make():
        p, small = normal(1, 3000), {}
        if bits == 8:
            small = {k: [torch.zeros(12, dtype=torch.int8, device="cuda")] for k in ("m_exp", "v_exp")}
        m, v = (torch.zeros(3000, dtype=torch.uint8 if bits == 8 else torch.float32, device="cuda") for _ in range(2))
        return [p, m, v], ops.AdamW([p], [m], [v], **small)

    g = [normal(2, 3000)]
    numbers = {"lr": 1e-2, "step": 3, "seed": 9}
    (captured, a), (eager, b) = make(), make()
    start = [t.clone() for t in captured]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        make()[1].step(g, **numbers)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(g, **numbers)
    assert all(torch.equal(x, y) for x, y in zip(captured, start))
    for _ in range(3):
        graph.replay()
        b.step(g, **numbers)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(captured, eager))
