"""The kernels that only large calls take, by value: products of odd sizes in 128 x 128 tiles, AdamW's streaming
form, the gradient of combine between 128 and 384 MB, the widest rows of combine."""
import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_operators import (HYPER, TINY, U32, UNIT, check_products, close, make_optimizer, normal, say,   # noqa: E402
                                 step_ref)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gather", [0, 2])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("N,K", [(4095, 1023), (1025, 4097)])
def test_products_of_odd_sizes_in_many_tiles(N, K, dtype, gather):
    """4,200 rows: 33 x 32 tiles of 128 x 128 of y (the first sizes) or of d_x (the second), 8 x 32 x 8 of d_w."""
    counts = [1029, 0, 640, 129, 1, 1500, 127, 770]
    say("odd sizes, many tiles", N, K, dtype, gather)
    check_products(counts, 4, N, K, dtype, gather, seed=N)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad,copy", [(torch.float32, torch.bfloat16), (torch.bfloat16, None), (torch.float16, torch.float16)])
def test_adamw_over_more_than_16_million_elements(bits, grad, copy):
    """Aligned tensors that end inside a workgroup's 4,096 elements, in whole blocks and not, and unaligned ones beside
    them."""
    say("adamw, streaming", bits, grad, copy)
    sizes = [[(1 << 23) + 1234, 4096, 5], [(1 << 23) + 256, 4099, 257, 8191]]
    parts = [make_optimizer(n, bits, copy, grad, seed=1000 * i, shift=i)[0] for i, n in enumerate(sizes)]
    s = {k: None if parts[0][k] is None else parts[0][k] + parts[1][k] for k in parts[0]}
    more = {k: s[k] for k in ("m_exp", "v_exp") if k in s}
    opt = ops.AdamW(s["param"], s["m"], s["v"], copies=s["copy"], weight_decay=s["decay"], **more)
    before = [p.clone() for p in s["param"]]
    m0, v0 = ([x.double().clone() for x in part] for part in opt.moments())
    opt.step(s["grad"], step=7, seed=99, **HYPER)
    m1, v1 = opt.moments()
    for i in range(len(before)):
        p, m, v, size, move = step_ref(before[i], s["grad"][i], m0[i], v0[i], s["decay"][i], 7, **HYPER)
        # the bounds of the smaller calls' test
        m_off = size * 3 * U32
        rel = torch.where(m.abs() > 0, m_off / m.abs().clamp_min(1e-300), 0.0)
        close(s["param"][i], p, move * (rel + 12 * U32) + (p.abs() + before[i].double().abs()) * 2 * U32, ("param", i))
        if copy is not None:
            assert torch.equal(s["copy"][i], s["param"][i].to(copy))
        if bits == 32:
            close(m1[i], m, m_off + 1e-44, ("m", i))
            close(v1[i], v, v * 6 * U32 + 1e-44, ("v", i))
            continue
        # the codes are held to those of smaller calls by the next test
        assert bool((m1[i].double() * m >= 0).all())
        assert bool((v1[i][v > 0] > 0).all())
    if bits == 8:   # the values in bf16 are those in fp32, in the streaming form and tensor by tensor
        m2, v2 = opt.moments(torch.bfloat16)
        for i in range(len(before)):
            small = ops.AdamW(*([s[k][i]] for k in ("param", "m", "v")), **{k: [x[i]] for k, x in more.items()}).moments()
            for a, b, c in ((m1[i], m2[i], small[0][0]), (v1[i], v2[i], small[1][0])):
                assert torch.equal(a, c) and torch.equal(a, b.float())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad,copy", [(torch.float32, torch.bfloat16), (torch.bfloat16, None), (torch.float16, torch.float16)])
def test_adamw_streams_to_the_same_bits(bits, grad, copy):
    """Tensors of a call of 15 million elements, and the same tensors, seed and indices in a call that one more makes
    too large for it."""
    say("adamw, both forms", bits, grad, copy)
    sizes = [[(1 << 22) + 1234, 4096, 5], [(1 << 23) + 256, 4099, 257, 8191], [1 << 21, 77]]
    last = make_optimizer([1 << 23], bits, copy, grad, seed=5)[0]
    out = []
    for more in (False, True):
        parts = [make_optimizer(n, bits, copy, grad, seed=1000 * i, shift=i % 2)[0] for i, n in enumerate(sizes)]
        s = {k: None if parts[0][k] is None else sum((p[k] for p in parts + [last] * more), []) for k in parts[0]}
        n = len(s["param"]) - more
        opt = ops.AdamW(s["param"], s["m"], s["v"], copies=s["copy"], weight_decay=s["decay"],
                        **{k: s[k] for k in ("m_exp", "v_exp") if k in s})
        assert (sum(p.numel() for p in s["param"]) > 1 << 24) == more
        opt.step(s["grad"], step=7, seed=99, **HYPER)
        out.append([t for k in ("param", "m", "v", "copy", "m_exp", "v_exp") if s.get(k) is not None for t in s[k][:n]]
                   + [t for part in opt.moments() for t in part[:n]])
    assert len(out[0]) == len(out[1]) and all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("dtype,H", [(torch.bfloat16, 4096), (torch.float16, 4104), (torch.float32, 2056)])
def test_combine_backward_of_200_megabytes(dtype, H):
    T, k = 3100, 8
    rows = T * k
    say("combine_backward", rows * H * y_bytes(dtype) >> 20, "MB")
    r = ops.route(normal(1, T, 64), k, keep=torch.arange(T, device="cuda") % 11 != 3)
    y, d_out = normal(2, rows, H, dtype=dtype), normal(3, T, H, dtype=dtype)
    y[int(r.offset[-1]):] = float("nan")
    d_y, d_weight = ops.combine_backward(d_out, y, r.slot, r.place, r.weight)
    slot, place, w = r.slot.long(), r.place.long(), r.weight.double().view(-1)
    for rows_here in torch.arange(rows, device="cuda").split(4096):
        at = slot[rows_here]
        want = torch.where(at[:, None] < 0, 0.0, w[at.clamp_min(0)][:, None] * d_out[at.clamp_min(0) // k].double())
        close(d_y[rows_here], want, want.abs() * (UNIT[dtype] + U32) + TINY[dtype], "d_y")
        p = place.view(-1)[rows_here]
        terms = torch.where(p[:, None] < 0, 0.0, d_out[rows_here // k].double() * y[p.clamp_min(0)].double())
        close(d_weight.view(-1)[rows_here], terms.sum(1), terms.abs().sum(1) * (H + 1) * U32 + 1e-38, "d_weight")


def y_bytes(dtype):
    return torch.empty(0, dtype=dtype).element_size()


@pytest.mark.parametrize("hidden", [(1 << 24) - 1, 1 << 24])
def test_combine_of_the_widest_rows(hidden):
    say("combine, hidden", hidden)
    y = torch.arange(hidden, device="cuda").remainder(251).to(torch.bfloat16).expand(3, hidden).contiguous()
    y[1] *= 2
    place = torch.tensor([[1, 0], [-1, 2]], dtype=torch.int32, device="cuda")
    out = ops.combine(y, place)
    assert torch.equal(out[0], (y[0].float() * 3).bfloat16()) and torch.equal(out[1], y[2])
