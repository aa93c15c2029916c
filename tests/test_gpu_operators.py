"""The training-step operators against their formulas in 64 bits, on the GPU.

Bounds follow from the arithmetic: u(type) is half a unit in the last place of a rounded result
(fp32 2^-24, fp16 2^-11 with 2^-25 below its normal range, bf16 2^-9 counted as 2^-8 of the value), and a
sum of n products in fp32 is off by at most n 2^-24 times the sum of the products' sizes.
"""
import math

import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
UNIT = {torch.float32: U32, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}
HALF = [torch.bfloat16, torch.float16]


def say(*a):
    print(*a, flush=True)


def close(got, want, bound, what=""):
    """|got - want| <= bound everywhere; an infinity or NaN only where the formula has it."""
    got, want = got.double(), want.double()
    fine = want.isfinite()
    assert torch.equal(fine, got.isfinite()), what
    over = ((got - want).abs() - bound)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, (what, float(over.max()))


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen(seed), device="cuda").to(dtype)


# ------------------------------------------------------------------ the router
def route_ref(logits, k, keep, renormalize):
    """expert, weight and order in 64 bits, token by token on the host."""
    x = logits.double().cpu()
    T, E = x.shape
    expert, weight = torch.full((T, k), -1), torch.zeros(T, k, dtype=torch.float64)
    probs = torch.zeros(T, E, dtype=torch.float64)
    for t in range(T):
        if keep is not None and not bool(keep[t]):
            continue
        row = [-math.inf if math.isnan(v) else v for v in x[t].tolist()]
        order = sorted((e for e in range(E) if row[e] > -math.inf), key=lambda e: (-row[e], e))[:k]
        if not order:
            continue
        top = row[order[0]]
        e = [1.0 if v == top else math.exp(v - top) if v > -math.inf else 0.0 for v in row]
        probs[t] = torch.tensor(e, dtype=torch.float64) / sum(e)
        total = sum(e[i] for i in order) if renormalize else sum(e)
        for j, i in enumerate(order):
            expert[t, j], weight[t, j] = i, e[i] / total
    flat = expert.reshape(-1).tolist()
    rows = [r for e in range(E) for r, f in enumerate(flat) if f == e] if T * k * E <= 1 << 22 else \
        [r for f, r in sorted((f, r) for r, f in enumerate(flat) if f >= 0)]
    place = [-1] * len(flat)
    for i, r in enumerate(rows):
        place[r] = i
    count = torch.bincount(torch.tensor([f for f in flat if f >= 0], dtype=torch.int64), minlength=E)
    return {"expert": expert, "weight": weight, "probs": probs, "count": count,
            "offset": torch.cat([torch.zeros(1, dtype=torch.int64), count.cumsum(0)]),
            "slot": torch.tensor(rows + [-1] * (len(flat) - len(rows)), dtype=torch.int64),
            "place": torch.tensor(place, dtype=torch.int64).view(T, k)}


def check_routing(r, ref, E, span=40.0):
    for name in ("expert", "count", "offset", "slot", "place"):
        assert torch.equal(getattr(r, name).cpu().long(), ref[name].long()), name
    # the exponent's argument is rounded once (span 2^-24 of the value), exp, E additions and the division
    close(r.weight.cpu(), ref["weight"], ref["weight"] * (E + span + 8) * U32 + 1e-38, "weight")


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("T,E,k,dtype", [
    (1, 1, 1, torch.float32), (1, 8, 8, torch.float32), (4, 64, 8, torch.bfloat16), (63, 60, 6, torch.float16),
    (64, 256, 8, torch.float32), (65, 256, 8, torch.bfloat16), (129, 100, 17, torch.float32),
    (257, 512, 32, torch.float16), (70, 1024, 32, torch.float32), (33, 1000, 3, torch.bfloat16),
    (2049, 16, 2, torch.float32)])
def test_route(T, E, k, dtype, renormalize):
    say("route", T, E, k, dtype, renormalize)
    logits = normal(T + E, T, E, dtype=dtype) * 3
    keep = torch.rand(T, generator=gen(7), device="cuda") < 0.8
    for kp in (None, keep):
        r = ops.route(logits, k, keep=kp, renormalize=renormalize)
        check_routing(r, route_ref(logits, k, kp, renormalize), E)


@pytest.mark.parametrize("renormalize", [False, True])
def test_route_ties_masks_and_infinities(renormalize):
    low = torch.finfo(torch.float32).min
    inf, nan = math.inf, math.nan
    rows = [[0.0] * 6, [1, 1, 2, 2, 1, 1], [-inf] * 6, [nan] * 6, [nan, 3, -inf, 3, nan, -inf], [low] * 6,
            [low, 0, low, low, low, low], [inf, 0, inf, 1, nan, -inf], [-0.0, 0.0, -0.0, 0.0, -1, -1],
            [inf, -inf, -inf, -inf, -inf, -inf], [5, -inf, -inf, -inf, -inf, -inf]]
    logits = torch.tensor(rows * 8, device="cuda")   # 88 tokens: more than one workgroup
    for n in (len(rows), len(rows) * 8):
        r = ops.route(logits[:n], 3, renormalize=renormalize)
        check_routing(r, route_ref(logits[:n], 3, None, renormalize), 6)
        d_weight = normal(3, n, 3)
        d = ops.route_backward(logits[:n], r, d_weight, renormalize=renormalize)
        assert d.isfinite().all()
        closed = logits[:n].isnan() | (logits[:n] == -inf)
        assert (d[closed] == 0).all()


def test_route_strided_rows_kept_buffers_and_no_tokens():
    wide = normal(1, 300, 70)
    r = ops.Routing(300, 64, 4, "cuda")
    for lo in (0, 3):
        logits = wide[:, lo:lo + 64]
        assert ops.route(logits, 4, out=r) is r
        check_routing(r, route_ref(logits, 4, None, True), 64)
        g = normal(2, 300, 4)
        for renormalize in (True, False):
            q = ops.route(logits, 4, renormalize=renormalize)
            a = ops.route_backward(logits, q, g, renormalize=renormalize)
            b = ops.route_backward(logits.contiguous(), q, g, renormalize=renormalize)
            assert torch.equal(a, b)
    r = ops.route(torch.empty(0, 8, device="cuda"), 2)
    assert r.count.tolist() == [0] * 8 and r.offset.tolist() == [0] * 9
    assert ops.route_backward(torch.empty(0, 8, device="cuda"), r, torch.empty(0, 2, device="cuda")).shape == (0, 8)


@pytest.mark.parametrize("T,E,k", [(40000, 64, 8), (32768, 256, 8), (5000, 1024, 4)])
def test_route_many_tokens(T, E, k):
    """The order of many workgroups, against a stable sort."""
    say("route", T, E, k)
    logits = normal(9, T, E)
    r = ops.route(logits, k)
    value, index = torch.sort(logits, dim=1, descending=True, stable=True)
    assert torch.equal(r.expert.long(), index[:, :k])
    order = torch.sort(index[:, :k].reshape(-1), stable=True).indices
    assert torch.equal(r.slot.long(), order)
    assert torch.equal(r.place.view(-1)[order].long(), torch.arange(T * k, device="cuda"))
    assert torch.equal(r.count.long(), torch.bincount(index[:, :k].reshape(-1), minlength=E))
    assert torch.equal(r.offset[1:].long(), r.count.long().cumsum(0)) and int(r.offset[0]) == 0
    want = torch.softmax(value[:, :k].double(), 1)
    close(r.weight, want, want * (E + 48) * U32, "weight")


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("T,E,k,dtype", [(1, 8, 2, torch.float32), (37, 60, 6, torch.float32),
                                         (100, 256, 8, torch.bfloat16), (19, 512, 32, torch.float16),
                                         (5, 1024, 1, torch.float32)])
def test_route_backward(T, E, k, dtype, renormalize):
    say("route_backward", T, E, k, dtype, renormalize)
    logits = normal(T, T, E, dtype=dtype) * 2
    logits[torch.rand((T, E), generator=gen(3), device="cuda") < 0.2] = -math.inf
    keep = torch.rand(T, generator=gen(4), device="cuda") < 0.8
    d_weight = normal(5, T, k)
    r = ops.route(logits, k, keep=keep, renormalize=renormalize)
    d = ops.route_backward(logits, r, d_weight, keep=keep, renormalize=renormalize)
    ref = route_ref(logits, k, keep, renormalize)
    ok = ref["expert"] >= 0
    g = torch.where(ok, d_weight.double().cpu(), 0.0)
    spread = torch.zeros(T, E + 1, dtype=torch.float64)
    index = torch.where(ok, ref["expert"], E)
    if renormalize:
        want = spread.scatter(1, index, ref["weight"] * (g - (g * ref["weight"]).sum(1, keepdim=True)))[:, :E]
        p = spread.scatter(1, index, ref["weight"])[:, :E]
    else:
        full = spread.scatter(1, index, g)[:, :E]
        p = ref["probs"]
        want = p * (full - (full * p).sum(1, keepdim=True))
    size = p * (g.abs().amax(1, keepdim=True) * 2)
    close(d.cpu(), want, want.abs() * UNIT[dtype] + TINY[dtype] + size * (E + k + 56) * U32, "d_logits")


@pytest.mark.parametrize("renormalize", [False, True])
def test_route_gradient_against_differences(renormalize):
    """d(sum g w)/d logits by central differences of the formula in 64 bits: the choice does not change within the
    step, which is small beside the gaps."""
    T, E, k, h = 3, 10, 3, 1e-5
    logits = torch.stack([torch.randperm(E, generator=gen(t), device="cuda").float() * 0.3 for t in range(T)])
    g = normal(6, T, k)
    r = ops.route(logits, k, renormalize=renormalize)
    d = ops.route_backward(logits, r, g, renormalize=renormalize).cpu().double()
    index = r.expert.long().cpu()

    def value(x):
        p = torch.softmax(x, 1).gather(1, index)
        return float((g.double().cpu() * (p / p.sum(1, keepdim=True) if renormalize else p)).sum())

    x = logits.double().cpu()
    for t in range(T):
        for e in range(E):
            step = torch.zeros_like(x)
            step[t, e] = h
            slope = (value(x + step) - value(x - step)) / (2 * h)
            assert abs(float(d[t, e]) - slope) < 1e-6   # h^2 / 6 of the third derivative, 2^-52 / h, fp32 of the kernel


# --------------------------------------------------- a token's expert outputs
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,k,H", [(1, 1, 1), (3, 2, 8), (17, 8, 4096), (5, 32, 2056), (40, 6, 1001), (9, 3, 7168)])
def test_combine_and_backward(T, k, H, dtype):
    say("combine", T, k, H, dtype)
    E = 40
    logits = normal(T + k, T, E)
    keep = torch.rand(T, generator=gen(1), device="cuda") < 0.7 if T > 2 else None
    r = ops.route(logits, k, keep=keep)
    rows = T * k
    y = normal(2, rows, H, dtype=dtype)
    used = int(r.offset[-1])
    y[used:] = math.nan   # rows that no place names are not read
    d_out = normal(3, T, H, dtype=dtype)
    out = ops.combine(y, r.place, r.weight)
    d_y, d_weight = ops.combine_backward(d_out, y, r.slot, r.place, r.weight)
    place, w = r.place.long().cpu(), r.weight.double().cpu()
    yd, dd = y.double().cpu(), d_out.double().cpu()
    want, size = torch.zeros(T, H, dtype=torch.float64), torch.zeros(T, H, dtype=torch.float64)
    want_y = torch.zeros(rows, H, dtype=torch.float64)
    want_w, size_w = torch.zeros(T, k, dtype=torch.float64), torch.zeros(T, k, dtype=torch.float64)
    for t in range(T):
        for j in range(k):
            p = int(place[t, j])
            if p >= 0:
                want[t] += w[t, j] * yd[p]
                size[t] += (w[t, j] * yd[p]).abs()
                want_y[p] = w[t, j] * dd[t]
                want_w[t, j] = (dd[t] * yd[p]).sum()
                size_w[t, j] = (dd[t] * yd[p]).abs().sum()
    u, tiny = UNIT[dtype], TINY[dtype]
    close(out.cpu(), want, want.abs() * u + tiny + size * (k + 1) * U32, "out")
    close(d_y.cpu(), want_y, want_y.abs() * (u + U32) + tiny, "d_y")
    close(d_weight.cpu(), want_w, size_w * (H + 1) * U32 + 1e-38, "d_weight")
    # without weights: the sum, as the gradient of gathered rows
    plain = ops.combine(y, r.place)
    ones = torch.where(place >= 0, 1.0, 0.0).float().cuda()
    assert torch.equal(plain, ops.combine(y, r.place, ones))


def test_combine_index_out_of_range_counts_as_none():
    y = normal(1, 4, 16)
    place = torch.tensor([[0, 4], [-7, 2]], dtype=torch.int32, device="cuda")
    out = ops.combine(y, place, torch.ones(2, 2, device="cuda"))
    assert torch.equal(out, torch.stack([y[0], y[2]]))
    assert ops.combine(y, place[:0], None).shape == (0, 16)
    assert ops.combine(y[:0], place, None).abs().sum() == 0


# ------------------------------------------------- products grouped by expert
def offsets(counts):
    return torch.tensor([0] + list(counts), device="cuda").cumsum(0).int()


def product_ref(x, w, off, row):
    """y, the sum of the products' sizes."""
    R, N = len(row), w.shape[1]
    y, size = (torch.zeros(R, N, dtype=torch.float64, device="cuda") for _ in range(2))
    for e in range(len(off) - 1):
        a, b = off[e], off[e + 1]
        if b > a:
            xe, we = x[row[a:b]].double(), w[e].double().T.contiguous()
            y[a:b], size[a:b] = xe @ we, xe.abs() @ we.abs()
    return y, size


def check_products(counts, extra, N, K, dtype, gather_k=0, seed=0, out_dtypes=(torch.float32, None), pad=0):
    """All three products for experts of these counts; `extra` rows that no expert has; gather_k: rows come through
    slot, gather_k choices a token; pad: the rows of x and d_y lie this many elements further apart."""
    E, used = len(counts), sum(counts)
    R = used + extra
    off = offsets(counts)
    if gather_k:
        R = -(-R // gather_k) * gather_k
        T = R // gather_k
        slot = torch.randperm(R, generator=gen(seed), device="cuda").int()
        slot[used:] = -1
        row = torch.where(slot >= 0, slot // gather_k, 0).long()
        x_rows = T
    else:
        slot, row, x_rows = None, torch.arange(R, device="cuda"), R
    x = normal(seed + 1, x_rows, K + pad, dtype=dtype)[:, :K]
    w = (normal(seed + 2, E, N, K) * K ** -0.5).to(dtype)
    d_y = normal(seed + 3, R, N + pad, dtype=dtype)[:, :N]
    d_y[used:] = math.nan   # rows of no expert are not read
    if not gather_k:
        x[used:] = math.nan
    o = off.tolist()
    u, tiny = UNIT[dtype], TINY[dtype]
    y = ops.expert_matmul(x, w, off, slot=slot, top_k=max(gather_k, 1))
    want, size = product_ref(x, w, o, row)
    close(y, want, want.abs() * u + tiny + size * K * U32, "y")
    d_x = ops.expert_matmul_grad_x(d_y, w, off)
    want, size = product_ref(d_y, w.mT.contiguous(), o, torch.arange(R, device="cuda"))
    close(d_x, want, want.abs() * u + tiny + size * N * U32, "d_x")
    for out in out_dtypes:
        out = out or dtype
        d_w = ops.expert_matmul_grad_w(d_y, x, off, slot=slot, top_k=max(gather_k, 1), dtype=out)
        assert d_w.dtype == out
        for e in range(E):
            a, b = o[e], o[e + 1]
            de, xe = d_y[a:b].double().T.contiguous(), x[row[a:b]].double()
            want, size = de @ xe, de.abs() @ xe.abs()
            close(d_w[e], want, want.abs() * UNIT[out] + TINY[out] + size * max(b - a, 1) * U32, ("d_w", e))


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("counts,extra,N,K,gather", [
    ([1], 0, 1, 1, 0), ([0], 1, 8, 8, 0), ([0, 1, 0], 0, 16, 32, 1), ([3, 0, 5], 2, 17, 33, 2),
    ([128, 129, 127, 1], 0, 128, 64, 0), ([200, 0, 0, 56], 77, 136, 200, 4), ([64] * 5, 3, 72, 1023, 2),
    ([1, 2, 3, 4, 5, 6, 7, 8], 0, 256, 512, 8), ([300, 5, 700], 0, 264, 520, 2), ([16] * 9, 0, 640, 264, 1),
    ([257, 256, 255, 513], 10, 512, 384, 2), ([40, 0, 33], 0, 129, 130, 0)])
def test_products(counts, extra, N, K, gather, dtype):
    say("products", counts, extra, N, K, gather, dtype)
    check_products(counts, extra, N, K, dtype, gather)


@pytest.mark.parametrize("pad", [1, 8])
@pytest.mark.parametrize("N,K", [(128, 256), (130, 250)])
def test_products_strided_rows(N, K, pad):
    say("products strided", N, K, pad)
    check_products([100, 0, 31], 5, N, K, torch.bfloat16, 2, pad=pad)
    check_products([100, 0, 31], 5, N, K, torch.float16, 0, pad=pad)


def test_products_many_experts_and_skew():
    counts = [0] * 300
    for i, c in ((0, 700), (63, 3), (64, 1), (65, 129), (200, 31), (299, 260)):
        counts[i] = c
    check_products(counts, 100, 128, 192, torch.bfloat16, 4)


@pytest.mark.parametrize("rows", [2, 24, 100, 400])
def test_products_by_rows_an_expert(rows):
    """The number of rows an expert decides which kernel runs: a few, some, many, with odd counts among them."""
    say("rows an expert", rows)
    counts = [max(0, rows + (i * 7) % 5 - 2) for i in range(8)]
    check_products(counts, 1, 384, 320, torch.bfloat16, 2, seed=rows)
    check_products(counts, 0, 250, 328, torch.float16, 0, seed=rows)


@pytest.mark.parametrize("shift", [0, 1, 4])
def test_products_unaligned_bases(shift):
    """Tensors that begin 2 and 8 bytes past a vector's boundary."""
    E, N, K, R = 3, 128, 192, 200
    flat = [normal(i, n + 8).to(torch.bfloat16)[shift:shift + n] for i, n in enumerate((R * K, E * N * K, R * N))]
    x, w, d_y = flat[0].view(R, K), flat[1].view(E, N, K), flat[2].view(R, N)
    off = offsets([77, 0, 123])
    for a, b in ((ops.expert_matmul(x, w, off), ops.expert_matmul(x.clone(), w.clone(), off)),
                 (ops.expert_matmul_grad_x(d_y, w, off), ops.expert_matmul_grad_x(d_y.clone(), w.clone(), off)),
                 (ops.expert_matmul_grad_w(d_y, x, off), ops.expert_matmul_grad_w(d_y.clone(), x.clone(), off))):
        close(a, b, b.double().abs() * 2 * UNIT[a.dtype] + 4 * K * U32 * K, "unaligned")
    want, size = product_ref(x, w, off.tolist(), torch.arange(R, device="cuda"))
    close(ops.expert_matmul(x, w, off), want, want.abs() * 2.0 ** -8 + size * K * U32, "y")


def test_products_without_rows():
    x, w = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), normal(1, 4, 32, 64, dtype=torch.bfloat16)
    off = offsets([0] * 4)
    assert ops.expert_matmul(x, w, off).shape == (0, 32)
    assert ops.expert_matmul_grad_x(x.new_empty(0, 32), w, off).shape == (0, 64)
    d_w = ops.expert_matmul_grad_w(x.new_empty(0, 32), x, off)
    assert d_w.shape == (4, 32, 64) and (d_w == 0).all()


def test_products_indices_out_of_range():
    """A slot past x's rows is a row of zeros, an offset past the rows ends there."""
    x, w = normal(1, 4, 64, dtype=torch.bfloat16), normal(2, 2, 32, 64, dtype=torch.bfloat16)
    slot = torch.tensor([0, 9, 3, -5, 1], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 3, 900], dtype=torch.int32, device="cuda")
    y = ops.expert_matmul(x, w, off, slot=slot)
    assert (y[1] == 0).all() and (y[3] == 0).all()
    want = torch.stack([x[0].double() @ w[0].double().T, x[3].double() @ w[0].double().T])
    close(y[[0, 2]], want, want.abs() * 2.0 ** -8 + 1e-3, "y")


def test_products_infinities_stay_in_their_rows():
    x = normal(1, 300, 128, dtype=torch.bfloat16)
    w = normal(2, 2, 64, 128, dtype=torch.bfloat16)
    off = offsets([130, 170])
    clean = ops.expert_matmul(x, w, off)
    x[7, 3], x[131, 0] = math.inf, math.nan
    y = ops.expert_matmul(x, w, off)
    bad = torch.zeros(300, dtype=torch.bool, device="cuda")
    bad[7] = bad[131] = True
    assert torch.equal(y[~bad], clean[~bad]) and not y[bad].isfinite().any()


def test_products_past_32_bits():
    """Weights of more than 2^31 elements, and a gradient as large."""
    E, N, K = 3, 28000, 28672
    say("products past 32 bits")
    w = torch.empty(E, N, K, dtype=torch.bfloat16, device="cuda")
    for e in range(E):
        w[e] = torch.randn(N, K, generator=gen(e), device="cuda") * K ** -0.5
    x, off = normal(5, 6, K, dtype=torch.bfloat16), offsets([1, 0, 5])
    y = ops.expert_matmul(x, w, off)
    want = torch.cat([x[:1].double() @ w[0].double().T.contiguous(), x[1:].double() @ w[2].double().T.contiguous()])
    close(y, want, want.abs() * 2.0 ** -8 + K * U32 * 4, "y")
    d_y = normal(6, 6, N, dtype=torch.bfloat16)
    d_x = ops.expert_matmul_grad_x(d_y, w, off)
    want = torch.cat([d_y[:1].double() @ w[0].double(), d_y[1:].double() @ w[2].double()])
    close(d_x, want, want.abs() * 2.0 ** -8 + N * U32 * 4, "d_x")
    del w
    d_w = ops.expert_matmul_grad_w(d_y, x, off, dtype=torch.bfloat16)
    assert (d_w[1] == 0).all()
    for e, a, b in ((0, 0, 1), (2, 1, 6)):
        for n in (0, N // 2, N - 1):
            want = d_y[a:b, n].double() @ x[a:b].double()
            close(d_w[e, n], want, want.abs() * 2.0 ** -8 + 1e-4, "d_w")


def test_product_gradients_against_differences():
    """The slope of sum(d_y * y) along x and along w, from the forward formula in 64 bits at two points."""
    counts, N, K = [3, 0, 6], 24, 40
    off, R = offsets(counts), 9
    x, w, d_y = normal(1, R, K, dtype=torch.bfloat16), normal(2, 3, N, K, dtype=torch.bfloat16), \
        normal(3, R, N, dtype=torch.bfloat16)
    d_x, d_w = ops.expert_matmul_grad_x(d_y, w, off), ops.expert_matmul_grad_w(d_y, x, off)
    dx, dw, h = normal(4, R, K).double(), normal(5, 3, N, K).double(), 1e-3

    def value(a, b):
        y, _ = product_ref(a, b, off.tolist(), torch.arange(R, device="cuda"))
        return float((d_y.double() * y).sum())

    slope = (value(x.double() + h * dx, w.double()) - value(x.double() - h * dx, w.double())) / (2 * h)
    bound = float((d_x.double().abs() * dx.abs()).sum()) * 2.0 ** -8 + 1e-6
    assert abs(float((d_x.double() * dx).sum()) - slope) < bound
    slope = (value(x.double(), w.double() + h * dw) - value(x.double(), w.double() - h * dw)) / (2 * h)
    assert abs(float((d_w.double() * dw).sum()) - slope) < float((d_w.double().abs() * dw.abs()).sum()) * 1e-6 + 1e-6


def test_products_are_the_same_every_time():
    counts = [500, 3, 0, 700, 41]
    x, w = normal(1, 1244, 512, dtype=torch.bfloat16), normal(2, 5, 384, 512, dtype=torch.bfloat16)
    d_y, off = normal(3, 1244, 384, dtype=torch.bfloat16), offsets(counts)
    first = None
    for _ in range(3):
        got = (ops.expert_matmul(x, w, off), ops.expert_matmul_grad_x(d_y, w, off),
               ops.expert_matmul_grad_w(d_y, x, off))
        if first is not None:
            assert all(torch.equal(a, b) for a, b in zip(first, got))
        first = got


# -------------------------------------------------------------- the optimizer
def bounds(values, bias, least):
    """For blocks of 256: the neighbours below and above each size that 8 bits can hold, in 64 bits."""
    n = values.numel()
    padded = torch.zeros(-(-n // 256) * 256, dtype=torch.float64, device="cuda")
    padded[:n] = values.abs()
    blocks = padded.view(-1, 256)
    big = blocks.amax(1, keepdim=True)
    scale = torch.where(big > 0, torch.frexp(big).exponent.double() - 1, -127.0).clamp_min(least) - bias
    a = blocks * 2.0 ** -scale
    unit = 2.0 ** ((torch.frexp(a).exponent.double() - 1).clamp_min(1 - bias) - 3)
    unit = torch.where(a > 0, unit, 2.0 ** (-2 - bias))
    low = (a / unit).floor() * unit
    return (low * 2.0 ** scale).view(-1)[:n], ((low + unit) * 2.0 ** scale).view(-1)[:n]


def make_optimizer(sizes, bits, copy, grad, seed=0, zero=False, shift=0):
    def cut(total, dtype, fill):
        whole = fill(total + shift).to(dtype)
        return whole[shift:shift + total]
    s = {"param": [cut(n, torch.float32, lambda t: normal(seed + i, t) * 0.1) for i, n in enumerate(sizes)],
         "grad": [cut(n, grad, lambda t: normal(seed + 50 + i, t) * 1e-2) for i, n in enumerate(sizes)],
         "copy": None if copy is None else [cut(n, copy, lambda t: torch.zeros(t, device="cuda")) for n in sizes],
         "decay": [0.1 if i % 2 else 0.0 for i in range(len(sizes))]}
    if bits == 32:
        s["m"] = [torch.zeros(n, device="cuda") if zero else normal(seed + 100 + i, n) * 1e-2
                  for i, n in enumerate(sizes)]
        s["v"] = [torch.zeros(n, device="cuda") if zero else normal(seed + 150 + i, n).square() * 1e-4
                  for i, n in enumerate(sizes)]
        more = {}
    else:
        # any codes but NaN's, and scales of a running step
        def codes(i, n, mark):
            c = torch.randint(0, 256, (n,), generator=gen(seed + i), device="cuda").to(torch.uint8)
            return torch.where(c & 127 == 127, 5, c).to(torch.uint8) if mark == 127 else c.clamp(max=254)
        blocks = [-(-n // 256) for n in sizes]
        z = lambda n, t: torch.zeros(n, dtype=t, device="cuda")   # noqa: E731
        s["m"] = [z(n, torch.uint8) if zero else codes(200 + i, n, 127) for i, n in enumerate(sizes)]
        s["v"] = [z(n, torch.uint8) if zero else codes(250 + i, n, 255) for i, n in enumerate(sizes)]
        more = {"m_exp": [z(b, torch.int8) - (0 if zero else 14) for b in blocks],
                "v_exp": [z(b, torch.int8) - (0 if zero else 29) for b in blocks]}
        s.update(more)
    return s, ops.AdamW(s["param"], s["m"], s["v"], copies=s["copy"], weight_decay=s["decay"], **more)


HYPER = {"lr": 1e-2, "beta1": 0.9, "beta2": 0.99, "eps": 1e-8, "grad_scale": 0.25}
SIZES = [1, 255, 256, 257, 4096, 4097, 3, 10000, 1024]


def step_ref(p, g, m, v, decay, step, lr, beta1, beta2, eps, grad_scale):
    g = g.double() * grad_scale
    a, b = beta1 * m, (1 - beta1) * g
    c, d = beta2 * v, (1 - beta2) * g * g
    m, v = a + b, c + d
    move = lr * (m / (1 - beta1 ** step)) / ((v / (1 - beta2 ** step)).sqrt() + eps)
    return p.double() - move - lr * decay * p.double(), m, v, a.abs() + b.abs(), move.abs()


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("copy", [None, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits, grad, copy, shift):
    say("adamw", bits, grad, copy, shift)
    for zero, step in ((True, 1), (False, 7)):
        s, opt = make_optimizer(SIZES, bits, copy, grad, zero=zero, shift=shift)
        before = [p.clone() for p in s["param"]]
        m0, v0 = ([x.double().clone() for x in part] for part in opt.moments())
        opt.step(s["grad"], step=step, seed=99, **HYPER)
        m1, v1 = opt.moments()
        for i, n in enumerate(SIZES):
            p, m, v, size, move = step_ref(before[i], s["grad"][i], m0[i], v0[i], s["decay"][i], step, **HYPER)
            # m: two products and a sum.  The move: m cancels (size / |m| of its 3 roundings), five roundings more, and
            # the constants'.  The parameter: the move, its decay and the difference.
            m_off = size * 3 * U32
            rel = torch.where(m.abs() > 0, m_off / m.abs().clamp_min(1e-300), 0.0)
            p_off = move * (rel + 12 * U32) + (p.abs() + before[i].double().abs()) * 2 * U32
            close(s["param"][i], p, p_off, ("param", i))
            if copy is not None:
                assert torch.equal(s["copy"][i], s["param"][i].to(copy))
            if bits == 32:
                close(m1[i], m, m_off + 1e-44, ("m", i))
                close(v1[i], v, v * 6 * U32 + 1e-44, ("v", i))
                continue
            # a neighbour of what is stored; the fp32 value may be past the neighbour by its own roundings
            for got, want, off, bias, least in ((m1[i], m, m_off, 7, -119), (v1[i], v, v * 6 * U32, 15, -111)):
                low, high = bounds(want, bias, least)
                size_now = got.double().abs()
                assert bool((size_now >= low - off - low * 1e-6).all()), i
                assert bool((size_now <= high + off + high * 1e-6).all()), i
                assert bool((got.double() * want >= 0).all())
            assert bool((v1[i][v > 0] > 0).all())


def test_adamw_8bit_rounds_without_bias():
    """Steps from one state with many seeds: the mean of the stored moments is the moment, within five deviations of the
    mean of as many roundings (each off by less than a unit, of variance at most a quarter of its square)."""
    n, seeds = 1 << 16, 24
    total_m = total_v = 0
    for seed in range(seeds):
        s, opt = make_optimizer([n], 8, None, torch.float32)
        m0, v0 = ([x.double() for x in part] for part in opt.moments())
        opt.step(s["grad"], step=100, seed=seed * 77777777777, **HYPER)
        m1, v1 = opt.moments()
        total_m, total_v = total_m + m1[0].double(), total_v + v1[0].double()
    _, m, v, _, _ = step_ref(s["param"][0], s["grad"][0], m0[0], v0[0], 0.0, 100, **HYPER)
    for got, want, bias, least in ((total_m / seeds, m.abs(), 7, -119), (total_v / seeds, v, 15, -111)):
        low, high = bounds(want, bias, least)
        unit = high - low
        z = ((got.abs() - want) / unit).sum() / math.sqrt(n * seeds * 0.25) * seeds
        # v's floor above zero adds to elements below the least unit: there are none to speak of here
        assert abs(float(z)) < 5 + 1e-3 * math.sqrt(n), float(z)
        assert float(((got.abs() - want).abs() / unit).max()) < 1.001


def test_adamw_8bit_two_seeds_differ_and_one_repeats():
    out = []
    for seed in (5, 5, 6, 5 + 2**40):
        s, opt = make_optimizer([5000, 300], 8, None, torch.float32)
        opt.step(s["grad"], step=3, seed=seed, **HYPER)
        out.append(torch.cat(s["m"] + s["v"]))
    assert torch.equal(out[0], out[1])
    assert not torch.equal(out[0], out[2]) and not torch.equal(out[0], out[3])


def test_adamw_8bit_decays_and_grows():
    """v follows its mean through many steps, which rounding to nearest would hold where it is."""
    n, steps = 1024, 400
    s, opt = make_optimizer([n], 8, None, torch.float32, zero=True)
    g = [torch.full((n,), 1e-2, device="cuda")]
    hyper = {"lr": 0.0, "beta1": 0.9, "beta2": 0.99, "eps": 1e-8}
    for k in range(steps):
        opt.step(g, step=k + 1, seed=k, **hyper)
    v = opt.moments()[1][0]
    assert abs(float(v.mean()) / (1e-4 * (1 - 0.99 ** steps)) - 1) < 0.05
    g[0].zero_()
    for k in range(steps):
        opt.step(g, step=steps + k + 1, seed=steps + k, **hyper)
    v = opt.moments()[1][0]
    assert 0.5 < float(v.mean()) / (1e-4 * 0.99 ** steps) < 2.0


def test_adamw_infinite_gradients_skip_and_empty():
    for bits in (32, 8):
        s, opt = make_optimizer([600, 0, 40], bits, torch.bfloat16, torch.float32)
        kept = [x.clone() for x in s["param"] + s["m"] + s["v"] + s["copy"]]
        s["grad"][0][3] = math.inf
        flag = torch.ones(1, dtype=torch.int32, device="cuda")
        opt.step(s["grad"], step=2, skip=flag, **HYPER)
        assert all(torch.equal(a, b) for a, b in zip(kept, s["param"] + s["m"] + s["v"] + s["copy"]))
        flag.zero_()
        opt.step(s["grad"], step=2, skip=flag, **HYPER)
        p = s["param"][0]
        assert not p[3].isfinite() and p.isfinite().sum() == 599 and s["param"][2].isfinite().all()
        if bits == 8:
            m, v = opt.moments()
            assert m[0][3].isnan() and v[0][3].isnan() and m[0].isnan().sum() == 1


def test_adamw_many_tensors():
    """More tensors than one launch takes, some empty."""
    sizes = [(i * 37) % 700 for i in range(130)]
    for bits in (32, 8):
        s, opt = make_optimizer(sizes, bits, None, torch.float32)
        before = [p.clone() for p in s["param"]]
        m0, v0 = ([x.double().clone() for x in part] for part in opt.moments())
        opt.step(s["grad"], step=4, seed=1, **HYPER)
        for i in range(len(sizes)):
            p, _, _, size, move = step_ref(before[i], s["grad"][i], m0[i], v0[i], s["decay"][i], 4, **HYPER)
            close(s["param"][i], p, move * 1e-3 + (p.abs() + before[i].double().abs()) * 2 * U32, i)


# ------------------------------------------------------------------ together
def layer_step(state):
    """One layer's step, as the profile runs it: router, products, sum, and back."""
    logits, x, w, g = state
    r = ops.route(logits, 2)
    y = ops.expert_matmul(x, w, r.offset, slot=r.slot, top_k=2)
    out = ops.combine(y, r.place, r.weight)
    d_y, d_weight = ops.combine_backward(g, y, r.slot, r.place, r.weight)
    d_x = ops.combine(ops.expert_matmul_grad_x(d_y, w, r.offset), r.place)
    d_w = ops.expert_matmul_grad_w(d_y, x, r.offset, slot=r.slot, top_k=2)
    return out, d_x, d_w, ops.route_backward(logits, r, d_weight)


def layer_inputs(seed, T=500, E=8, N=256, K=128):
    return [normal(seed, T, E), normal(seed + 1, T, K, dtype=torch.bfloat16),
            (normal(seed + 2, E, N, K) * K ** -0.5).to(torch.bfloat16), normal(seed + 3, T, N, dtype=torch.bfloat16)]


def test_captured_step_replays():
    state = layer_inputs(1)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        layer_step(state)
    side.synchronize()
    s, opt = make_optimizer([4000, 100], 32, torch.bfloat16, torch.float32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer_step(state)
        opt.step(s["grad"], step=5, **HYPER)
    for seed in (20, 30, 40):
        for a, b in zip(state, layer_inputs(seed)):
            a.copy_(b)
        t, other = make_optimizer([4000, 100], 32, torch.bfloat16, torch.float32, seed=seed)
        for name in ("param", "grad", "m", "v"):
            for a, b in zip(s[name], t[name]):
                a.copy_(b)
        want = layer_step(state)
        other.step(t["grad"], step=5, **HYPER)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), seed
        for name in ("param", "m", "v", "copy"):
            assert all(torch.equal(a, b) for a, b in zip(s[name], t[name])), (seed, name)


def test_on_another_stream():
    state = layer_inputs(3)
    want = layer_step(state)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer_step(state)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------------- refusals
def refused(f, *a, **k):
    with pytest.raises(ValueError):
        f(*a, **k)


def test_refusals():
    x, w, off = normal(1, 8, 16, dtype=torch.bfloat16), normal(2, 2, 4, 16, dtype=torch.bfloat16), offsets([3, 5])
    refused(ops.expert_matmul, x.float(), w, off)
    refused(ops.expert_matmul, x, w.half(), off)
    refused(ops.expert_matmul, x, w[:1], off)
    refused(ops.expert_matmul, x, w, off.long())
    refused(ops.expert_matmul, x.cpu(), w, off)
    refused(ops.expert_matmul, x.T, w, off)
    refused(ops.expert_matmul, x, w.mT, off)
    refused(ops.expert_matmul, x[:, :8], w, off)
    refused(ops.expert_matmul, x, w, off, slot=torch.zeros(8, device="cuda"))
    with pytest.raises(ops.binding.HapmoeError):
        ops.expert_matmul(x, w, off, slot=torch.zeros(8, dtype=torch.int32, device="cuda"), top_k=0)
    refused(ops.expert_matmul_grad_x, x, w, off)
    refused(ops.expert_matmul_grad_w, x, x[:7], off)
    refused(ops.expert_matmul_grad_w, x, x, off, dtype=torch.float16)
    logits = normal(3, 5, 8)
    refused(ops.route, logits, 9)
    refused(ops.route, logits, 0)
    refused(ops.route, logits.double(), 2)
    refused(ops.route, logits[0], 2)
    refused(ops.route, logits, 2, keep=torch.ones(4, dtype=torch.bool, device="cuda"))
    refused(ops.route, logits, 2, out=ops.Routing(4, 8, 2))
    refused(ops.route, torch.zeros(2, 1025, device="cuda"), 2)
    r = ops.route(logits, 2)
    refused(ops.route_backward, logits, r, torch.zeros(5, 3, device="cuda"))
    refused(ops.route_backward, logits, r, torch.zeros(5, 2, device="cuda", dtype=torch.bfloat16))
    y = normal(4, 10, 6)
    refused(ops.combine, y.T, r.place)
    refused(ops.combine, y, r.place.long())
    refused(ops.combine, y, r.place, r.weight[:4])
    refused(ops.combine_backward, y[:5], y[:9], r.slot, r.place, r.weight)
    refused(ops.combine_backward, y[:4], y, r.slot, r.place, r.weight)
    p = [torch.zeros(300, device="cuda")]
    z8, e8 = torch.zeros(300, dtype=torch.uint8, device="cuda"), torch.zeros(2, dtype=torch.int8, device="cuda")
    refused(ops.AdamW, p, p, [])
    refused(ops.AdamW, p, [z8], [z8])
    refused(ops.AdamW, p, [z8], [z8], m_exp=[e8])
    refused(ops.AdamW, p, [z8], [z8], m_exp=[e8[:1]], v_exp=[e8])
    refused(ops.AdamW, p, p, p, copies=[torch.zeros(300, device="cuda")])
    refused(ops.AdamW, p, p, p, weight_decay=-1.0)
    refused(ops.AdamW, [p[0].bfloat16()], p, p)
    opt = ops.AdamW(p, [p[0].clone()], [p[0].clone()])
    refused(opt.step, [], lr=1e-3, step=1)
    refused(opt.step, [p[0][:299]], lr=1e-3, step=1)
    refused(opt.step, [p[0].double()], lr=1e-3, step=1)
    for bad in ({"lr": -1.0, "step": 1}, {"lr": 1e-3, "step": 0}, {"lr": 1e-3, "step": 1, "beta1": 1.0},
                {"lr": 1e-3, "step": 1, "eps": math.nan}):
        with pytest.raises(ops.binding.HapmoeError):
            opt.step(p, **bad)


# ------------------------------------------------- more workgroups than one axis of a launch holds
def test_route_past_one_axis_of_workgroups():
    """2^28 tokens: the gradient takes 2^24 workgroups of 256 threads."""
    T = (1 << 28) + 5
    say("route", T)
    logits = torch.zeros(T, 2, dtype=torch.bfloat16, device="cuda")
    second = torch.arange(T, device="cuda") % 3 == 0
    logits[:, 1] = torch.where(second, 1.0, -1.0)
    r = ops.route(logits, 1, renormalize=False)
    assert torch.equal(r.expert[:, 0] == 1, second)
    n = int(second.sum())
    assert r.count.tolist() == [T - n, n] and r.offset.tolist() == [0, T - n, T]
    assert torch.equal(torch.sort(r.place[:, 0][second]).values, torch.arange(T - n, T, device="cuda", dtype=torch.int32))
    assert torch.equal(r.slot[r.place[:, 0].long()], torch.arange(T, device="cuda", dtype=torch.int32))
    d = ops.route_backward(logits, r, torch.ones_like(r.weight), renormalize=False)
    p = 1 / (1 + math.exp(-1.0))
    unit = p * (1 - p) * 2.0 ** -8
    del logits
    for e in (0, 1):
        want = torch.where(second == (e == 1), p * (1 - p), -p * (1 - p))
        assert (d[:, e].float() - want.float()).abs().max() <= 2 * unit


@pytest.mark.parametrize("hidden", [3, 8])
def test_combine_past_one_axis_of_workgroups(hidden):
    """2^24 tokens are 2^24 workgroups of 256 threads; of the gradient, 2^26 rows."""
    T = (1 << 24) + 7
    say("combine", T, hidden)
    y = torch.arange(T, device="cuda").remainder(251).to(torch.bfloat16)[:, None].expand(T, hidden).contiguous()
    place = torch.arange(T - 1, -1, -1, device="cuda", dtype=torch.int32)[:, None].contiguous()
    assert torch.equal(ops.combine(y, place), y.flip(0))
    T = (1 << 26) + 9
    d_out = torch.arange(T, device="cuda").remainder(127).to(torch.bfloat16)[:, None].expand(T, hidden).contiguous()
    y = torch.ones_like(d_out)
    place = torch.arange(T - 1, -1, -1, device="cuda", dtype=torch.int32)
    d_y, d_weight = ops.combine_backward(d_out, y, place, place[:, None].contiguous(),
                                         torch.full((T, 1), 2.0, device="cuda"))
    assert torch.equal(d_y, (d_out * 2).flip(0))
    assert torch.equal(d_weight[:, 0], d_out[:, 0].float() * hidden)


def test_products_past_one_axis_of_workgroups():
    """2^30 rows of one column are 2^24 tiles of 64 rows."""
    R = (1 << 30) + 100
    say("products", R)
    x = torch.arange(R, device="cuda", dtype=torch.int32).remainder(127).to(torch.bfloat16)[:, None]
    w = torch.full((2, 1, 1), 2.0, dtype=torch.bfloat16, device="cuda")
    w[1] = 0.5
    cut = (1 << 30) - 5
    off = torch.tensor([0, cut, R], dtype=torch.int32, device="cuda")
    for y in (ops.expert_matmul(x, w, off), ops.expert_matmul_grad_x(x, w, off)):
        assert torch.equal(y[:cut], x[:cut] * 2) and torch.equal(y[cut:], x[cut:] * 0.5)


# -------------------------------------------------- products large enough for the larger tiles
@pytest.mark.parametrize("gather", [0, 2])
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("counts,N,K", [
    # rows that end in the first and in the second half of a tile, one row, none; a last tile of summands that ends early
    ([1000, 257, 384, 0, 129, 1, 1920, 128, 385], 1416, 1544),
    ([4608, 64, 256, 320, 40], 1408, 1608),
    # some 150 rows an expert
    ([150 + (i * 37) % 41 - 20 for i in range(28)] + [0, 1, 17, 300], 1416, 1528),
    ([150 + (i * 29) % 37 - 18 for i in range(32)], 520, 4104)])
def test_products_larger_tiles(counts, N, K, dtype, gather):
    say("larger tiles", len(counts), N, K, dtype, gather)
    check_products(counts, 6 if gather == 0 else 0, N, K, dtype, gather)


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("E,k", [(128, 8), (129, 5), (256, 8), (300, 32), (512, 17), (700, 8), (1024, 32)])
def test_route_ties_and_closed_experts_of_wide_routers(E, k, renormalize):
    """Many equal logits, of neighbouring lanes and within one; infinities, NaN, rows all closed or with fewer open experts
    than choices."""
    say("route ties", E, k, renormalize)
    T = 70
    logits = torch.randint(-2, 3, (T, E), generator=gen(E), device="cuda").float()
    logits[torch.rand((T, E), generator=gen(1), device="cuda") < 0.1] = -math.inf
    logits[torch.rand((T, E), generator=gen(2), device="cuda") < 0.05] = math.nan
    logits[0], logits[1], logits[2], logits[3] = 0.0, -math.inf, math.nan, torch.finfo(torch.float32).min
    logits[4] = -math.inf
    logits[4, E - 1], logits[4, E // 2] = 1.0, 2.0
    logits[5, 3], logits[5, E - 2] = math.inf, math.inf
    logits[6] = torch.where(torch.arange(E, device="cuda") % 2 == 0, -0.0, 0.0)
    logits[7] = -1.0
    logits[7, E - 9:] = 1.0
    for n in (9, T):   # one workgroup, several
        x = logits[:n]
        for dtype in (torch.float32, torch.bfloat16):
            y = x.to(dtype)
            r = ops.route(y, k, renormalize=renormalize)
            ref = route_ref(y, k, None, renormalize)
            check_routing(r, ref, E)
            d = ops.route_backward(y, r, normal(3, n, k), renormalize=renormalize)
            assert d.isfinite().all() and (d[y.isnan() | (y == -math.inf)] == 0).all()
