"""The operators around a mixture-of-experts layer -- balanced router, layer norm, embedding, dropout -- against their
formulas in 64 bits, on the GPU.

Bounds follow from the arithmetic: UNIT(type) bounds the rounding of a result, U32 = 2^-24 that of an fp32 operation, and a
sum whose elements each pass through at most D additions is off by at most D U32 times the sum of the sizes.
"""
import math

import numpy as np
import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_operators import TINY, U32, UNIT, close, gen, normal, say   # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
inf, nan = math.inf, math.nan


# ------------------------------------------------------------------ the router
def balanced_ref(logits, k, bias=None, scores="sigmoid", groups=1, top_groups=None, group_best=2, keep=None,
                 renormalize=True, scale=1.0):
    """The definition in 64 bits, on the host: choices, weights and the rows' order."""
    x = logits.double().cpu().numpy()
    T, E = x.shape
    top_groups = groups if top_groups is None else top_groups
    shut = ~(x > -np.inf)
    if keep is not None:
        shut |= ~keep.cpu().numpy()[:, None]
    with np.errstate(all="ignore"):
        if scores == "sigmoid":
            s = np.where(x >= 0, 1 / (1 + np.exp(-x)), np.exp(np.minimum(x, 0)) / (1 + np.exp(np.minimum(x, 0))))
        else:
            y = np.where(shut, -np.inf, x)
            top = y.max(1, keepdims=True)
            e = np.where(y == top, 1.0, np.exp(y - top))
            s = e / e.sum(1, keepdims=True)
        s = np.where(shut, 0.0, s)
        c = s + (0.0 if bias is None else bias.double().cpu().numpy())
    c = np.where(shut | ~(c > -np.inf), -np.inf, c)
    if top_groups < groups:
        each = E // groups
        best = -np.sort(-c.reshape(T, groups, each), axis=2)[:, :, :group_best]
        score = best[:, :, 0] + (np.where(best[:, :, 1:] > -np.inf, best[:, :, 1:], 0.0)).sum(2)
        rank = np.argsort(np.argsort(-score, axis=1, kind="stable"), axis=1, kind="stable")
        c[np.repeat(rank >= top_groups, each, axis=1)] = -np.inf
    by = c if bias is not None else np.where(c > -np.inf, x, -np.inf)
    expert = np.argsort(-by, axis=1, kind="stable")[:, :k]
    live = np.take_along_axis(c, expert, 1) > -np.inf
    chosen = np.take_along_axis(s, expert, 1) * live
    weight = chosen * scale
    if renormalize:
        with np.errstate(all="ignore"):
            weight = np.where(live, weight / chosen.sum(1, keepdims=True), 0.0)
    flat = np.where(live, expert, -1).reshape(-1)
    rows = np.argsort(np.where(flat < 0, E, flat), kind="stable")[:int((flat >= 0).sum())]
    place, slot = np.full(T * k, -1), np.full(T * k, -1)
    place[rows], slot[:len(rows)] = np.arange(len(rows)), rows
    count = np.bincount(flat[flat >= 0], minlength=E)
    out = {"expert": flat.reshape(T, k), "count": count, "offset": np.concatenate([[0], np.cumsum(count)]),
           "slot": slot, "place": place.reshape(T, k)}
    return {n: torch.from_numpy(v.astype(np.int64)) for n, v in out.items()} | {
        "weight": torch.from_numpy(weight), "scores": torch.from_numpy(s)}


def check_balanced(r, ref, E, span=40.0):
    for name in ("expert", "count", "offset", "slot", "place"):
        assert torch.equal(getattr(r, name).cpu().long(), ref[name]), name
    # an exponent's argument is rounded once (span U32 of the value) and there are two, sums of at most E, a quotient
    close(r.weight.cpu(), ref["weight"], ref["weight"] * (E + 2 * span + 32) * U32 + 1e-36, "weight")


ROUTES = [   # tokens, experts, top_k, groups, top_groups, group_best, scores, bias, type
    (1, 1, 1, 1, 1, 1, "sigmoid", True, F32), (1, 8, 8, 1, 1, 1, "softmax", False, F32),
    (4, 256, 8, 8, 4, 2, "sigmoid", True, F32), (64, 64, 6, 8, 3, 1, "softmax", True, BF16),
    (65, 60, 6, 5, 2, 2, "sigmoid", False, F16), (129, 100, 17, 1, 1, 2, "sigmoid", True, F32),
    (257, 512, 32, 16, 16, 2, "sigmoid", True, F16), (70, 1024, 32, 64, 5, 2, "softmax", True, F32),
    (33, 1000, 3, 8, 1, 2, "sigmoid", True, BF16), (2049, 16, 2, 16, 7, 2, "softmax", False, F32),
    (300, 256, 8, 8, 4, 2, "softmax", True, BF16), (300, 256, 8, 4, 1, 1, "sigmoid", False, BF16),
    (777, 128, 8, 2, 1, 2, "sigmoid", True, F32), (100, 63, 5, 63, 9, 2, "sigmoid", True, F32),
    (40, 192, 4, 8, 3, 2, "sigmoid", True, F32), (50, 96, 8, 3, 2, 2, "softmax", True, F16)]


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("T,E,k,G,TG,best,scores,biased,dtype", ROUTES)
def test_route_balanced(T, E, k, G, TG, best, scores, biased, dtype, renormalize):
    say("route_balanced", T, E, k, G, TG, best, scores, biased, dtype, renormalize)
    logits = (normal(T + E, T, E) * 3).to(dtype)
    logits[torch.rand((T, E), generator=gen(2), device="cuda") < 0.05] = -inf
    bias = normal(5, E) * 0.2 if biased else None
    keep = torch.rand(T, generator=gen(7), device="cuda") < 0.8
    how = {"bias": bias, "scores": scores, "groups": G, "top_groups": TG, "group_best": best, "scale": 2.5,
           "renormalize": renormalize}
    for kp in (None, keep):
        r = ops.route_balanced(logits, k, keep=kp, **how)
        check_balanced(r, balanced_ref(logits, k, keep=kp, **how), E)


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T,E,k,G,TG", [(40000, 64, 8, 1, 1), (32768, 256, 8, 8, 4), (5000, 1024, 4, 32, 6)])
def test_route_balanced_many_tokens(T, E, k, G, TG, scores):
    say("route_balanced", T, E, k, scores)
    logits, bias = normal(9, T, E), normal(10, E) * 0.1
    how = {"bias": bias, "scores": scores, "groups": G, "top_groups": TG}
    check_balanced(ops.route_balanced(logits, k, **how), balanced_ref(logits, k, **how), E)


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T,E,k,G,TG", [(50, 64, 8, 1, 1), (3000, 256, 8, 8, 4), (500, 60, 4, 6, 2)])
def test_route_balanced_sums_nearer_than_fp32(T, E, k, G, TG, scores):
    """Biases that bring every expert of the first token to nearly the same sum: the other tokens have its logits with
    changes of a few units in the last place, so that many sums lie within 2^-24 of each other."""
    logits = normal(3, 1, E).repeat(T, 1)
    x = logits[0].double().cpu().numpy()
    s = 1 / (1 + np.exp(-x)) if scores == "sigmoid" else np.exp(x) / np.exp(x).sum()
    bias = torch.from_numpy((1.5 - s).astype(np.float32)).cuda()
    change = torch.randint(-3, 4, (T, E), generator=gen(4), device="cuda", dtype=torch.int32)
    logits = (logits.view(torch.int32) + change).view(F32)
    how = {"bias": bias, "scores": scores, "groups": G, "top_groups": TG}
    ref = balanced_ref(logits, k, **how)
    c = ref["scores"] + bias.double().cpu()
    assert float((c.max(1).values - c.min(1).values).max()) < 64 * 2.0 ** -24   # as meant
    check_balanced(ops.route_balanced(logits, k, **how), ref, E)


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T,E,k,G,TG", [(500, 16, 3, 4, 2), (500, 256, 8, 8, 4), (300, 60, 4, 6, 2), (200, 512, 8, 16, 3)])
def test_route_balanced_sums_below_zero_and_closed_groups(T, E, k, G, TG, scores):
    """Biases that leave every sum below zero, groups closed to a token, lanes without experts beside those with."""
    logits = normal(1, T, E)
    logits.view(T, G, E // G)[torch.rand((T, G), generator=gen(2), device="cuda") < 0.3] = -inf
    how = {"bias": normal(3, E) * 0.3 - 4, "scores": scores, "groups": G, "top_groups": TG}
    check_balanced(ops.route_balanced(logits, k, **how), balanced_ref(logits, k, **how), E)


@pytest.mark.parametrize("m", [1, 2, 4, 8])
def test_route_balanced_equal_groups(m):
    """Groups of one to eight lanes whose scores are the same: the lowest stay."""
    E, G = 64, 16 // m
    logits = normal(5, 1, E // G).repeat(70, G)
    for TG in range(1, G + 1):
        how = {"bias": normal(6, E // G).repeat(G) * 0.1, "groups": G, "top_groups": TG}
        check_balanced(ops.route_balanced(logits, 4, **how), balanced_ref(logits, 4, **how), E)


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("G,TG", [(1, 1), (3, 2), (6, 1)])
def test_route_balanced_ties_masks_and_infinities(scores, G, TG, renormalize):
    low = torch.finfo(F32).min
    rows = [[0.0] * 6, [1, 1, 2, 2, 1, 1], [-inf] * 6, [nan] * 6, [nan, 3, -inf, 3, nan, -inf], [low] * 6,
            [low, 0, low, low, low, low], [inf, 0, inf, 1, nan, -inf], [-0.0, 0.0, -0.0, 0.0, -1, -1],
            [inf, -inf, -inf, -inf, -inf, -inf], [5, -inf, -inf, -inf, -inf, -inf], [-200.0, -201, -202, -203, -204, -205],
            [30.0, 31, 32, 33, 34, 35]]
    logits = torch.tensor(rows * 8, device="cuda")   # 104 tokens: more than one workgroup
    biases = [None, torch.zeros(6, device="cuda"), torch.tensor([0.0, -inf, nan, 0.5, -2.0, inf], device="cuda")]
    for n in (len(rows), len(rows) * 8):
        for bias in biases:
            how = {"scores": scores, "groups": G, "top_groups": TG, "renormalize": renormalize}
            r = ops.route_balanced(logits[:n], 3, bias=bias, **how)
            ref = balanced_ref(logits[:n], 3, bias=bias, **how)
            for name in ("expert", "count", "offset", "slot", "place"):
                assert torch.equal(getattr(r, name).cpu().long(), ref[name]), (name, bias)
            # far logits: exponents up to 205 (200 where the difference is cut) and fp32's range
            fine = ref["weight"].isfinite()
            assert r.weight.isfinite().all()
            close(r.weight.cpu()[fine], ref["weight"][fine], ref["weight"][fine] * 500 * U32 + 1e-36, "weight")
            d = ops.route_balanced_backward(logits[:n], r, normal(3, n, 3), scores=scores, renormalize=renormalize)
            assert d.isfinite().all()
            assert (d[logits[:n].isnan() | (logits[:n] == -inf)] == 0).all()


def test_route_balanced_without_bias_or_groups_is_route():
    """By softmax without bias, groups or scale: route's choices, and its weights but for the last bits."""
    logits = normal(1, 300, 64) * 2
    for renormalize in (False, True):
        a = ops.route(logits, 6, renormalize=renormalize)
        b = ops.route_balanced(logits, 6, scores="softmax", renormalize=renormalize)
        assert torch.equal(a.expert, b.expert) and torch.equal(a.slot, b.slot)
        close(b.weight, a.weight, a.weight.double() * 2 * (64 + 48) * U32)


def test_route_balanced_strided_rows_kept_buffers_no_tokens():
    wide, bias = normal(1, 300, 70), normal(2, 64) * 0.1
    r = ops.Routing(300, 64, 4, "cuda")
    g = normal(2, 300, 4)
    for lo in (0, 3):
        logits = wide[:, lo:lo + 64]
        how = {"groups": 4, "top_groups": 2}
        assert ops.route_balanced(logits, 4, bias=bias, out=r, **how) is r
        check_balanced(r, balanced_ref(logits, 4, bias=bias, **how), 64)
        for scores in ("sigmoid", "softmax"):
            for renormalize in (True, False):
                q = ops.route_balanced(logits, 4, bias=bias, scores=scores, renormalize=renormalize, **how)
                a = ops.route_balanced_backward(logits, q, g, scores=scores, renormalize=renormalize)
                b = ops.route_balanced_backward(logits.contiguous(), q, g, scores=scores, renormalize=renormalize)
                assert torch.equal(a, b)
    none = torch.empty(0, 8, device="cuda")
    r = ops.route_balanced(none, 2, groups=2, top_groups=1)
    assert r.count.tolist() == [0] * 8 and r.offset.tolist() == [0] * 9
    assert ops.route_balanced_backward(none, r, torch.empty(0, 2, device="cuda")).shape == (0, 8)


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T,E,k,dtype", [(1, 8, 2, F32), (37, 60, 6, F32), (100, 256, 8, BF16), (19, 512, 32, F16),
                                         (5, 1024, 1, F32)])
def test_route_balanced_backward(T, E, k, dtype, scores, renormalize):
    say("route_balanced_backward", T, E, k, dtype, scores, renormalize)
    logits = (normal(T, T, E) * 2).to(dtype)
    logits[torch.rand((T, E), generator=gen(3), device="cuda") < 0.2] = -inf
    keep = torch.rand(T, generator=gen(4), device="cuda") < 0.8
    bias, g = normal(6, E) * 0.2, normal(5, T, k)
    how = {"scores": scores, "keep": keep, "renormalize": renormalize, "scale": 2.5}
    r = ops.route_balanced(logits, k, bias=bias, **how)
    d = ops.route_balanced_backward(logits, r, g, **how)
    ref = balanced_ref(logits, k, bias=bias, **how)
    ok = ref["expert"] >= 0
    index, s = ref["expert"].clamp_min(0), ref["scores"]
    gd = torch.where(ok, g.double().cpu(), 0.0) * 2.5
    chosen = torch.where(ok, s.gather(1, index), 0.0)
    if renormalize:
        total = torch.where(chosen.sum(1, keepdim=True) > 0, chosen.sum(1, keepdim=True), 1.0)
        d_s = torch.where(ok, (gd - (gd * chosen).sum(1, keepdim=True) / total) / total, 0.0)
    else:
        total, d_s = torch.ones(T, 1, dtype=torch.float64), gd
    whole = torch.zeros(T, E, dtype=torch.float64).scatter_add_(1, index, d_s)
    want = whole * s * (1 - s) if scores == "sigmoid" else s * (whole - (whole * s).sum(1, keepdim=True))
    # of the terms before they cancel: a weight's share times twice the largest gradient
    size = s / total * gd.abs().amax(1, keepdim=True) * 2
    close(d.cpu(), want, want.abs() * UNIT[dtype] + TINY[dtype] + size * (E + k + 96) * U32, "d_logits")


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
def test_route_balanced_gradient_against_differences(scores, renormalize):
    """d(sum g w)/d logits by central differences of the formula in 64 bits, the choice held."""
    T, E, k, h = 3, 10, 3, 1e-5
    logits = torch.stack([torch.randperm(E, generator=gen(t), device="cuda").float() * 0.3 for t in range(T)])
    g, bias = normal(6, T, k), normal(7, E) * 0.1
    how = {"scores": scores, "renormalize": renormalize, "scale": 1.5}
    r = ops.route_balanced(logits, k, bias=bias, groups=5, top_groups=3, **how)
    d = ops.route_balanced_backward(logits, r, g, **how).cpu().double()
    index = r.expert.long().cpu()

    def value(x):
        p = (torch.sigmoid(x) if scores == "sigmoid" else torch.softmax(x, 1)).gather(1, index)
        return float((g.double().cpu() * 1.5 * (p / p.sum(1, keepdim=True) if renormalize else p)).sum())

    x = logits.double().cpu()
    for t in range(T):
        for e in range(E):
            step = torch.zeros_like(x)
            step[t, e] = h
            slope = (value(x + step) - value(x - step)) / (2 * h)
            assert abs(float(d[t, e]) - slope) < 1e-6   # h^2 / 6 of the third derivative, 2^-52 / h, fp32 of the kernel


# ------------------------------------------------------------------ layer norm
def norm_ref(x, weight, bias, eps, center, d_y=None, add=None):
    """The formulas in 64 bits and, of every result, the bound of an fp32 computation before its last rounding."""
    x, w = x.double(), weight.double()
    R, H = x.shape
    D = H / 64 + 16   # additions that an element passes through: 64 lanes at least share a row
    mean = x.mean(1, keepdim=True) if center else x.new_zeros(R, 1)
    e_mean = (D + 2) * U32 * x.abs().mean(1, keepdim=True) if center else x.new_zeros(R, 1)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    # the squares are about a mean that is off: e_mean^2 more, and each difference is rounded
    e_rstd = ((D + 6) * U32 + (e_mean.square() + 4 * U32 * e_mean * var.sqrt()) / (var + eps)) / 2 + 4 * U32   # relative
    hat = (x - mean) * rstd
    e_hat = e_mean * rstd + hat.abs() * (e_rstd + 4 * U32)
    y = hat * w + (0 if bias is None else bias.double())
    e_y = w.abs() * e_hat + 4 * U32 * ((hat * w).abs() + y.abs())
    out = {"y": (y, e_y), "mean": (mean[:, 0], e_mean[:, 0]), "rstd": (rstd[:, 0], (rstd * e_rstd)[:, 0])}
    if d_y is not None:
        d_y = d_y.double()
        g = d_y * w
        a = g.mean(1, keepdim=True) if center else 0.0 * mean
        e_a = (D + 3) * U32 * g.abs().mean(1, keepdim=True)
        b = (g * hat).mean(1, keepdim=True)
        e_b = (D + 4) * U32 * (g * hat).abs().mean(1, keepdim=True) + (g.abs() * e_hat).mean(1, keepdim=True)
        d = rstd * (g - a - hat * b)
        e_d = rstd * (6 * U32 * (g.abs() + a.abs() + (hat * b).abs()) + e_a + e_hat * (b.abs() + e_b) + hat.abs() * e_b) \
            + d.abs() * (e_rstd + 4 * U32)
        d_x = d if add is None else d + add.double()
        out["d_x"] = d_x, e_d + 2 * U32 * d_x.abs()
        out["d_weight"] = (d_y * hat).sum(0), (d_y.abs() * e_hat).sum(0) + (R + 4) * U32 * (d_y * hat).abs().sum(0)
        out["d_bias"] = d_y.sum(0), (R + 2) * U32 * d_y.abs().sum(0)
    return out


def check_norm(x, weight, bias, eps, center, d_y=None, add=None):
    y, mean, rstd = ops.layer_norm(x, weight, bias, eps=eps, center=center)
    got = {"y": y, "rstd": rstd}
    if center:
        got["mean"] = mean
    else:
        assert mean is None
    if d_y is not None:
        got["d_x"], got["d_weight"], got["d_bias"] = ops.layer_norm_backward(d_y, x, weight, mean, rstd, add=add)
    ref = norm_ref(x, weight, bias, eps, center, d_y, add)
    for name, t in got.items():
        want, bound = ref[name]
        assert t.shape == want.shape and t.is_contiguous()
        assert t.dtype == (x.dtype if name in ("y", "d_x") else F32)
        last = want.abs() * UNIT[t.dtype] + TINY[t.dtype] if name in ("y", "d_x") else 1e-38
        close(t, want, bound + last, name)
    return got


NORMS = [(1, 1), (1, 7), (3, 64), (16, 7168), (17, 1023), (129, 1024), (40, 4096), (5, 8192), (9, 16384), (3, 20000),
         (700, 72), (2, 100001), (1030, 520)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("R,H", NORMS)
def test_layer_norm_and_backward(R, H, dtype):
    for center in (True, False):
        for wide in (True, False):
            say("layer_norm", R, H, dtype, center, wide)
            wt = F32 if wide else dtype
            x = (normal(R + H, R, H) + normal(1, R, 1)).to(dtype)
            weight, bias = (1 + 0.2 * normal(2, H)).to(wt), (0.2 * normal(3, H)).to(wt) if wide else None
            d_y = normal(4, R, H, dtype=dtype)
            add = normal(5, R, H, dtype=dtype) if center else None
            got = check_norm(x, weight, bias, 1e-5, center, d_y, add)
            mean, rstd = got.get("mean"), got["rstd"]
            d_x, d_weight, none = ops.layer_norm_backward(d_y, x, weight, mean, rstd, add=add, bias=False)
            assert none is None
            for a, b in ((d_x, got["d_x"]), (d_weight, got["d_weight"])):
                assert torch.equal(a, b)   # a fixed order: the same bits again


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H", [1024, 1000, 17])
def test_layer_norm_strided_rows(H, dtype):
    """Rows out of wider matrices, at offsets of whole vectors and of single elements."""
    for lo, gap in ((0, 8), (8, 24), (1, 3), (3, 64)):
        wide = [normal(i, 37, H + gap + lo, dtype=dtype)[:, lo:lo + H] for i in range(3)]
        weight = normal(5, H + 1, dtype=dtype)[lo % 2:lo % 2 + H]
        a = check_norm(wide[0], weight, weight, 1e-6, True, wide[1], wide[2])
        b = check_norm(*(t.contiguous() for t in (wide[0], weight.clone(), weight.clone())), 1e-6, True,
                       wide[1].contiguous(), wide[2].contiguous())
        assert a.keys() == b.keys()


@pytest.mark.parametrize("center", [True, False])
def test_layer_norm_far_rows_equal_elements_and_zeros(center):
    H = 1000
    x = torch.cat([normal(1, 4, H) + 3000, torch.full((3, H), 2.5, device="cuda"), torch.zeros(3, H, device="cuda"),
                   normal(2, 2, H) * 1e-18, normal(3, 2, H) * 1e15])
    w, d_y = normal(4, H), normal(5, len(x), H)
    check_norm(x, w, w, 1e-5, center)
    got = check_norm(x[:10], w, w, 1e-5, center, d_y[:10])
    assert (got["y"][7:10] == w).all()
    if not center:
        return
    # equal elements of a mean that fp32 holds exactly: xhat is 0
    assert (got["y"][4:7] == w).all()


def test_layer_norm_bad_rows_stay_alone():
    """A NaN or an infinity spoils its own row and the weight's gradient, no other row."""
    x, w, d_y = normal(1, 40, 513), normal(2, 513), normal(3, 40, 513)
    want, m0, r0 = ops.layer_norm(x, w)
    d_want = ops.layer_norm_backward(d_y, x, w, m0, r0)[0]
    x[7, 100], x[30, 0] = nan, inf
    y, mean, rstd = ops.layer_norm(x, w)
    d_x, d_w, _ = ops.layer_norm_backward(d_y, x, w, mean, rstd)
    others = torch.tensor([i for i in range(40) if i not in (7, 30)], device="cuda")
    assert torch.equal(y[others], want[others]) and torch.equal(d_x[others], d_want[others])
    assert y[7].isnan().all() and y[30].isnan().any() and d_w.isnan().any()


def test_layer_norm_without_rows():
    x, w = torch.empty(0, 64, device="cuda"), normal(1, 64)
    y, mean, rstd = ops.layer_norm(x, w)
    assert y.shape == (0, 64) and mean.shape == rstd.shape == (0,)
    d_x, d_w, d_b = ops.layer_norm_backward(x, x, w, mean, rstd)
    assert d_x.shape == (0, 64) and (d_w == 0).all() and (d_b == 0).all()


@pytest.mark.parametrize("center", [True, False])
def test_layer_norm_gradient_against_differences(center):
    R, H, h = 2, 9, 1e-6
    x, w, b, d_y = normal(1, R, H), normal(2, H), normal(3, H), normal(4, R, H)
    y, mean, rstd = ops.layer_norm(x, w, b, eps=1e-3, center=center)
    got = [t.double().cpu() for t in ops.layer_norm_backward(d_y, x, w, mean, rstd)]
    leaves = [t.double().cpu() for t in (x, w, b)]

    def value(x, w, b):
        dev = x - x.mean(1, keepdim=True) if center else x
        return float((d_y.double().cpu() * (dev / (dev.square().mean(1, keepdim=True) + 1e-3).sqrt() * w + b)).sum())

    for n, leaf in enumerate(leaves):
        for i in range(leaf.numel()):
            step = [torch.zeros_like(t) for t in leaves]
            step[n].view(-1)[i] = h
            slope = (value(*(a + s for a, s in zip(leaves, step))) - value(*(a - s for a, s in zip(leaves, step)))) / (2 * h)
            assert abs(float(got[n].view(-1)[i]) - slope) < 2e-5   # fp32 of the kernel at sizes of some 10


# ------------------------------------------------------------------- embedding
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,V,H", [(1, 1, 1), (3, 10, 7), (16, 1000, 7168), (100, 513, 1023), (64, 33, 2056)])
def test_embed(T, V, H, dtype):
    say("embed", T, V, H, dtype)
    token = torch.randint(-2, V + 2, (T,), generator=gen(1), device="cuda")
    token[0] = V - 1
    wide = normal(2, V, H + 5, dtype=dtype)
    real = (token >= 0) & (token < V)
    for table in (wide[:, :H], wide[:, 2:H + 2].contiguous()):
        want = torch.where(real[:, None], table.double()[token.clamp(0, V - 1)] * 0.37, 0.0)
        for t in (token, token.int()):
            out = ops.embed(t, table, scale=0.37)
            close(out, want, want.abs() * (UNIT[dtype] + 3 * U32) + TINY[dtype])
    if T > 2:
        token = torch.tensor([2**32, -1, -2**63 + 1, 2**31], device="cuda")
        assert (ops.embed(token, table) == 0).all()


def embed_grad_ref(d_out, token, V, scale, into=None):
    """The sums in 64 bits, and their bound: a row's number of additions, two more for scale and into."""
    real = (token >= 0) & (token < V)
    d, at = d_out.double()[real] * scale, token[real].long()
    want = torch.zeros(V, d_out.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, d)
    size = torch.zeros_like(want).index_add_(0, at, d.abs())
    n = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, at, torch.ones_like(at).double())
    if into is not None:
        want, size = want + into.double(), size + into.double().abs()
    return want, size * (n[:, None] + 4) * U32 * (n[:, None] > 0), n


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,V,H,share", [
    (1, 1, 1, 0.0), (7, 3, 5, 0.0), (100, 50, 1024, 0.5), (1000, 100000, 64, 0.0), (2000, 1000, 1023, 0.9),
    (8191, 300, 136, 0.3), (16384, 513, 72, 0.1), (16385, 511, 40, 0.6), (40000, 70000, 33, 0.5), (9000, 1, 24, 0.0),
    (140001, 997, 16, 0.2), (65537, 100, 9, 0.0), (300, 40, 4100, 0.3), (20000, 300, 3, 0.9)])
def test_embed_backward(T, V, H, share, dtype):
    """share: of the places that hold one and the same token."""
    say("embed_backward", T, V, H, share, dtype)
    token = torch.randint(-1, V + 1, (T,), generator=gen(T), device="cuda")
    token[torch.rand(T, generator=gen(2), device="cuda") < share] = V // 2
    d_out = normal(3, T, H, dtype=dtype)
    want, bound, n = embed_grad_ref(d_out, token, V, 1.7)
    got = ops.embed_backward(d_out, token, V, scale=1.7)
    close(got, want, bound, "d_table")
    assert torch.equal(got, ops.embed_backward(d_out, token.int(), V, scale=1.7))   # a fixed order
    into = normal(4, V, H)
    before = into.clone()
    want, bound, n = embed_grad_ref(d_out, token, V, 1.7, before)
    assert ops.embed_backward(d_out, token, V, scale=1.7, into=into) is into
    close(into, want, bound, "into")
    assert torch.equal(into[n == 0], before[n == 0])   # rows without a token are left


def test_embed_backward_strides_and_no_token():
    wide = normal(1, 500, 300, dtype=BF16)
    token = torch.randint(0, 40, (500,), generator=gen(2), device="cuda")
    for lo, H in ((0, 256), (8, 256), (1, 255)):
        a = ops.embed_backward(wide[:, lo:lo + H], token, 40)
        assert torch.equal(a, ops.embed_backward(wide[:, lo:lo + H].contiguous(), token, 40))
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert (ops.embed_backward(wide[:0], none, 40) == 0).all()
    kept = normal(3, 40, 300)
    assert torch.equal(ops.embed_backward(wide[:0], none, 40, into=kept.clone()), kept)
    far = torch.full((500,), 2**32 + 1, device="cuda")   # no token of the table: its low 32 bits are not its number
    assert (ops.embed_backward(wide, far, 40) == 0).all()
    assert torch.equal(ops.embed_backward(wide, far, 40, into=kept.clone()), kept)


def test_embed_backward_bad_rows_stay_alone():
    d_out = normal(1, 300, 64)
    token = torch.arange(300, device="cuda") % 30
    want = ops.embed_backward(d_out, token, 40)
    d_out[7] = nan
    got = ops.embed_backward(d_out, token, 40)
    others = torch.tensor([i for i in range(40) if i != 7], device="cuda")
    assert torch.equal(got[others], want[others]) and got[7].isnan().all()


# --------------------------------------------------------------------- dropout
M32 = 0xFFFFFFFF


def philox(counter, key):
    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = b >> 32 ^ c1 ^ k0, b & M32, a >> 32 ^ c3 ^ k1, a & M32
        k0, k1 = k0 + 0x9E3779B9 & M32, k1 + 0xBB67AE85 & M32
    return c0, c1, c2, c3


def test_philox_by_its_published_answers():
    assert philox((0, 0, 0, 0), (0, 0)) == (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)
    assert philox((M32,) * 4, (M32,) * 2) == (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)


def kept_ref(n, p, seed, offset):
    seed, offset = seed % 2**64, offset % 2**64
    out = []
    for i in range((n + 7) // 8):
        w = philox((i & M32, i >> 32, offset & M32, offset >> 32), (seed & M32, seed >> 32))
        out += [h >= math.floor(p * 65536 + 0.5) for v in w for h in (v & 0xffff, v >> 16)]
    return torch.tensor(out[:n])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("R,C", [(1, 1), (1, 8), (3, 7), (5, 64), (33, 40), (9, 1001), (16, 256)])
def test_dropout(R, C, dtype):
    say("dropout", R, C, dtype)
    x, residual = normal(1, R, C, dtype=dtype), normal(2, R, C, dtype=dtype)
    for p, seed, offset in ((0.1, 0, 0), (0.5, 12345678901234567890, 3), (0.25, -5, 2**40 + 9), (0.0, 1, 1), (1.0, 2, 2)):
        kept = kept_ref(R * C, p, seed, offset).view(R, C)
        cut = math.floor(p * 65536 + 0.5)
        factor = 65536 / (65536 - cut) if cut < 65536 else 0.0
        want = torch.where(kept, x.double().cpu() * factor, 0.0)
        got = ops.dropout(x, p, seed, offset)
        # the factor and the product are rounded, then the result
        close(got.cpu(), want, want.abs() * (UNIT[dtype] + 3 * U32) + TINY[dtype], "out")
        assert torch.equal(got, ops.dropout_backward(x, p, seed, offset))
        got = ops.dropout(x, p, seed, offset, residual=residual)
        whole = want + residual.double().cpu()
        close(got.cpu(), whole, whole.abs() * (UNIT[dtype] + U32) + want.abs() * 3 * U32 + TINY[dtype], "with residual")
        counter = torch.tensor([offset - 7 if offset < 2**63 else 0], device="cuda")
        assert torch.equal(got, ops.dropout(x, p, seed, offset - int(counter), residual=residual, counter=counter))
        if p == 0.0:
            assert torch.equal(ops.dropout(x, p, seed, offset), x)
        if p == 1.0:
            assert torch.equal(got, residual)


def test_dropout_strided_rows_have_the_mask_of_contiguous_ones():
    for dtype in (F32, BF16):
        wide, other = normal(1, 50, 300, dtype=dtype), normal(2, 50, 320, dtype=dtype)
        for lo, C in ((0, 256), (8, 256), (1, 256), (3, 255)):
            x, residual = wide[:, lo:lo + C], other[:, lo:lo + C]
            a = ops.dropout(x, 0.3, 7, 1, residual=residual)
            assert torch.equal(a, ops.dropout(x.contiguous(), 0.3, 7, 1, residual=residual.contiguous()))
    assert ops.dropout(wide[:0], 0.3, 7).shape == (0, 300)


def test_dropout_leaves_nothing_of_what_it_drops():
    x = torch.full((64, 128), nan, device="cuda")
    kept = ops.dropout(torch.ones(64, 128, device="cuda"), 0.5, 3, 4) != 0
    out = ops.dropout(x, 0.5, 3, 4)
    assert torch.equal(out.isnan(), kept) and (out[~kept] == 0).all()
    x[:] = inf
    assert (ops.dropout(x, 0.5, 3, 4)[~kept] == 0).all()


def test_dropout_shares():
    """Of 2^22 elements the kept are within six standard deviations, and two offsets or seeds agree as chance has it."""
    x, n, p = torch.ones(1024, 4096, device="cuda"), 2 ** 22, 0.3
    q = math.floor(p * 65536 + 0.5) / 65536
    a, b, c = (ops.dropout(x, p, *k) != 0 for k in ((1, 1), (1, 2), (2, 1)))
    dev = 6 * math.sqrt(q * (1 - q) / n)
    for m in (a, b, c):
        assert abs(float(m.float().mean()) - (1 - q)) < dev
    same = q * q + (1 - q) ** 2
    dev = 6 * math.sqrt(same * (1 - same) / n)
    for m in (b, c):
        assert abs(float((a == m).float().mean()) - same) < dev


# ------------------------------------------------- streams, graphs, all of them
def test_captured_calls_replay():
    """Every operator captured into a graph, whose inputs change between replays."""
    T, H, E, k, V = 200, 256, 16, 2, 300
    token = torch.randint(0, V, (T,), generator=gen(1), device="cuda")
    table, w, b = normal(2, V, H), normal(3, H), normal(4, H)
    logits, bias, g = normal(5, T, E), normal(6, E) * 0.1, normal(7, T, k)
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step():
        x = ops.embed(token, table)
        h = ops.dropout(x, 0.2, 5, 1, residual=x, counter=counter)
        y, mean, rstd = ops.layer_norm(h, w, b)
        r = ops.route_balanced(logits, k, bias=bias, groups=4, top_groups=2)
        d_logits = ops.route_balanced_backward(logits, r, g)
        d_h, d_w, d_b = ops.layer_norm_backward(y, h, w, mean, rstd, add=y)
        d_x = ops.dropout_backward(d_h, 0.2, 5, 1, counter=counter)
        d_table = ops.embed_backward(d_x, token, V)
        return x, h, y, mean, rstd, r.expert, r.weight, r.place, r.slot, d_logits, d_h, d_w, d_b, d_x, d_table

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    masks = []
    for i in range(4):
        logits.copy_(normal(20 + i, T, E))
        table.copy_(normal(30 + i, V, H))
        token.copy_(torch.randint(0, V, (T,), generator=gen(40 + i), device="cuda"))
        counter.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        for n, (a, want) in enumerate(zip(outs, step())):
            assert torch.equal(a, want), (i, n)
        masks.append((outs[13] == 0).clone())
    assert not torch.equal(masks[0], masks[1])


def test_two_streams_at_once():
    """The same calls on two streams, each with its own workspaces, as on one."""
    token = torch.randint(0, 5000, (20000,), generator=gen(1), device="cuda")
    d_out, x, w = normal(2, 20000, 64), normal(3, 4000, 1024), normal(4, 1024)
    logits, bias = normal(5, 4000, 256), normal(6, 256) * 0.1

    def all_of():
        y, mean, rstd = ops.layer_norm(x, w)
        r = ops.route_balanced(logits, 8, bias=bias, groups=8, top_groups=4)
        return (ops.embed_backward(d_out, token, 5000), y, *ops.layer_norm_backward(y, x, w, mean, rstd), r.expert, r.slot,
                r.weight)

    want = all_of()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams * 2:
        with torch.cuda.stream(s):
            got.append(all_of())
    torch.cuda.synchronize()
    for one in got:
        assert all(torch.equal(a, b) for a, b in zip(one, want))


def test_a_step_of_the_model_against_autograd():
    """Embedding, norm, balanced router, experts, the rows' sum, dropout onto the residual, all of it backward, against
    automatic differentiation in 64 bits.  Every bf16 rounding between an input and a result costs up to 2^-8 of it; there
    are at most ten one after another."""
    T, V, H, F, E, k = 90, 50, 64, 40, 8, 2
    token = torch.randint(0, V, (T,), generator=gen(1), device="cuda")
    table, w_norm = normal(2, V, H, dtype=BF16), (1 + 0.2 * normal(3, H)).to(BF16)
    b_norm, router = normal(4, H, dtype=BF16) * 0.1, normal(5, E, H) * H ** -0.5
    up, down = (normal(6, E, F, H) * H ** -0.5).to(BF16), (normal(7, E, H, F) * F ** -0.5).to(BF16)
    bias, d_out = normal(8, E) * 0.1, normal(9, T, H, dtype=BF16)
    p, seed = 0.2, 99
    how = {"scores": "sigmoid", "scale": 2.5}

    x = ops.embed(token, table, scale=2.0)
    n, mean, rstd = ops.layer_norm(x, w_norm, b_norm)
    logits = n.float() @ router.T
    r = ops.route_balanced(logits, k, bias=bias, groups=4, top_groups=2, **how)
    u = ops.expert_matmul(n, up, r.offset, slot=r.slot, top_k=k)
    y = ops.expert_matmul(u, down, r.offset)
    c = ops.combine(y, r.place, r.weight)
    out = ops.dropout(c, p, seed, residual=x)

    d_c = ops.dropout_backward(d_out, p, seed)
    d_y, d_weight = ops.combine_backward(d_c, y, r.slot, r.place, r.weight)
    d_u = ops.expert_matmul_grad_x(d_y, down, r.offset)
    d_down = ops.expert_matmul_grad_w(d_y, u, r.offset)
    d_up = ops.expert_matmul_grad_w(d_u, n, r.offset, slot=r.slot, top_k=k)
    d_logits = ops.route_balanced_backward(logits, r, d_weight, **how)
    d_n = ops.combine(ops.expert_matmul_grad_x(d_u, up, r.offset), r.place).float() + d_logits @ router
    d_x, d_w, d_b = ops.layer_norm_backward(d_n.to(BF16), x, w_norm, mean, rstd, add=d_out)
    d_table = ops.embed_backward(d_x, token, V, scale=2.0)

    leaves = [t.double().cpu().requires_grad_() for t in (table, w_norm, b_norm, router, up, down)]
    tb, wn, bn, ro, upd, dn = leaves
    xr = 2.0 * tb[token.cpu()]
    dev = xr - xr.mean(1, keepdim=True)
    nr = dev / (dev.square().mean(1, keepdim=True) + 1e-5).sqrt() * wn + bn
    expert = r.expert.long().cpu()   # the step's own choices
    assert (expert >= 0).all()
    s = torch.sigmoid(nr @ ro.T).gather(1, expert)
    weight = 2.5 * s / s.sum(1, keepdim=True)
    cr = torch.zeros(T, H, dtype=torch.float64)
    for j in range(k):
        e = expert[:, j]
        cr = cr + weight[:, j, None] * torch.bmm(dn[e], torch.bmm(upd[e], nr[:, :, None]))[:, :, 0]
    kept = kept_ref(T * H, p, seed, 0).view(T, H)
    cut = math.floor(p * 65536 + 0.5)
    want_out = xr + torch.where(kept, cr * (65536 / (65536 - cut)), 0.0)
    want_out.backward(d_out.double().cpu())
    d_router = d_logits.T @ n.float()
    have = [out, d_table, d_w, d_b, d_router, d_up, d_down]
    for name, a, want in zip(("out", "d_table", "d_w", "d_b", "d_router", "d_up", "d_down"), have,
                             [want_out.detach()] + [t.grad for t in leaves]):
        error = float((a.double().cpu() - want).norm() / want.norm())
        assert error < 10 * 2.0 ** -8, (name, error)
