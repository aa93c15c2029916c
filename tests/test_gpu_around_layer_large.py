"""The operators around a layer on matrices of more than 2^32 elements: rows at their ends against the formulas in 64 bits."""
import math

import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_around_layer import M32, norm_ref, philox   # noqa: E402
from .test_gpu_operators import TINY, U32, UNIT, close, gen, normal, say   # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
H, ROWS = 4096, (1 << 20) + 3   # more than 2^32 elements


@pytest.fixture(scope="module")
def big():
    x = torch.empty(ROWS, H, dtype=BF16, device="cuda")
    few = normal(1, 64, H, dtype=BF16)
    for part in x.split(1 << 16):
        part.copy_(few[torch.arange(len(part), device="cuda") % 64])
    return x


def ends(x):
    return torch.cat([x[:2], x[-3:]])


def test_layer_norm(big):
    say("layer_norm", tuple(big.shape))
    w, b = normal(2, H), normal(3, H)
    y, mean, rstd = ops.layer_norm(big, w, b)
    d_y, add = ends(big).flip(0).contiguous(), ends(big)
    ref = norm_ref(ends(big), w, b, 1e-5, True, d_y, add)
    for name, got in (("y", ends(y)), ("mean", ends(mean)), ("rstd", ends(rstd))):
        want, bound = ref[name]
        close(got, want, bound + (want.abs() * UNIT[BF16] + TINY[BF16] if name == "y" else 0), name)
    d_x, d_w, d_b = ops.layer_norm_backward(y, big, w, mean, rstd)
    one = ops.layer_norm_backward(ends(y), ends(big), w, ends(mean), ends(rstd))[0]
    # rows of the same 16 bits have the same gradient, wherever they lie
    assert torch.equal(ends(d_x), one)
    assert d_w.isfinite().all() and d_b.isfinite().all()


def test_dropout(big):
    say("dropout", tuple(big.shape))
    out = ops.dropout(big, 0.4, 11, 12)
    cut = math.floor(0.4 * 65536 + 0.5)
    for row in (0, ROWS - 1):
        words = [philox((i & M32, i >> 32, 12, 0), (11, 0)) for i in range(row * H // 8, (row + 1) * H // 8)]
        kept = torch.tensor([h >= cut for v in words for w in v for h in (w & 0xffff, w >> 16)])
        want = torch.where(kept, big[row].double().cpu() * (65536 / (65536 - cut)), 0.0)
        close(out[row].cpu(), want, want.abs() * (UNIT[BF16] + 3 * U32) + TINY[BF16], row)


def test_embed(big):
    say("embed", tuple(big.shape))
    token = torch.randint(0, ROWS, (500,), generator=gen(4), device="cuda")
    token[:4] = torch.tensor([0, ROWS - 1, ROWS, ROWS - 1], device="cuda")
    out = ops.embed(token, big)
    want = torch.where((token < ROWS)[:, None], big[token.clamp_max(ROWS - 1)], 0)
    assert torch.equal(out, want)
    d_table = ops.embed_backward(out, token, ROWS)
    want = out[token == ROWS - 1].double().sum(0)
    close(d_table[-1], want, out[token == ROWS - 1].double().abs().sum(0) * 4 * U32)
    named = torch.zeros(ROWS, dtype=torch.bool, device="cuda")
    named[token[token < ROWS]] = True
    for at in range(0, ROWS, 1 << 17):
        part, mark = d_table[at:at + (1 << 17)], named[at:at + (1 << 17)]
        assert torch.equal((part != 0).any(1), mark)


def test_layer_norm_weight_gradient(big):
    """The sums over 2^20 rows against sums in 64 bits, taken in pieces."""
    say("layer_norm_backward", tuple(big.shape))
    w, b = normal(2, H), normal(3, H)
    y, mean, rstd = ops.layer_norm(big, w, b)
    _, d_w, d_b = ops.layer_norm_backward(y, big, w, mean, rstd)
    sums = torch.zeros(4, H, dtype=torch.float64, device="cuda")
    for at in range(0, ROWS, 1 << 14):
        g, x = y[at:at + (1 << 14)].double(), big[at:at + (1 << 14)].double()
        hat = (x - mean[at:at + (1 << 14), None].double()) * rstd[at:at + (1 << 14), None].double()
        for n, terms in enumerate((g * hat, g)):
            sums[2 * n] += terms.sum(0)
            sums[2 * n + 1] += terms.abs().sum(0)
    # additions: a workgroup's rows, of 512, a run of the parts, the runs; product and xhat
    D = -(-ROWS // 512) + 32 + 16 + 10
    for name, got, n in (("d_weight", d_w, 0), ("d_bias", d_b, 1)):
        close(got, sums[2 * n], D * U32 * sums[2 * n + 1], name)
