"""The operators around a layer at sizes where a workgroup goes round its loop more than once: rows of the norm beyond the
grid, chunks of the embedding's gradient of more than eight places."""
import ctypes as C

import pytest
import torch

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_39350_amd import operators as ops   # noqa: E402
from .test_gpu_around_layer import check_norm   # noqa: E402
from .test_gpu_operators import U32, close, gen, normal, say   # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


# ------------------------------------------------------------------ layer norm
# threads of a row 64 (one and two vectors), 256 (one and two), 512 and 1,024, ragged rows and full ones; at least
# three rows, and an odd number of them, for a place of the grid in the gradient, two in the forward pass
NORMS = [(8200, 500), (8195, 512), (8197, 1000), (8193, 1024), (2049, 2000), (2051, 2048), (2050, 4090), (2049, 4096),
         (1027, 7168), (1025, 8192), (777, 16000), (775, 16384)]


@pytest.mark.parametrize("R,H", NORMS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layer_norm_of_more_rows_than_the_grid(R, H, dtype):
    for center, added in ((True, True), (True, False), (False, True), (False, False)):
        say("layer_norm", R, H, dtype, center, added)
        x = (normal(R + H, R, H) + normal(1, R, 1)).to(dtype)
        weight, bias = 1 + 0.2 * normal(2, H), 0.2 * normal(3, H)
        d_y, add = normal(4, R, H, dtype=dtype), normal(5, R, H, dtype=dtype) if added else None
        got = check_norm(x, weight, bias, 1e-5, center, d_y, add)
        # an element's additions in the weight's sums: its workgroup's rows, of 256 workgroups at least, then the others of
        # a wave (3), a run of the parts (512 / 16), the runs (16); 10 more for product, xhat and the margin.  A lost or
        # doubled row is far beyond it
        D = -(-R // 256) + 3 + 32 + 16 + 10
        hat = (x.double() - (got["mean"].double()[:, None] if center else 0)) * got["rstd"].double()[:, None]
        for name, terms in (("d_weight", d_y.double() * hat), ("d_bias", d_y.double())):
            size = terms.abs().sum(0)
            close(got[name], terms.sum(0), D * U32 * size, name)


# ------------------------------------------------------------------- embedding
def chunk_by_workspace(T, H):
    """The places of a chunk, from the workspace's size: sorted places, twice beyond 4,096, and two rows a chunk."""
    need = C.c_int64(0)
    assert ops._lib().hapmoe_embed_ws_bytes(T, H, C.byref(need)) == 0
    rest = need.value - (2 if T > 4096 else 1) * ((T + 1) // 2) * 16
    return [c for c in (8, 16, 32, 64, 128) if rest == -(-T // c) * 2 * H * 4]


def runs(chunk, T, seed):
    """Tokens whose sorted places end on and next to the chunks' borders, the last five of them none of the table's; every
    other token has none."""
    lengths = [chunk, chunk - 1, 1, 1, chunk + 1, 2 * chunk - 1, 1, 3 * chunk, 7, 1, chunk - 9, 8, 1, 5 * chunk + 3, chunk - 3]
    token, v = torch.full((T,), -1, dtype=torch.int64), 0
    at, cut = 0, T - 5
    while at < cut:
        n = min(lengths[v % len(lengths)], cut - at)
        token[at:at + n] = 2 * v
        at, v = at + n, v + 1
    order = torch.randperm(T, generator=torch.Generator().manual_seed(seed))
    return token[order].cuda(), 2 * v


# 16, 32, 64 and 128 places a chunk; rows of several workgroups, of one, of eight lanes
CHUNKS = [(4096, 4096, 16), (8192, 4104, 32), (16389, 4100, 64), (32771, 4096, 128), (262147, 64, 16), (40000, 1023, 32),
          (2097157, 72, 128), (600000, 40, 16)]


@pytest.mark.parametrize("T,H,chunk", CHUNKS)
@pytest.mark.parametrize("which", ["one", "runs", "any"])
def test_embed_backward_by_long_chunks(T, H, chunk, which):
    """Whole numbers of up to 2: every sum is exact in fp32, in any order, and has to be equal."""
    say("embed_backward", T, H, chunk, which)
    assert chunk_by_workspace(T, H) == [chunk]
    if which == "one":
        V, token = 3, torch.full((T,), 1, device="cuda")
    elif which == "runs":
        token, V = runs(chunk, T, T)
    else:
        V = 1013
        u = torch.rand(T, generator=gen(T), device="cuda")
        token = (V * u.square() * 1.01).long() - 3   # the low ones often, some out of the table
    assert int((token < 0).sum() + (token >= V).sum()) > 0 or which == "one"
    assert T * 2 + 4 < 2 ** 24
    for dtype in (F32, BF16):
        d_out = torch.randint(-2, 3, (T, H), generator=gen(2), device="cuda", dtype=torch.int8).to(dtype)
        real = (token >= 0) & (token < V)
        want = torch.zeros(V, H, device="cuda", dtype=torch.float64)
        for lo in range(0, T, 1 << 16):
            part = slice(lo, lo + (1 << 16))
            if which == "one":   # not one after another
                want[1] += d_out[part].double().sum(0)
            else:
                want.index_add_(0, token[part][real[part]], d_out[part][real[part]].double())
        got = ops.embed_backward(d_out, token, V, scale=0.5)
        assert torch.equal(got.double(), 0.5 * want)
        into = torch.randint(-2, 3, (V, H), generator=gen(3), device="cuda").float()
        whole = into.double() + 0.5 * want
        ops.embed_backward(d_out, token, V, scale=0.5, into=into)
        assert torch.equal(into.double(), whole)
