"""The layer norm's gradient needs no more workspace than its CTAs' sums take, and stays inside of it."""

import pytest
import torch

from paper_2501_17392_b200 import brace as B
from paper_2501_17392_b200 import build as brace_build

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def size(clients, rows, dim):
    return int(B.lib().brace_layer_norm_workspace_bytes(clients, rows, dim))


@pytest.fixture(scope="module", autouse=True)
def _built():
    brace_build.build()


def test_workspace_is_what_the_sums_take():
    """Two float32 vectors of a CTA; of rows that come through rings two or three CTAs of 256 threads share an SM (narrower ones
    of up to 4096 columns as many more), and a client has at least one."""
    assert size(1, 1 << 20, 8192) <= 148 * 2 * 2 * 8192 * 4
    assert size(1, 1 << 20, 768) <= 148 * 4 * 2 * 768 * 4
    assert size(1, 1 << 20, 4096) <= 148 * 4 * 2 * 4096 * 4
    for c in (1, 3, 700):
        for d in (1, 7, 64, 255, 256, 333, 768, 1024, 1032, 2048, 4096, 4104, 8192, 8200, 70001):
            sizes = [size(c, n, d) for n in (0, 1, 4, 31, 100, 1000, 10000, 100000, 1 << 30)]
            assert sizes == sorted(sizes) and all(s >= c * 2 * d * 4 for s in sizes)
            assert sizes[-1] <= max(148 * 16 * 2 * d * 4, c * 2 * d * 4 + 256, 256 * 148 * 16 * 8)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [40, 256, 333, 768, 1024, 1032, 2048, 4096, 8192, 8200])
@pytest.mark.parametrize("c,n", [(1, 3001), (5, 700)])
def test_workspace_of_exactly_the_size(d, c, n):
    need = size(c, n, d)
    whole = torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda")
    at = -whole.data_ptr() % 256
    g = torch.Generator(device="cuda").manual_seed(d)
    for tx, ty in ((F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16), (F16, F16)):
        for pad in (0, 1):      # rows on 16-byte boundaries, and not
            x, dy = (torch.randn(c, n, d + pad, device="cuda", generator=g).to(t)[:, :, :d] for t in (tx, ty))
            mean, rstd = x.float().mean(-1), (x.float().var(-1, correction=0) + 1e-5).rsqrt()
            dx, dw, db = torch.empty(c, n, d, device="cuda", dtype=tx), torch.empty(c, d, device="cuda"), torch.empty(c, d, device="cuda")
            plan = B.LayerNorm(d, n, clients=c, workspace=whole[at:at + need])
            plan.grad(dy, x, mean, rstd, dx, dweight=dw, dbias=db)
            assert bool((whole[:at] == 255).all()) and bool((whole[at + need:] == 255).all())
            # n terms in any order, each within 4 roundings of 2^-24
            xh = (x.double() - mean.double()[..., None]) * rstd.double()[..., None]
            for got, terms in ((dw, dy.double() * xh), (db, dy.double())):
                off = (got.double() - terms.sum(1)).abs()
                assert bool((off <= (n + 5) * 2.0 ** -24 * terms.abs().sum(1) + 2.0 ** -24 * terms.sum(1).abs()).all())
