"""Results of the quantised linear layers that do not depend on how the operands lie, and calls that repeat themselves bit for bit."""
import numpy as np
import pytest
import torch

import linear_util as lu
from linear_util import DEV, TORCH
from paper_2509_09679_amd import binding as B

pytestmark = pytest.mark.gpu


def _at(a, extra, offset):
    """a's bytes with rows `extra` further apart, starting `offset` bytes into a buffer."""
    return lu.strided(a.reshape(-1, a.shape[-1]), extra, offset)


@pytest.mark.parametrize("bits", [(8, 8), (8, 4), (8, 2), (4, 8), (4, 4), (4, 2)])
@pytest.mark.parametrize("T,N,K", [(3, 70, 256), (40, 200, 1088), (300, 1000, 576), (700, 520, 4160)])
def test_products_of_any_layout_are_those_of_the_fast_one(T, N, K, bits):
    rng = np.random.default_rng([T, N, K, *bits])
    x, w = (torch.from_numpy(lu.pack(lu.draw_codes(rng, (r, K), b), b)) for r, b in ((T, bits[0]), (N, bits[1])))
    xs, ws = (torch.from_numpy(np.exp(rng.normal(size=r))).float().to(DEV) for r in (T, N))
    bias = torch.from_numpy(rng.normal(size=N) * K).float().to(DEV)
    for b in (None, bias):
        got = []
        for extra, offset in ((0, 0), (1, 3), (16, 1)):
            xx, ww, y = _at(x, extra, offset), _at(w, extra, offset), torch.empty(T, N, device=DEV)
            B.bq_linear_fwd(xx, xs, ww, ws, b, y, B.make_linear(xx, ww, ws, y, xbits=bits[0], wbits=bits[1], inputs=K))
            got.append(y)
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K,E", [(8, 4096, 4096, 0), (700, 1100, 1600, 0), (300, 2050, 51, 0), (200, 1000, 512, 6)])
def test_gradients_repeat_themselves(T, N, K, E, dtype):
    rng = np.random.default_rng([T, N, K, E])
    e = max(1, E)
    w = torch.from_numpy(lu.pack(lu.draw_codes(rng, (e * N, K), 8), 8)).to(DEV)
    ws, dy = torch.rand(e * N, device=DEV), torch.randn(T, N, device=DEV).to(TORCH[dtype])
    if E:
        w, ws, off = w.view(E, N, K), ws.view(E, N), lu.offsets_tensor([0, 0, 30, 31, 150, T - 5, T])
    want = None
    for i in range(5):
        dx = torch.full((T, K), 3.0, dtype=TORCH[dtype], device=DEV)
        d = B.make_linear_bwd(dy, w, ws, dx)
        work = torch.full((B.bq_linear_bwd_workspace_bytes(d),), (0xA5, 0xFF, 0x7C, 0, 0x3C)[i], dtype=torch.uint8, device=DEV)
        if E:
            B.bq_linear_grouped_bwd(dy, w, ws, off, dx, work, d)
        else:
            B.bq_linear_bwd(dy, w, ws, dx, work, d)
        want = dx if want is None else want
        assert torch.equal(dx, want)
