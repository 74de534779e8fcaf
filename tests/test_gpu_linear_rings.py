"""Every kernel of the quantised linear layers on random codes and sums so long that its ring in LDS turns (tests/linear_rings.py): a place
that is read too early, or loaded again too early, shows in the sums."""
import pytest
import torch

import linear_rings as R
import linear_util as lu
from linear_util import DEV, TORCH
from paper_2509_09679_amd import binding as B
from test_gpu_linear import _codes_on_device, _ragged, _within

pytestmark = pytest.mark.gpu


def _layer(T, N, K, experts, wbits):
    gen = torch.Generator(device=DEV).manual_seed(T + N + K)
    E, offsets = max(1, experts), _ragged(T, experts) if experts else [0, T]
    qw, w = _codes_on_device(gen, (E, N, K), wbits)
    ws = torch.rand((E, N), generator=gen, device=DEV) * 0.01 + 1e-3
    return gen, offsets, qw, w if experts else w[0], ws if experts else ws[0]


@pytest.mark.parametrize("T,N,K,experts,xbits,wbits", R.FORWARD_CASES)
def test_forward(T, N, K, experts, xbits, wbits):
    gen, offsets, qw, w, ws = _layer(T, N, K, experts, wbits)
    qx, x = _codes_on_device(gen, (T, K), xbits)
    xs = torch.rand(T, generator=gen, device=DEV) * 0.01 + 1e-3
    y = torch.full((T, N), 3.0, device=DEV)
    d = B.make_linear(x, w, ws, y, xbits=xbits, wbits=wbits)
    if experts:
        B.bq_linear_grouped_fwd(x, xs, w, ws, None, lu.offsets_tensor(offsets), y, d)
    else:
        B.bq_linear_fwd(x, xs, w, ws, None, y, d)
    scales = ws.view(-1, N).double()
    for e, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        want = (qx[a:b] @ qw[e].t()) * xs[a:b, None].double() * scales[e]
        _within(y[a:b], want, 4 * 2.0 ** -24 * want.abs() + 1e-40)
    assert (y[:offsets[0]] == 3).all() and (y[offsets[-1]:] == 3).all()


def _check_gradient(T, N, K, experts, wbits, dtype):
    gen, offsets, qw, w, ws = _layer(T, N, K, experts, wbits)
    dy = torch.randn((T, N), generator=gen, device=DEV).to(TORCH[dtype])
    dx = torch.full((T, K), 3.0, dtype=TORCH[dtype], device=DEV)
    d = B.make_linear_bwd(dy, w, ws, dx, wbits=wbits)
    work = torch.full((B.bq_linear_bwd_workspace_bytes(d),), 0xA5, dtype=torch.uint8, device=DEV)
    if experts:
        B.bq_linear_grouped_bwd(dy, w, ws, lu.offsets_tensor(offsets), dx, work, d)
    else:
        B.bq_linear_bwd(dy, w, ws, dx, work, d)
    # a term: 2^-24 and 2^-22 or 2^-33 of itself, 2^-50 of the row's largest; the sum: a rounding per 32 terms, and 22 (test_gpu_linear_grad_range.py)
    term = 2.0 ** -24 + (2.0 ** -33 if dtype == "f32" else 2.0 ** -22) + (N / 32 + 22) * 2.0 ** -23
    scales = ws.view(-1, N).double()
    for e, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        if a == b:
            continue
        v, q = dy[a:b].double() * scales[e], qw[e].abs()
        want = v @ qw[e]
        f32 = term * (v.abs() @ q) + 2.0 ** -50 * v.abs().amax(1, keepdim=True) * q.sum(0)
        _within(dx[a:b], want, f32 + (lu.half_step(dtype) * (want.abs() + f32) + lu.smallest(dtype) if dtype != "f32" else 1e-40))
    assert (dx[:offsets[0]] == 3).all() and (dx[offsets[-1]:] == 3).all()


@pytest.mark.parametrize("T,N,K,experts,wbits,terms", R.GRADIENT_CASES)
def test_gradient(T, N, K, experts, wbits, terms):
    _check_gradient(T, N, K, experts, wbits, "f32" if terms == 3 else "f16" if T % 2 else "bf16")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N", [2504, 4095, 5063, 8000, 16376, 16383, 16400])
def test_gradients_of_wide_layers_on_weights_as_they_lie(N, dtype):
    # rows of terms from one piece of a wave to the widest that stay in registers, and those that do not, beside no transposition
    T, K = 1100, 4160
    for experts, wbits in ((0, 8), (3, 4)):
        assert R.gradient_choice(T, N, K, experts, wbits, 3 if dtype == "f32" else 2).kernel.across
        _check_gradient(T, N, K, experts, wbits, dtype)
