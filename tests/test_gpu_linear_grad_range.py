"""Gradients of the quantised linear layers on rows whose entries span many binades: the bounds are relative to the terms themselves, as a
float32 product's would be, not to a row's largest entry.

Bounds.  A term is v = dy ws in float32 (2^-24 of it), taken to 22 bits for 16-bit rows (2^-22) or whole for float32 rows (2^-33), and
besides that to 2^-50 of the row's largest.  In the sum, of products that are exact, a term goes through five roundings within a matrix
instruction of 32 terms, one per later instruction and at most sixteen where the parts of the sum are joined and scaled; 2^-23 each,
whichever way the matrix cores round.  Then the result's own rounding."""
import numpy as np
import pytest
import torch

import linear_util as lu
from linear_util import DEV, TORCH
from paper_2509_09679_amd import binding as B

pytestmark = pytest.mark.gpu

FLOOR = 2.0 ** -50
# few rows, with the weights transposed first; many, with the weights as they lie; rows of weights that are no whole 16-byte pieces
SHAPES = [(5, 256, 64), (40, 4096, 96), (300, 520, 2112), (700, 1100, 1600), (33, 1000, 51)]


def _term(dtype):
    return 2.0 ** -24 + (2.0 ** -33 if dtype == "f32" else 2.0 ** -22)


def _layer(q, dy, ws, wbits, dtype, offsets=None):
    """dx of codes q [E, N, K], dy [T, N] (float64) and scales ws [E, N] (float64), and dy and ws as the call had them."""
    E, N, K = q.shape
    w = torch.from_numpy(lu.pack(q.reshape(E * N, K), wbits)).to(DEV)
    dy, ws = torch.from_numpy(dy).to(TORCH[dtype]).to(DEV), torch.from_numpy(ws).float().to(DEV)
    dx = torch.full((dy.shape[0], K), 3.0, dtype=TORCH[dtype], device=DEV)
    wd, wsd = (w.view(E, N, -1), ws) if offsets else (w, ws[0])
    d = B.make_linear_bwd(dy, wd, wsd, dx, wbits=wbits)
    work = torch.full((B.bq_linear_bwd_workspace_bytes(d),), 0xA5, dtype=torch.uint8, device=DEV)
    if offsets:
        B.bq_linear_grouped_bwd(dy, wd, wsd, lu.offsets_tensor(offsets), dx, work, d)
    else:
        B.bq_linear_bwd(dy, wd, wsd, dx, work, d)
    return lu.f64(dx), lu.f64(dy), lu.f64(ws)


def _check(dx, dy, ws, q, dtype, offsets, roundings):
    for e, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        v, w = dy[a:b] * ws[e], q[e].astype(np.float64)
        want, size = v @ w, np.abs(v) @ np.abs(w)
        f32 = (_term(dtype) + roundings * 2.0 ** -23) * size + FLOOR * np.abs(v).max(1, keepdims=True, initial=0.0) * np.abs(w).sum(0)
        lu.check(dx[a:b], want, f32 + (lu.half_step(dtype) * (np.abs(want) + f32) + lu.smallest(dtype) if dtype != "f32" else 2.0 ** -140), f"expert {e}")


def _roundings(N):
    return N / 32 + 1 + 5 + 16


@pytest.mark.parametrize("wbits", [8, 4, 2])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_every_term_by_itself(T, N, K, dtype, wbits):
    # an input that one output alone reads: its gradient is that term, however small it is beside the row's others
    rng = np.random.default_rng([T, N, K, wbits])
    q, o = np.zeros((1, N, K), dtype=np.int64), rng.integers(0, N, size=K)
    q[0, o, np.arange(K)] = np.where(rng.random(K) < 0.5, -(1 << (wbits - 1)), 1)
    span = 20 if dtype == "f16" else 40
    dy = rng.choice([-1.0, 1.0], size=(T, N)) * np.exp2(rng.uniform(-span, 0, size=(T, N))) * np.exp2(rng.integers(-4, 5, size=(T, 1)))
    dx, dy, ws = _layer(q, dy, np.exp2(rng.uniform(-4, 4, size=(1, N))), wbits, dtype)
    _check(dx, dy, ws, q, dtype, [0, T], 2)  # one product: the sums add zeros, the rest is scaling by powers of two and joining


@pytest.mark.parametrize("wbits", [8, 4, 2])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_the_largest_entry_meets_codes_of_zero(T, N, K, dtype, wbits):
    rng = np.random.default_rng([T, N, K, wbits, 1])
    q = lu.draw_codes(rng, (1, N, K), wbits)
    dy = rng.normal(size=(T, N)) * (1e-4 if dtype == "f16" else 1.0)
    top = rng.integers(0, N)
    dy[:, top] = 1e4 if dtype == "f16" else 1e8
    q[0, top] = 0
    dx, dy, ws = _layer(q, dy, rng.uniform(0.5, 2.0, size=(1, N)), wbits, dtype)
    _check(dx, dy, ws, q, dtype, [0, T], _roundings(N))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,N,K,wbits", [(4, 131071, 64, 8), (4, 32000, 64, 4), (200, 32000, 256, 2), (600, 11008, 1056, 8)])
def test_softmax_less_one_hot(T, N, K, wbits, dtype):
    # the gradient of a cross entropy: one entry near -1, the others share what it leaves; codes whose mean is not zero
    rng = np.random.default_rng([T, N, K])
    q = lu.draw_codes(rng, (1, N, K), wbits)
    q[0] = np.maximum(q[0], -1)
    p = np.exp(rng.normal(size=(T, N)))
    p /= p.sum(1, keepdims=True)
    p[np.arange(T), rng.integers(0, N, size=T)] -= 1.0
    dx, dy, ws = _layer(q, p, rng.uniform(0.5, 2.0, size=(1, N)), wbits, dtype)
    _check(dx, dy, ws, q, dtype, [0, T], _roundings(N))


@pytest.mark.parametrize("dtype,wbits", [("f32", 8), ("f16", 4), ("bf16", 2), ("bf16", 8)])
@pytest.mark.parametrize("T,N,K,offsets", [(60, 300, 64, [0, 20, 20, 41, 60]), (900, 200, 1056, [0, 150, 150, 700, 900])])
def test_experts(T, N, K, offsets, dtype, wbits):
    rng = np.random.default_rng([T, N, K, wbits, 2])
    q = lu.draw_codes(rng, (len(offsets) - 1, N, K), wbits)
    dy = rng.normal(size=(T, N)) * np.exp2(rng.uniform(-12 if dtype == "f16" else -30, 0, size=(T, N)))
    dx, dy, ws = _layer(q, dy, rng.uniform(0.5, 2.0, size=(len(offsets) - 1, N)), wbits, dtype, offsets)
    _check(dx, dy, ws, q, dtype, offsets, _roundings(N))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_rows_of_any_size(T, N, K, dtype):
    # rows from float32's smallest normal numbers to where the results come near its largest
    rng = np.random.default_rng([T, N, K, 3])
    q = lu.draw_codes(rng, (1, N, K), 8)
    dy = rng.uniform(-1, 1, size=(T, N)) * np.exp2(np.linspace(-100, 100, T).round())[:, None]
    dx, dy, ws = _layer(q, dy, rng.uniform(0.5, 1.0, size=(1, N)), 8, dtype)
    _check(dx, dy, ws, q, dtype, [0, T], _roundings(N))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_rows_of_subnormal_numbers(T, N, K, dtype):
    # scales of 1 leave dy as it is: rows of float32's or bfloat16's smallest numbers have all their digits
    rng = np.random.default_rng([T, N, K, 4])
    q = lu.draw_codes(rng, (1, N, K), 4)
    dy = np.rint(rng.uniform(-9, 9, size=(T, N))) * np.exp2(np.linspace(-149 if dtype == "f32" else -133, -125, T).round())[:, None]
    dx, dy, ws = _layer(q, dy, np.ones((1, N)), 4, dtype)
    v, w = dy * ws[0], q[0].astype(np.float64)
    want, size = v @ w, np.abs(v) @ np.abs(w)
    f32 = (_term(dtype) + _roundings(N) * 2.0 ** -23) * size + 2.0 ** -150  # (the result may be subnormal, too)
    lu.check(dx, want, f32 + (lu.half_step(dtype) * (np.abs(want) + f32) + lu.smallest(dtype) if dtype != "f32" else 0.0), "rows")
    assert (np.abs(dx) > 0).any()
