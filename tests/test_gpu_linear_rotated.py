"""Linear layers as they are used: weights rotated and quantised once, activations rotated, quantised and multiplied per call, gradients
back through the product and the rotation to the inputs and the angles.  Every step is checked against 64 bits from what went into it,
and the whole against the layer that was never rotated or quantised."""
import numpy as np
import pytest
import torch

import linear_util as lu
import oracle
from gpu_util import check_dtheta, check_rotated
from linear_util import DEV, TORCH
from paper_2509_09679_amd import binding as B
from paper_2509_09679_amd import synth

pytestmark = pytest.mark.gpu

ROTATION = 2e-5  # error of the float32 cascade, relative to max(|value|, rms of the row)


class Rotated:
    """A layer of E experts: y = W x + b as W' x', x' = B(theta) x and W' = W B(theta)^T, both quantised per row."""

    def __init__(self, n, N, T, dtype, xbits, wbits, scale, E=1, offsets=None):
        self.n, self.N, self.T, self.dtype, self.xbits, self.wbits, self.E, self.offsets = n, N, T, dtype, xbits, wbits, E, offsets
        self.x0, self.theta0 = synth.small_case(n, T, dtype, seed=n + N + T)[:2]
        rng = np.random.default_rng([n, N, T, xbits, wbits, E])
        self.w0 = synth.cast_storage(rng.normal(size=(E * N, n)) / np.sqrt(n), dtype)
        self.x, self.w = (synth.storage_to_torch(a, dtype, DEV) for a in (self.x0, self.w0))
        self.x[T // 2] = 0
        self.x0 = synth.torch_to_storage(self.x, dtype)
        self.dy = torch.from_numpy(rng.normal(size=(T, N))).to(TORCH[dtype]).to(DEV)
        self.bias = torch.from_numpy(rng.normal(size=E * N)).to(TORCH[dtype]).to(DEV)
        self.theta = torch.from_numpy(self.theta0).to(DEV)
        self.plan = B.alloc_plan(self.theta, n, 1)
        self.qw, self.ws = self._codes(E * N, wbits, scale)
        self._quantise(self.w, torch.empty_like(self.w), self.qw, self.ws, wbits)
        self.shape = (E, N, self.qw.shape[1]) if offsets else self.qw.shape
        self.qx, self.xs = self._codes(T, xbits, scale)
        self.xr, self.y = torch.empty_like(self.x), torch.full((T, N), 3.0, dtype=self.x.dtype, device=DEV)
        self.dxr, self.dx = (torch.full_like(self.x, 3.0) for _ in range(2))
        self.dtheta = torch.empty_like(self.theta)
        qw = self.qw.view(self.shape)
        self.fwd = B.make_linear(self.qx, qw, self.ws, self.y, xbits=xbits, wbits=wbits)
        self.bwd = B.make_linear_bwd(self.dy, qw, self.ws, self.dxr, wbits=wbits)
        self.rows = B.make_rows(self.x, n, 1)
        self.work = torch.empty(B.bq_linear_bwd_workspace_bytes(self.bwd), dtype=torch.uint8, device=DEV)
        self.work_rotation = torch.empty(max(256, B.bq_butterfly_bwd_workspace_bytes(self.rows)), dtype=torch.uint8, device=DEV)
        self.off = lu.offsets_tensor(offsets) if offsets else None

    def _codes(self, rows, bits, scale):
        if bits == 8:
            return B.alloc_rows_quant8(rows, self.n, scale, DEV)
        return B.alloc_quant_outputs(rows, self.n, 1, bits, self.n, scale, DEV)

    def _quantise(self, v, rotated, codes, scales, bits):
        if bits == 8:
            B.bq_butterfly_fwd(v, rotated, self.plan, B.make_rows(v, self.n, 1))
            B.bq_rows_quant8(rotated, codes, scales)
        else:
            B.bq_butterfly_fwd_quant(v, self.plan, codes, scales, B.make_quant(bits, self.n, "f16" if scales.dtype is torch.float16 else "f32"),
                                     B.make_rows(v, self.n, 1))

    def forward(self):
        self._quantise(self.x, self.xr, self.qx, self.xs, self.xbits)
        qw = self.qw.view(self.shape)
        if self.off is None:
            B.bq_linear_fwd(self.qx, self.xs, qw, self.ws, self.bias, self.y, self.fwd)
        else:
            B.bq_linear_grouped_fwd(self.qx, self.xs, qw, self.ws, self.bias, self.off, self.y, self.fwd)

    def backward(self):
        qw = self.qw.view(self.shape)
        if self.off is None:
            B.bq_linear_bwd(self.dy, qw, self.ws, self.dxr, self.work, self.bwd)
        else:
            B.bq_linear_grouped_bwd(self.dy, qw, self.ws, self.off, self.dxr, self.work, self.bwd)
        B.bq_butterfly_bwd(self.x, self.dxr, self.plan, self.dx, self.dtheta, self.work_rotation, self.rows)

    def codes_of(self, codes, bits):
        a = codes.cpu().numpy()
        return a.astype(np.int64) if bits == 8 else oracle.unpack_codes(a, bits).astype(np.int64)

    def moved(self, rotated, scales, bits):
        """How far quantised values may lie from the exactly rotated ones: half a step, the cascade's error, the storage type's rounding of
        rows that were rotated first, and the roundings of v / s, each 2^-23 of at most 128 steps."""
        rms = np.sqrt((rotated ** 2).mean(1, keepdims=True))
        stored = lu.half_step(self.dtype) if bits == 8 else 0.0
        return lu.f64(scales).reshape(-1, 1) * (0.5 + 4 * 128 * 2.0 ** -23) + ROTATION * np.maximum(np.abs(rotated), rms) + stored * np.abs(rotated) + 2.0 ** -25


CASES = [(256, 96, 40, "f32", 8, 8, "f32"), (1024, 200, 130, "bf16", 8, 4, "f16"), (512, 264, 300, "f16", 4, 4, "f32"), (2048, 64, 7, "bf16", 8, 2, "f32"),
         (4096, 130, 1, "f16", 8, 8, "f16"), (128, 48, 600, "f16", 4, 2, "f16")]


def _groups(T):
    return [0, T // 3, T // 3, T - T // 7]


@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("n,N,T,dtype,xbits,wbits,scale", CASES)
def test_a_rotated_layer(n, N, T, dtype, xbits, wbits, scale, grouped):
    offsets = _groups(T) if grouped else [0, T]
    L = Rotated(n, N, T, dtype, xbits, wbits, scale, *((3, offsets) if grouped else ()))
    L.forward()
    L.backward()
    torch.cuda.synchronize()
    qx, qw = L.codes_of(L.qx, xbits), L.codes_of(L.qw, wbits).reshape(L.E, N, n)
    y, dy, last = lu.f64(L.y), L.dy, offsets[-1]
    # the product, from the codes and scales that the quantisers wrote
    want, size = lu.reference_fwd(qx, L.xs.view(-1), qw, L.ws, L.bias, offsets)
    lu.check(y[:last], want[:last], lu.bound_fwd(want, size, dtype)[:last], "product")
    assert (y[last:] == 3).all()
    # the layer without rotation and quantisation
    xr, wr = oracle.forward(synth.to_f64(L.x0, dtype), L.theta0, n), oracle.forward(synth.to_f64(L.w0, dtype), L.theta0, n)
    ex, ew = L.moved(xr, L.xs, xbits), L.moved(wr, L.ws, wbits).reshape(L.E, N, n)
    x64, w64, b64 = synth.to_f64(L.x0, dtype), synth.to_f64(L.w0, dtype).reshape(L.E, N, n), lu.f64(L.bias).reshape(L.E, N)
    wr = wr.reshape(L.E, N, n)
    for e in range(L.E):
        a, b = offsets[e], offsets[e + 1]
        plain = x64[a:b] @ w64[e].T + b64[e]
        far = ex[a:b] @ np.abs(wr[e]).T + np.abs(xr[a:b]) @ ew[e].T + ex[a:b] @ ew[e].T
        lu.check(y[a:b], plain, far + lu.bound_fwd(want, size, dtype)[a:b] + 1e-9 * np.abs(plain), "layer")
    # the gradient through the product, and from there through the rotation
    dwant, weight, top = lu.reference_bwd(dy, qw, L.ws, offsets)
    dxr = lu.f64(L.dxr)
    lu.check(dxr[:last], dwant[:last], lu.bound_bwd(dwant, weight, top, dtype)[:last], "gradient of the rotated rows")
    assert (dxr[last:] == 3).all()
    dx, dth, absacc = oracle.backward(x64, dxr, L.theta0, n)
    check_rotated(synth.torch_to_storage(L.dx, dtype), dx, dtype, "gradient of the rows")
    check_dtheta(L.dtheta.cpu().numpy(), dth, absacc, what="gradient of the angles")


@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("n,N,T,dtype,xbits,wbits,scale", [CASES[1], CASES[2], CASES[4]])
def test_a_rotated_layer_captured(n, N, T, dtype, xbits, wbits, scale, grouped):
    L = Rotated(n, N, T, dtype, xbits, wbits, scale, *((3, _groups(T)) if grouped else ()))
    outs = [L.qx, L.xs, L.y, L.dxr, L.dx, L.dtheta]

    def step():
        B.bq_plan_build(L.theta, n, 1, L.plan)
        L.forward()
        L.backward()

    step()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for _ in range(3):
        for o in outs:
            o.fill_(3)
        L.work.fill_(0xA5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
        step()
        torch.cuda.synchronize()
