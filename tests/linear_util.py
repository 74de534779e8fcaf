"""Codes, references in 64 bits and error bounds for the tests of the quantised linear layers."""
import numpy as np
import torch

from paper_2509_09679_amd import binding as B

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
QMAX = {2: 32639.0, 3: 8355711.0}  # the gradient's digits: the largest number that 2 or 3 of them hold


def half_step(dtype):
    """A rounding to the type is off by at most this, relative to the value."""
    return torch.finfo(TORCH[dtype]).eps / 2


def smallest(dtype):
    """... and by this where the value is subnormal."""
    t = torch.finfo(TORCH[dtype])
    return t.smallest_normal * t.eps / 2


def draw_codes(rng, shape, bits):
    """Codes over the whole range of the fields, the extremes among them."""
    lo, hi = -(1 << (bits - 1)), (1 << (bits - 1)) - 1
    q = rng.integers(lo, hi + 1, size=shape)
    pick = rng.random(shape)
    return np.where(pick < 0.05, lo, np.where(pick > 0.95, hi, q)).astype(np.int64)


def pack(q, bits):
    """Two's-complement fields, lowest channel in the lowest bits; the last byte's unused fields hold ones."""
    per = 8 // bits
    width = q.shape[-1]
    full = -(-width // per) * per
    padded = np.full((*q.shape[:-1], full), -1, dtype=np.int64)
    padded[..., :width] = q
    f = (padded & ((1 << bits) - 1)).reshape(*q.shape[:-1], full // per, per)
    byte = np.zeros(f.shape[:-1], dtype=np.int64)
    for j in range(per):
        byte |= f[..., j] << (bits * j)
    return byte.astype(np.uint8).view(np.int8)


def strided(a, extra, offset=0):
    """A device tensor with a's values whose rows lie `extra` elements further apart and start `offset` elements into a buffer; what
    lies between the rows is not zero."""
    a = torch.from_numpy(np.ascontiguousarray(a)) if isinstance(a, np.ndarray) else a
    if not extra and not offset:
        return a.to(DEV)
    rows, width = a.shape
    ld = width + extra
    buf = torch.full((rows * ld + offset,), 7, dtype=a.dtype, device=DEV)
    v = buf[offset:].as_strided((rows, width), (ld, 1))
    v.copy_(a)
    return v


def scale_tensor(rng, shape, scale):
    s = np.exp(rng.normal(size=shape) * 0.5) * 2.0 ** -7
    return torch.from_numpy(s).to(TORCH[scale]).to(DEV)


def expert_of_rows(offsets, rows):
    e = np.full(rows, -1)
    for i, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        e[a:b] = i
    return e


def reference_fwd(qx, xs, qw, ws, bias, offsets):
    """(y, what its float32 steps act on) in float64: qx [T, K], qw [E, N, K]."""
    T, E, N = qx.shape[0], qw.shape[0], qw.shape[1]
    xs, ws = xs.double().cpu().numpy(), ws.double().cpu().numpy().reshape(E, N)
    y, size = np.zeros((T, N)), np.zeros((T, N))
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        p = (qx[a:b].astype(np.float64) @ qw[e].astype(np.float64).T) * xs[a:b, None] * ws[e]
        add = bias.double().cpu().numpy().reshape(E, N)[e] if bias is not None else 0.0
        y[a:b], size[a:b] = p + add, np.abs(p) + np.abs(add)
    return y, size


def bound_fwd(y, size, dtype):
    """Conversion of the sum, two scales, the bias: at most five float32 roundings; then the output's."""
    f32 = 5 * 2.0 ** -24 * size
    return f32 + half_step(dtype) * (np.abs(y) + f32) * (dtype != "f32") + smallest(dtype) + 2.0 ** -140


def reference_bwd(dy, qw, ws, offsets):
    """(dx, the sum of |w| per entry of dx, the largest |dy ws| of every row)."""
    E, N, K = qw.shape
    dy, ws = dy.double().cpu().numpy(), ws.double().cpu().numpy().reshape(E, N)
    dx, weight, top = np.zeros((dy.shape[0], K)), np.zeros((dy.shape[0], K)), np.zeros(dy.shape[0])
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        v = dy[a:b] * ws[e]
        dx[a:b] = v @ qw[e].astype(np.float64)
        weight[a:b] = np.abs(qw[e]).sum(0)
        top[a:b] = np.abs(v).max(1) if b > a else 0.0
    return dx, weight, top


def bound_bwd(dx, weight, top, dtype):
    """A term: half of the last digit, and float32 roundings of dy ws (which moves it and the row's largest), of m / largest, of the product
    with it and of the factor, each 2^-24 of at most the largest; their sum times |w|.  Then the sum's conversion, the factor, the output."""
    term = 0.5 / QMAX[3 if dtype == "f32" else 2] + 5 * 2.0 ** -24
    f32 = term * top[:, None] * weight + 2 * 2.0 ** -24 * np.abs(dx)
    return f32 + half_step(dtype) * (np.abs(dx) + f32) * (dtype != "f32") + smallest(dtype) + 2.0 ** -140


def check(got, want, bound, what):
    err = np.abs(got - want)
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} beyond the bound, the worst by {np.nanmax(err / bound):.3g}, first at {np.argwhere(bad)[0]}"


class Layer:
    """A random layer: codes, scales, bias and their device tensors."""

    def __init__(self, rng, T, N, K, E=None, xbits=8, wbits=8, dtype="bf16", scale="f32", bias=False, pad_x=0, pad_w=0, pad_y=0, shift=0):
        e = 1 if E is None else E
        self.dtype, self.bits, self.T, self.N, self.K, self.E = dtype, (xbits, wbits), T, N, K, e
        self.qx, self.qw = draw_codes(rng, (T, K), xbits), draw_codes(rng, (e, N, K), wbits)
        self.x = strided(pack(self.qx, xbits), pad_x, shift)
        w = strided(pack(self.qw, wbits).reshape(e * N, -1), pad_w, shift)
        self.w = w if E is None else w.as_strided((e, N, w.shape[1]), (N * w.stride(0) if e * N > 1 else w.shape[1], w.stride(0), 1), w.storage_offset())
        self.xs = scale_tensor(rng, (T,), scale)
        self.ws = scale_tensor(rng, (N,) if E is None else (e, N), scale)
        self.bias = torch.from_numpy(rng.normal(size=self.ws.shape)).to(TORCH[dtype]).to(DEV) if bias else None
        self.pad_y = pad_y

    def out(self, width):
        return strided(torch.full((self.T, width), 3.0, dtype=TORCH[self.dtype]), self.pad_y, 1 if self.pad_y % 2 else 0)

    def forward(self, offsets=None):
        y = self.out(self.N)
        d = B.make_linear(self.x, self.w, self.ws, y, xbits=self.bits[0], wbits=self.bits[1], inputs=self.K)
        if offsets is None:
            B.bq_linear_fwd(self.x, self.xs, self.w, self.ws, self.bias, y, d)
        else:
            B.bq_linear_grouped_fwd(self.x, self.xs, self.w, self.ws, self.bias, offsets, y, d)
        return y

    def backward(self, dy, offsets=None):
        dx = self.out(self.K)
        d = B.make_linear_bwd(dy, self.w, self.ws, dx, wbits=self.bits[1])
        ws = torch.full((B.bq_linear_bwd_workspace_bytes(d),), 0xA5, dtype=torch.uint8, device=DEV)
        if offsets is None:
            B.bq_linear_bwd(dy, self.w, self.ws, dx, ws, d)
        else:
            B.bq_linear_grouped_bwd(dy, self.w, self.ws, offsets, dx, ws, d)
        return dx


def offsets_tensor(offsets):
    return torch.tensor(offsets, dtype=torch.int32, device=DEV)


def f64(t):
    return t.double().cpu().numpy()
