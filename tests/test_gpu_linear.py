"""The quantised linear layers on the GPU: every call against the same arithmetic in 64 bits, at the sizes, strides and groups where it
can go wrong.  The bounds count roundings (tests/linear_util.py)."""
import numpy as np
import pytest
import torch

import linear_util as lu
from linear_util import DEV, Layer, TORCH
from paper_2509_09679_amd import binding as B

pytestmark = pytest.mark.gpu


# ---- INT8 codes per row -------------------------------------------------------------------------------


def _quant8_reference(x, scale):
    """The steps of the contract in numpy float32."""
    v = x.float().cpu().numpy()
    s = np.abs(v).max(1) / np.float32(127.0)
    if scale == "f16":
        s = np.minimum(s, np.float32(65504.0)).astype(np.float16).astype(np.float32)
    s = np.where(s < np.float32(2.0 ** -126), np.float32(0.0), s)
    with np.errstate(divide="ignore"):
        inv = np.where(s == 0, np.float32(0.0), np.float32(1.0) / s)
    q = np.clip(np.rint(v * inv[:, None]), -128, 127).astype(np.int8)
    return q, s


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 8), (1, 4096), (37, 512), (9, 520), (6, 1024), (7, 1032), (4, 2048), (5, 2056), (2, 5120),
                                       (3, 8200), (2, 16384), (2, 16392), (1, 32768), (2, 32776), (3, 11008), (1030, 40), (67, 120), (35, 200),
                                       (21, 225), (13, 505), (6, 1001), (5, 2047), (3, 4081), (3, 8189), (2, 16383), (2, 32767), (2, 32769)])
def test_rows_quant8_is_bit_exact(dtype, rows, cols):
    rng = np.random.default_rng([rows, cols, len(dtype)])
    for scale, pad, shift in (("f32", 0, 0), ("f16", 8, 0), ("f32", 3, 1)):
        v = rng.standard_t(3, size=(rows, cols)) * np.exp(rng.normal(size=(rows, 1)) * 3)
        x = lu.strided(torch.from_numpy(np.clip(v, -6e4, 6e4)).to(TORCH[dtype]), pad, shift)
        codes = lu.strided(np.full((rows, cols), 77, dtype=np.int8), pad, shift)
        scales = torch.empty(rows, dtype=TORCH[scale], device=DEV)
        B.bq_rows_quant8(x, codes, scales)
        q, s = _quant8_reference(x, scale)
        np.testing.assert_array_equal(scales.float().cpu().numpy(), s)
        np.testing.assert_array_equal(codes.cpu().numpy(), q)
        if pad and rows > 1:  # what lies between the rows stays
            gap = codes.as_strided((rows - 1, pad), (cols + pad, 1), codes.storage_offset() + cols)
            assert (gap == 7).all()


@pytest.mark.parametrize("cols", [5, 64, 131, 1024, 2047, 5120, 40000])
def test_rows_quant8_special_rows(cols):
    x = torch.randn(7, cols, device=DEV)
    x[0] = 0
    x[1, cols // 2] = float("inf")
    x[2, cols - 1] = float("nan")
    x[3] *= 2.0 ** -124  # a scale below 2^-126
    x[4] *= 2.0 ** -100
    x[5, 0] = -float("inf")
    codes, scales = B.alloc_rows_quant8(7, cols, "f32", DEV)
    B.bq_rows_quant8(x, codes, scales)
    for r in (0, 3):
        assert scales[r] == 0 and (codes[r] == 0).all()
    for r in (1, 2, 5):
        assert torch.isnan(scales[r]) and (codes[r] == 0).all()
    for r in (4, 6):
        assert codes[r].abs().max() == 127
        assert (codes[r].double() * scales[r].double() - x[r].double()).abs().max() <= scales[r].double() * (0.5 + 1e-5)
    half = torch.empty(7, dtype=torch.float16, device=DEV)
    B.bq_rows_quant8(x * 3e7, codes, half)  # beyond binary16: saturates
    assert half[6] == 65504 and torch.isnan(half[1])


def test_rows_quant8_of_no_rows():
    codes, scales = B.alloc_rows_quant8(0, 64, "f32", DEV)
    B.bq_rows_quant8(torch.empty(0, 64, device=DEV), codes, scales)


# ---- products ------------------------------------------------------------------------------------------

SIZES = [(1, 1, 1), (1, 16, 64), (2, 100, 37), (5, 33, 128), (16, 64, 256), (17, 48, 320), (31, 256, 64), (33, 130, 1024), (64, 257, 192),
         (65, 512, 448), (100, 1000, 144), (128, 128, 128), (129, 384, 640), (257, 300, 832), (300, 520, 2048), (513, 264, 16)]
BITS = [(8, 8), (8, 4), (8, 2), (4, 8), (4, 4), (4, 2)]


@pytest.mark.parametrize("xbits,wbits", BITS)
@pytest.mark.parametrize("T,N,K", SIZES)
def test_linear_fwd(T, N, K, xbits, wbits):
    rng = np.random.default_rng([T, N, K, xbits, wbits])
    for dtype, scale, bias in (("f32", "f32", True), ("f16", "f16", False), ("bf16", "f32", True)):
        L = Layer(rng, T, N, K, xbits=xbits, wbits=wbits, dtype=dtype, scale=scale, bias=bias)
        want, size = lu.reference_fwd(L.qx, L.xs, L.qw, L.ws, L.bias, [0, T])
        lu.check(lu.f64(L.forward()), want, lu.bound_fwd(want, size, dtype), f"{dtype}")


@pytest.mark.parametrize("T,N,K", [(4, 40, 96), (70, 200, 512), (300, 264, 256), (600, 2051, 384)])
@pytest.mark.parametrize("pads", [(16, 16, 8, 0), (16, 0, 1, 0), (1, 3, 1, 1), (0, 0, 5, 0), (32, 0, 0, 16), (0, 0, 0, 5)])
def test_linear_fwd_strides_and_alignment(T, N, K, pads):
    rng = np.random.default_rng([T, N, K, *pads])
    for bits in ((8, 8), (4, 2)):
        L = Layer(rng, T, N, K, xbits=bits[0], wbits=bits[1], dtype="f16", bias=True, pad_x=pads[0], pad_w=pads[1], pad_y=pads[2], shift=pads[3])
        y = L.forward()
        want, size = lu.reference_fwd(L.qx, L.xs, L.qw, L.ws, L.bias, [0, T])
        lu.check(lu.f64(y), want, lu.bound_fwd(want, size, "f16"), f"{bits}")
        if pads[2]:
            gap = y.as_strided((T - 1, pads[2]), (N + pads[2], 1), y.storage_offset() + N)
            assert (gap == 7).all()


def test_linear_fwd_extreme_sums():
    # every product +2^14 over the widest rows: the sum reaches 131071 * 2^14, the last one that 32 bits hold
    for K, bits in ((131071, (8, 8)), (131008, (8, 8)), (131008, (4, 4)), (131008, (8, 2))):
        lo = [-(1 << (b - 1)) for b in bits]
        x = torch.from_numpy(lu.pack(np.full((3, K), lo[0]), bits[0])).to(DEV)
        w = torch.from_numpy(lu.pack(np.full((18, K), lo[1]), bits[1])).to(DEV)
        one, y = torch.ones(18, device=DEV), torch.empty(3, 18, device=DEV)
        B.bq_linear_fwd(x, one[:3], w, one, None, y, B.make_linear(x, w, one, y, xbits=bits[0], wbits=bits[1], inputs=K))
        assert (y == float(np.float32(K * lo[0] * lo[1]))).all()


def test_linear_fwd_scales_carry_nan_and_zero():
    rng = np.random.default_rng(5)
    L = Layer(rng, 40, 64, 128, dtype="f32")
    L.xs[3], L.ws[7], L.xs[5] = float("nan"), 0.0, 0.0
    y = L.forward()
    assert torch.isnan(y[3]).all() and (y[5] == 0).all() and (y[:3, 7] == 0).all() and torch.isfinite(y[4]).all()


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("T,N,K", [(3, 40, 128), (70, 200, 512), (300, 264, 256), (20, 30, 51)])
def test_linear_fwd_smallest_scales(T, N, K, bits):
    # scales of rows down to float32's smallest normal number, the smallest that the quantisers write
    L = Layer(np.random.default_rng([T, N, K, *bits]), T, N, K, xbits=bits[0], wbits=bits[1], dtype="f32")
    L.xs = L.xs * 0 + 2.0 ** -126 * (1 + torch.rand(T, device=DEV))
    L.ws = 1 + torch.rand(N, device=DEV)
    want, size = lu.reference_fwd(L.qx, L.xs, L.qw, L.ws, None, [0, T])
    lu.check(lu.f64(L.forward()), want, 5 * 2.0 ** -24 * size + 2.0 ** -148, f"{bits}")


GROUPS = [
    (40, [0, 40]),
    (40, [0, 0, 40, 40]),
    (64, [0, 1, 1, 18, 64]),
    (96, [5, 21, 22, 90]),  # rows before the first and behind the last expert
    (300, [0, 3, 3, 150, 151, 290, 290, 290, 300]),
    (700, [0, 0, 690, 700]),
    (30, [7] * 71 + [20] * 60),  # more experts than a wave looks at at once
    (1, [0, 0, 1]),
]


@pytest.mark.parametrize("N,K", [(40, 64), (200, 37), (264, 384)])
@pytest.mark.parametrize("T,offsets", GROUPS)
def test_grouped_fwd(T, offsets, N, K):
    rng = np.random.default_rng([T, len(offsets), N, K])
    for dtype, bits, bias in (("bf16", (8, 8), True), ("f32", (4, 4), False), ("f16", (8, 2), True)):
        L = Layer(rng, T, N, K, E=len(offsets) - 1, xbits=bits[0], wbits=bits[1], dtype=dtype, bias=bias)
        y = lu.f64(L.forward(lu.offsets_tensor(offsets)))
        want, size = lu.reference_fwd(L.qx, L.xs, L.qw, L.ws, L.bias, offsets)
        a, b = offsets[0], offsets[-1]
        lu.check(y[a:b], want[a:b], lu.bound_fwd(want, size, dtype)[a:b], f"{dtype}")
        assert (y[:a] == 3).all() and (y[b:] == 3).all()  # rows of no expert are left as they were


def test_grouped_offsets_outside_the_batch_are_taken_as_the_nearest_inside():
    rng = np.random.default_rng(8)
    L = Layer(rng, 50, 70, 64, E=3, dtype="f32")
    y = lu.f64(L.forward(lu.offsets_tensor([-9, 20, 45, 4000])))
    want, size = lu.reference_fwd(L.qx, L.xs, L.qw, L.ws, L.bias, [0, 20, 45, 50])
    lu.check(y, want, lu.bound_fwd(want, size, "f32"), "clamped")


# ---- gradients -----------------------------------------------------------------------------------------


def _gradient(rng, T, N, dtype, pad=0):
    g = rng.standard_t(4, size=(T, N)) * np.exp(rng.normal(size=(T, 1)) * 2) * 1e-3
    return lu.strided(torch.from_numpy(np.clip(g, -100, 100)).to(TORCH[dtype]), pad)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,N,K", [(1, 1, 1), (2, 37, 100), (5, 128, 33), (17, 320, 48), (64, 64, 64), (65, 200, 130), (130, 1000, 264), (200, 129, 512),
                                   (300, 2048, 96)])
def test_linear_bwd(T, N, K, dtype):
    rng = np.random.default_rng([T, N, K])
    for wbits, scale, pad in ((8, "f32", 0), (4, "f16", 8), (2, "f32", 3)):
        L = Layer(rng, T, N, K, wbits=wbits, dtype=dtype, scale=scale, pad_w=pad, pad_y=pad)
        dy = _gradient(rng, T, N, dtype, pad)
        dx = lu.f64(L.backward(dy))
        want, weight, top = lu.reference_bwd(dy, L.qw, L.ws, [0, T])
        lu.check(dx, want, lu.bound_bwd(want, weight, top, dtype), f"w{wbits}")


@pytest.mark.parametrize("N,K", [(40, 64), (200, 37), (264, 384)])
@pytest.mark.parametrize("T,offsets", GROUPS)
def test_grouped_bwd(T, offsets, N, K):
    rng = np.random.default_rng([T, len(offsets), N, K])
    for dtype, wbits in (("bf16", 8), ("f32", 4)):
        L = Layer(rng, T, N, K, E=len(offsets) - 1, wbits=wbits, dtype=dtype)
        dy = _gradient(rng, T, N, dtype)
        dx = lu.f64(L.backward(dy, lu.offsets_tensor(offsets)))
        want, weight, top = lu.reference_bwd(dy, L.qw, L.ws, offsets)
        a, b = offsets[0], offsets[-1]
        lu.check(dx[a:b], want[a:b], lu.bound_bwd(want, weight, top, dtype)[a:b], f"{dtype}")
        assert (dx[:a] == 3).all() and (dx[b:] == 3).all()


def test_bwd_is_the_derivative_of_fwd():
    # <dy, y(x + h e) - y(x - h e)> / 2h along single dequantised entries, which the layer is linear in: one code up, one down
    rng = np.random.default_rng(11)
    T, N, K = 6, 50, 40
    L = Layer(rng, T, N, K, dtype="f32")
    L.qx = np.clip(L.qx, -120, 120)
    dy = _gradient(rng, T, N, "f32")
    dx = lu.f64(L.backward(dy))
    _, weight, top = lu.reference_bwd(dy, L.qw, L.ws, [0, T])
    g, xs = lu.f64(dy), lu.f64(L.xs)
    for t, k in ((0, 0), (3, 17), (5, 39)):
        sides = []
        for h in (1, -1):
            q = L.qx.copy()
            q[t, k] += h
            L.x = torch.from_numpy(lu.pack(q, 8)).to(DEV)
            y = lu.f64(L.forward())
            sides.append(((g * y).sum(), (np.abs(g * y)).sum()))
        d = (sides[0][0] - sides[1][0]) / (2 * xs[t])
        err = lu.bound_bwd(np.array([[dx[t, k]]]), weight[t:t + 1, k:k + 1], top[t:t + 1], "f32")[0, 0]
        assert abs(d - dx[t, k]) <= err + 5 * 2.0 ** -24 * (sides[0][1] + sides[1][1]) / (2 * xs[t])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bwd_special_rows(dtype):
    rng = np.random.default_rng(12)
    T, N, K = 9, 130, 96
    L = Layer(rng, T, N, K, dtype=dtype)
    dy = _gradient(rng, T, N, dtype).clone()
    dy[0] = 0
    dy[1, 5] = float("nan")
    dy[2, 129] = float("inf")
    dy[3] = dy[4] * 2.0 ** -90   # tiny rows keep their relative accuracy
    dy[5] = dy[4] * 2.0 ** -119  # ... down to 2^-120
    dy[6, 1:] = 0                # one entry
    dx = lu.f64(L.backward(dy))
    assert (dx[0] == 0).all() and np.isnan(dx[1]).all() and np.isnan(dx[2]).all()
    want, weight, top = lu.reference_bwd(dy, L.qw, L.ws, [0, T])
    keep = [3, 4, 6, 7, 8]
    lu.check(dx[keep], want[keep], lu.bound_bwd(want, weight, top, dtype)[keep], "rows")
    assert np.isfinite(dx[5]).all() and (np.abs(dx[5] - want[5]) <= 2.0 ** -119 * weight[5]).all()


@pytest.mark.parametrize("wbits", [8, 4, 2])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K", [(5, 64, 48), (40, 200, 96), (300, 520, 2112)])
def test_bwd_of_tiny_rows(T, N, K, dtype, wbits):
    # row by row from 2^-60 to 2^-118, the last binade above the one that may count as 0
    rng = np.random.default_rng([T, N, K, wbits])
    L = Layer(rng, T, N, K, wbits=wbits, dtype=dtype)
    L.ws = 1 + torch.rand(N, device=DEV)
    g = rng.uniform(-1, 1, size=(T, N))
    g[:, 0] = 1
    dy = torch.from_numpy(g * 2.0 ** -np.linspace(60, 118, T).round()[:, None]).to(TORCH[dtype]).to(DEV)
    want, weight, top = lu.reference_bwd(dy, L.qw, L.ws, [0, T])
    f32 = (0.5 / lu.QMAX[3 if dtype == "f32" else 2] + 5 * 2.0 ** -24) * top[:, None] * weight + 2 * 2.0 ** -24 * np.abs(want)
    lu.check(lu.f64(L.backward(dy)), want, f32 + (lu.half_step(dtype) * (np.abs(want) + f32) if dtype != "f32" else 0) + 2.0 ** -148, "dx")


# ---- streams, graphs, a layer as it is used --------------------------------------------------------------


def test_captured_calls_replay_bit_exact():
    rng = np.random.default_rng(13)
    T, N, K, offsets = 200, 320, 512, [0, 70, 70, 180]
    x = torch.randn(T, K, device=DEV, dtype=torch.float16)
    codes, xs = B.alloc_rows_quant8(T, K, "f32", DEV)
    L, G = Layer(rng, T, N, K, dtype="f16", wbits=4), Layer(rng, T, N, K, E=3, dtype="f16")
    off = lu.offsets_tensor(offsets)
    y, yg, dx, dxg = (torch.zeros(T, w, dtype=torch.float16, device=DEV) for w in (N, N, K, K))
    d, dg = B.make_linear(codes, L.w, L.ws, y, wbits=4), B.make_linear(codes, G.w, G.ws, yg)
    b, bg = B.make_linear_bwd(y, L.w, L.ws, dx, wbits=4), B.make_linear_bwd(yg, G.w, G.ws, dxg)
    work, workg = (torch.empty(B.bq_linear_bwd_workspace_bytes(v), dtype=torch.uint8, device=DEV) for v in (b, bg))
    outs = [codes, xs, y, yg, dx, dxg]

    def sequence():
        B.bq_rows_quant8(x, codes, xs)
        B.bq_linear_fwd(codes, xs, L.w, L.ws, None, y, d)
        B.bq_linear_grouped_fwd(codes, xs, G.w, G.ws, None, off, yg, dg)
        B.bq_linear_bwd(y, L.w, L.ws, dx, work, b)
        B.bq_linear_grouped_bwd(yg, G.w, G.ws, off, dxg, workg, bg)

    sequence()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        sequence()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            sequence()
    torch.cuda.synchronize()
    for _ in range(3):
        for o in outs[:3] + outs[4:5]:
            o.fill_(3)
        yg[:180].fill_(3)
        dxg[:180].fill_(3)
        work.fill_(0xA5)
        workg.fill_(0xA5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)
        sequence()
        torch.cuda.synchronize()


def test_calls_go_to_the_stream_they_are_given():
    rng = np.random.default_rng(14)
    L = Layer(rng, 33, 64, 128, dtype="f32")
    want = L.forward()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y = torch.zeros_like(want)
    d = B.make_linear(L.x, L.w, L.ws, y)
    with torch.cuda.stream(side):
        B.bq_linear_fwd(L.x, L.xs, L.w, L.ws, None, y, d)
    side.synchronize()
    assert torch.equal(y, want)
    y.zero_()
    torch.cuda.synchronize()
    B.bq_linear_fwd(L.x, L.xs, L.w, L.ws, None, y, d, stream=side)
    side.synchronize()
    assert torch.equal(y, want)


def test_two_streams_at_once():
    rng = np.random.default_rng(15)
    layers = [Layer(rng, 300, 512, 1024, dtype="bf16", wbits=w) for w in (8, 4)]
    dys = [_gradient(rng, 300, 512, "bf16") for _ in layers]
    want = [(L.forward(), L.backward(g)) for L, g in zip(layers, dys)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    got = [[], []]
    for _ in range(4):
        for i, (L, g, s) in enumerate(zip(layers, dys, streams)):
            with torch.cuda.stream(s):
                got[i].append((L.forward(), L.backward(g)))
    torch.cuda.synchronize()
    for i, w in enumerate(want):
        for y, dx in got[i]:
            assert torch.equal(y, w[0]) and torch.equal(dx, w[1])


# ---- batches that take the large tiles: references in 64 bits on the device ------------------------------


def _codes_on_device(gen, shape, bits):
    q = torch.randint(-(1 << (bits - 1)), 1 << (bits - 1), shape, generator=gen, device=DEV)
    per = 8 // bits
    f = (q & ((1 << bits) - 1)).unflatten(-1, (shape[-1] // per, per))
    byte = sum(f[..., j] << (bits * j) for j in range(per))
    return q.double(), torch.where(byte > 127, byte - 256, byte).to(torch.int8)


def _within(got, want, bound):
    err = (got.double() - want).abs()
    assert (err <= bound).all(), f"{(~(err <= bound)).sum().item()} beyond the bound, the worst by {(err / bound).max().item():.3g}"


@pytest.mark.parametrize("xbits,wbits,K", [(8, 8, 208), (8, 4, 416), (8, 2, 192), (4, 8, 160), (4, 4, 1056), (4, 2, 320)])
@pytest.mark.parametrize("experts", [0, 5])
def test_large_tiles_fwd(xbits, wbits, K, experts):
    T, N = (4357, 4200) if not experts else (9001, 2300)
    gen = torch.Generator(device=DEV).manual_seed(K + experts)
    offsets = [3, 1500, 1500, 1501, 7000, 8990] if experts else [0, T]
    E = max(1, experts)
    qx, x = _codes_on_device(gen, (T, K), xbits)
    qw, w = _codes_on_device(gen, (E, N, K), wbits)
    xs, ws = (torch.rand(s, generator=gen, device=DEV) * 0.01 + 1e-3 for s in ((T,), (E, N)))
    bias = torch.randn((E, N), generator=gen, device=DEV).bfloat16()
    for dtype in ("bf16", "f32"):
        b = bias.to(TORCH[dtype])
        y = torch.full((T, N), 3.0, dtype=TORCH[dtype], device=DEV)
        if experts:
            B.bq_linear_grouped_fwd(x, xs, w, ws, b, lu.offsets_tensor(offsets), y, B.make_linear(x, w, ws, y, xbits=xbits, wbits=wbits))
        else:
            B.bq_linear_fwd(x, xs, w[0], ws[0], b[0], y, B.make_linear(x, w[0], ws[0], y, xbits=xbits, wbits=wbits))
        for e in range(E):
            lo, hi = offsets[e], offsets[e + 1]
            p = (qx[lo:hi] @ qw[e].t()) * xs[lo:hi, None].double() * ws[e].double()
            want = p + b[e].double()
            f32 = 5 * 2.0 ** -24 * (p.abs() + b[e].double().abs())
            _within(y[lo:hi], want, f32 + (lu.half_step(dtype) * (want.abs() + f32) if dtype != "f32" else 0) + 1e-40)
        assert (y[:offsets[0]] == 3).all() and (y[offsets[-1]:] == 3).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("experts", [0, 5])
def test_large_tiles_bwd(dtype, experts):
    T, N, K = (4357, 200, 4200) if not experts else (9001, 136, 2300)
    gen = torch.Generator(device=DEV).manual_seed(experts + 1)
    offsets = [3, 1500, 1500, 1501, 7000, 8990] if experts else [0, T]
    E = max(1, experts)
    qw, w = _codes_on_device(gen, (E, N, K), 4)
    ws = torch.rand((E, N), generator=gen, device=DEV) * 0.01 + 1e-3
    dy = (torch.randn((T, N), generator=gen, device=DEV) * torch.exp(torch.randn((T, 1), generator=gen, device=DEV))).to(TORCH[dtype])
    dx = torch.full((T, K), 3.0, dtype=TORCH[dtype], device=DEV)
    wd, wsd = (w, ws) if experts else (w[0], ws[0])
    d = B.make_linear_bwd(dy, wd, wsd, dx, wbits=4)
    work = torch.full((B.bq_linear_bwd_workspace_bytes(d),), 0xA5, dtype=torch.uint8, device=DEV)
    if experts:
        B.bq_linear_grouped_bwd(dy, wd, wsd, lu.offsets_tensor(offsets), dx, work, d)
    else:
        B.bq_linear_bwd(dy, wd, wsd, dx, work, d)
    term = 0.5 / lu.QMAX[3 if dtype == "f32" else 2] + 5 * 2.0 ** -24
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        if lo == hi:
            continue
        v = dy[lo:hi].double() * ws[e].double()
        want = v @ qw[e]
        f32 = term * v.abs().amax(1, keepdim=True) * qw[e].abs().sum(0) + 2 * 2.0 ** -24 * want.abs()
        _within(dx[lo:hi], want, f32 + (lu.half_step(dtype) * (want.abs() + f32) if dtype != "f32" else 0) + 1e-40)
    assert (dx[:offsets[0]] == 3).all() and (dx[offsets[-1]:] == 3).all()


@pytest.mark.parametrize("rows,cols", [((4 << 21) + 5, 8), ((2 << 20) + 3, 1032)])
def test_rows_quant8_of_more_rows_than_workgroups(rows, cols):
    x = torch.randn((rows, cols), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV, dtype=torch.bfloat16)
    codes, scales = B.alloc_rows_quant8(rows, cols, "f32", DEV)
    codes.fill_(99)
    B.bq_rows_quant8(x, codes, scales)
    for a in range(0, rows, 1 << 19):
        v = x[a:a + (1 << 19)].float()
        s = (v.abs().amax(1).double() / 127.0).float()
        assert torch.equal(scales[a:a + (1 << 19)], s)
        assert torch.equal(codes[a:a + (1 << 19)], torch.round(v * (1.0 / s.double()).float()[:, None]).clamp_(-128, 127).to(torch.int8))


# ---- every kernel that a product may take: batches of every size, odd numbers of tokens and channels, a short last step ----------------


def _ragged(T, experts):
    """Experts of uneven sizes, some empty, and rows of none at both ends."""
    cuts = np.sort(np.random.default_rng([T, experts]).integers(min(1, T), T + 1, size=experts + 1))
    cuts[experts // 2] = cuts[experts // 2 + 1]
    return [int(c) for c in cuts]


BATCHES_FWD = [(1, 18, 64, 0), (3, 1500, 64, 3), (115, 520, 64, 0), (200, 650, 64, 0), (830, 140, 64, 3), (45, 200, 64, 50), (500, 1000, 64, 0), (150, 200, 64, 3),
               (115, 2050, 64, 0), (450, 2050, 64, 0), (187, 520, 64, 3), (115, 1500, 64, 3), (115, 4100, 64, 0), (380, 330, 64, 0), (390, 4100, 832, 0),
               (200, 20000, 64, 3), (300, 20000, 64, 3), (4100, 2050, 64, 50), (4096, 16, 64, 64)]
BATCHES_BWD = [(1, 18, 0), (150, 200, 3), (200, 330, 0), (200, 300, 3), (700, 200, 0), (600, 200, 0), (830, 780, 0), (450, 520, 0), (390, 650, 0),
               (420, 1500, 0), (4100, 520, 50), (600, 6000, 3), (600, 6008, 3), (4100, 780, 50), (4096, 16, 64)]


@pytest.mark.parametrize("xbits,wbits", BITS)
@pytest.mark.parametrize("T,N,K,experts", BATCHES_FWD)
def test_batches_fwd(T, N, K, experts, xbits, wbits):
    gen = torch.Generator(device=DEV).manual_seed(T + N)
    E, offsets = max(1, experts), _ragged(T, experts) if experts else [0, T]
    qx, x = _codes_on_device(gen, (T, K), xbits)
    qw, w = _codes_on_device(gen, (E, N, K), wbits)
    xs, ws = (torch.rand(s, generator=gen, device=DEV) * 0.01 + 1e-3 for s in ((T,), (E, N)))
    b = torch.randn((E, N), generator=gen, device=DEV)
    y = torch.full((T, N), 3.0, device=DEV)
    if experts:
        B.bq_linear_grouped_fwd(x, xs, w, ws, b, lu.offsets_tensor(offsets), y, B.make_linear(x, w, ws, y, xbits=xbits, wbits=wbits))
    else:
        B.bq_linear_fwd(x, xs, w[0], ws[0], b[0], y, B.make_linear(x, w[0], ws[0], y, xbits=xbits, wbits=wbits))
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        p = (qx[lo:hi] @ qw[e].t()) * xs[lo:hi, None].double() * ws[e].double()
        _within(y[lo:hi], p + b[e].double(), 5 * 2.0 ** -24 * (p.abs() + b[e].double().abs()) + 1e-40)
    assert (y[:offsets[0]] == 3).all() and (y[offsets[-1]:] == 3).all()


def _check_bwd(T, N, K, experts, wbits, dtype, scale, seed, pad_w=0, pad_dx=0, shift=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    E, offsets = max(1, experts), _ragged(T, experts) if experts else [0, T]
    qw, w = _codes_on_device(gen, (E, N, K), wbits)
    ws = (torch.rand((E, N), generator=gen, device=DEV) * 0.01 + 1e-3).to(TORCH[scale])
    dy = (torch.randn((T, N), generator=gen, device=DEV) * torch.exp(torch.randn((T, 1), generator=gen, device=DEV))).to(TORCH[dtype])
    if shift:  # rows and scales that start at any element
        dy = lu.strided(dy, 3, shift)
        ws = lu.strided(ws.reshape(1, -1), 0, shift).view(E, N)
    w = torch.cat([w, torch.full((E, N, pad_w), 7, dtype=torch.int8, device=DEV)], 2)[..., :w.shape[2]]
    padded = torch.full((T, K + pad_dx), 3.0, dtype=TORCH[dtype], device=DEV)
    dx = padded[:, :K]
    wd, wsd = (w, ws) if experts else (w[0], ws[0])
    d = B.make_linear_bwd(dy, wd, wsd, dx, wbits=wbits)
    work = torch.full((B.bq_linear_bwd_workspace_bytes(d),), 0xA5, dtype=torch.uint8, device=DEV)
    if experts:
        B.bq_linear_grouped_bwd(dy, wd, wsd, lu.offsets_tensor(offsets), dx, work, d)
    else:
        B.bq_linear_bwd(dy, wd, wsd, dx, work, d)
    term = 0.5 / lu.QMAX[3 if dtype == "f32" else 2] + 5 * 2.0 ** -24
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        if lo == hi:
            continue
        v = dy[lo:hi].double() * ws[e].double()
        want = v @ qw[e]
        f32 = term * v.abs().amax(1, keepdim=True) * qw[e].abs().sum(0) + 2 * 2.0 ** -24 * want.abs()
        _within(dx[lo:hi], want, f32 + (lu.half_step(dtype) * (want.abs() + f32) + lu.smallest(dtype) if dtype != "f32" else 0) + 1e-40)
    assert (dx[:offsets[0]] == 3).all() and (dx[offsets[-1]:] == 3).all() and (padded[:, K:] == 3).all()


# as many rows as make it worth while to read the weights as they lie: the sum's length and the inputs around tiles' ends, the smallest sums
ACROSS = [(19, 10, 20000, 0, 0), (300, 520, 2080, 0, 16), (115, 10, 20000, 3, 0), (150, 10, 20000, 3, 32), (4100, 10, 544, 50, 0), (700, 1100, 1568, 0, 48),
          (1000, 130, 672, 3, 0), (255, 777, 992, 0, 0), (2040, 384, 256, 0, 16), (3000, 1, 288, 0, 0), (999, 128, 2336, 3, 0), (513, 129, 1056, 0, 0),
          (300, 520, 2112, 0, 16), (700, 1100, 1600, 0, 48), (1000, 130, 704, 3, 0), (255, 777, 1024, 0, 0), (4100, 10, 576, 50, 0), (19, 10, 20032, 0, 0),
          (115, 10, 20032, 3, 0), (150, 10, 20032, 3, 32), (600, 1024, 4096, 0, 0), (350, 640, 1536, 0, 0)]


@pytest.mark.parametrize("wbits", [8, 4, 2])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,N,K,experts,pad_w", ACROSS)
def test_bwd_on_weights_as_they_lie(T, N, K, experts, pad_w, dtype, wbits):
    _check_bwd(T, N, K, experts, wbits, dtype, "f32", T + N + K, pad_w=pad_w, pad_dx=5 if T % 2 else 8)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,N,K", [(33, 7, 40), (5, 500, 96), (70, 1003, 130), (300, 4096, 256), (9, 16384, 48), (12, 16390, 64)])
def test_bwd_of_rows_that_start_anywhere(T, N, K, dtype):
    for shift, experts in ((1, 0), (5, 3)):
        _check_bwd(T, N, K, experts, 8, dtype, "f16" if shift == 1 else "f32", T + N, shift=shift)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("T,K,experts", BATCHES_BWD)
def test_batches_bwd(T, K, experts, dtype):
    _check_bwd(T, 640 if K == 1500 else 72, K, experts, 8, dtype, "f32", T + K)


@pytest.mark.parametrize("wbits", [8, 4, 2])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N", [104, 2048, 2056, 4104, 8200, 16384, 16392, 1001, 2501, 7999, 16001, 16385])
def test_bwd_of_wide_layers(N, dtype, wbits):
    # rows of digits from one piece of a workgroup to the widest that stay in registers, and those that do not
    _check_bwd(5, N, 48, 0, wbits, dtype, "f16" if N % 3 else "f32", N)
    _check_bwd(37, N, 80, 4, wbits, dtype, "f32" if N % 3 else "f16", N + 1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N", [512, 1032, 2504, 8000, 16376, 505, 1411, 4095, 5063, 16383, 16400])
def test_bwd_of_wide_layers_on_weights_as_they_lie(N, dtype):
    _check_bwd(700, N, 1056, 0, 8, dtype, "f16", N)
    _check_bwd(390, N, 1056, 3, 4, dtype, "f32", N + 1)


def test_bwd_of_more_rows_than_workgroups():
    _check_bwd(4096 * 2 + 77, 256, 64, 0, 8, "bf16", "f32", 1)
    _check_bwd(4096 * 2 + 77, 250, 64, 3, 4, "f16", "f32", 2)
    _check_bwd(16384 * 2 + 77, 256, 128, 0, 8, "bf16", "f32", 3)
    _check_bwd(16384 * 2 + 77, 1024, 128, 3, 4, "f32", "f32", 4)


# ---- places beyond 2^32 ---------------------------------------------------------------------------------


def _spread(a, ld):
    """A device tensor with a's values whose rows lie ld elements apart."""
    buf = torch.empty((a.shape[0] - 1) * ld + a.shape[1], dtype=a.dtype, device=DEV)
    v = buf.as_strided(a.shape, (ld, 1))
    v.copy_(a)
    return v


def test_rows_quant8_beyond_32_bits():
    a = torch.randn(6, 520, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    want, scales = B.alloc_rows_quant8(6, 520, "f32", DEV)
    B.bq_rows_quant8(a, want, scales)
    x, codes, got = _spread(a, (1 << 30) - 24), _spread(torch.zeros_like(want), (1 << 30) - 8), torch.empty_like(scales)
    B.bq_rows_quant8(x, codes, got)
    assert torch.equal(codes, want) and torch.equal(got, scales)


@pytest.mark.parametrize("bits", [(8, 8), (4, 2)])
@pytest.mark.parametrize("T,N,ld_x,ld_w,ld_y", [(1100, 40, 1 << 22, 64, 64), (1300, 2200, 1 << 22, 1 << 21, 1 << 21), (40, 1500, 64, 1 << 22, 1 << 21),
                                                (6, 5, 1 << 30, 64, 1 << 29), (6, 5, 64, 1 << 30, 8)])
def test_linear_fwd_beyond_32_bits(T, N, ld_x, ld_w, ld_y, bits):
    L = Layer(np.random.default_rng([T, N]), T, N, 64, xbits=bits[0], wbits=bits[1], dtype="f32", bias=True)
    want, size = lu.reference_fwd(L.qx, L.xs, L.qw, L.ws, L.bias, [0, T])
    L.x, L.w = _spread(L.x, ld_x), _spread(L.w, ld_w)
    y = _spread(torch.full((T, N), 3.0, device=DEV), ld_y)
    B.bq_linear_fwd(L.x, L.xs, L.w, L.ws, L.bias, y, B.make_linear(L.x, L.w, L.ws, y, xbits=bits[0], wbits=bits[1], inputs=64))
    lu.check(lu.f64(y), want, lu.bound_fwd(want, size, "f32"), f"{bits}")


@pytest.mark.parametrize("T,N,K,ld_y,ld_x", [(9, 200, 48, 1 << 30, 1 << 29), (1100, 136, 96, 1 << 22, 1 << 21)])
def test_linear_bwd_rows_beyond_32_bits(T, N, K, ld_y, ld_x):
    rng = np.random.default_rng([T, N, K])
    L = Layer(rng, T, N, K, dtype="bf16")
    dy = _gradient(rng, T, N, "bf16")
    want, weight, top = lu.reference_bwd(dy, L.qw, L.ws, [0, T])
    dy, dx = _spread(dy, ld_y), _spread(torch.full((T, K), 3.0, dtype=torch.bfloat16, device=DEV), ld_x)
    d = B.make_linear_bwd(dy, L.w, L.ws, dx)
    B.bq_linear_bwd(dy, L.w, L.ws, dx, torch.empty(B.bq_linear_bwd_workspace_bytes(d), dtype=torch.uint8, device=DEV), d)
    lu.check(lu.f64(dx), want, lu.bound_bwd(want, weight, top, "bf16"), "dx")


def test_linear_bwd_workspace_beyond_32_bits():
    # the digits of 600000 rows of 4096, then 70 experts whose transposed weights fill 4.7 GB, of which two have rows
    _check_bwd(600000, 4096, 64, 0, 4, "bf16", "f32", 5)
    E, N, K, T = 70, 8192, 8192, 24
    gen = torch.Generator(device=DEV).manual_seed(6)
    w = torch.randint(-128, 128, (E, N, K), generator=gen, device=DEV, dtype=torch.int8)
    ws = torch.rand((E, N), generator=gen, device=DEV) * 0.01 + 1e-3
    dy = torch.randn((T, N), generator=gen, device=DEV).bfloat16()
    offsets = [0] + [9] * 68 + [9, T]
    dx = torch.full((T, K), 3.0, dtype=torch.bfloat16, device=DEV)
    d = B.make_linear_bwd(dy, w, ws, dx)
    assert B.bq_linear_bwd_workspace_bytes(d) > 1 << 32
    work = torch.empty(B.bq_linear_bwd_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    B.bq_linear_grouped_bwd(dy, w, ws, lu.offsets_tensor(offsets), dx, work, d)
    for e, lo, hi in ((0, 0, 9), (E - 1, 9, T)):
        v, q = dy[lo:hi].double() * ws[e].double(), w[e].double()
        want = v @ q
        f32 = (0.5 / lu.QMAX[2] + 5 * 2.0 ** -24) * v.abs().amax(1, keepdim=True) * q.abs().sum(0) + 2 * 2.0 ** -24 * want.abs()
        _within(dx[lo:hi], want, f32 + lu.half_step("bf16") * (want.abs() + f32) + 1e-40)
