"""Products in 8-bit integers, the experts' products, routing and combination: refusals (on the CPU), and results against plain
implementations in 64 bits.  The tolerances follow from the number of roundings, and are zero where the steps are prescribed."""
import ctypes as C
import math
import sys
import types

import numpy as np
import pytest
import torch

from paper_2605_26339_amd import qamw

gpu = pytest.mark.gpu
DEV = "cuda"


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# ------------------------------------------------------------------------------------------------------------ refusals


def _p(n=64):
    """A pointer that is never followed: every refusal comes before a launch."""
    return 1 << 20


def test_refusals_of_the_entry_points():
    L, I, S, U = qamw.lib(), qamw.ERR_INVALID_ARG, qamw.ERR_SHAPE, qamw.ERR_UNSUPPORTED
    p = _p()

    def quant(X=p, dtype=0, m=4, d=8, ldx=8, cs=None, codes=p, ldc=8, scales=p):
        return L.qamw_int8_quantize(X, dtype, m, d, ldx, cs, codes, ldc, scales, None)

    assert quant(X=None) == I and quant(codes=None) == I and quant(scales=None) == I
    assert quant(dtype=2) == I and quant(dtype=-1) == I and quant(m=-1) == I and quant(m=(1 << 22) + 1) == I and quant(d=0) == I
    assert quant(X=p + 2) == I and quant(scales=p + 2) == I and quant(cs=p + 1) == I
    assert quant(ldx=7) == S and quant(ldc=7) == S
    assert quant(m=0, X=None, codes=None, scales=None) == qamw.OK

    need = C.c_size_t()
    size = lambda t, m, n, k, g=0: L.qamw_int8_matmul_workspace_bytes(t, m, n, k, g, C.byref(need))  # noqa: E731
    assert size(0, 3, 8, 17) == qamw.OK and need.value == 3 * 32 + 16
    assert size(2, 3, 8, 17) == qamw.OK and need.value == 0
    assert size(2, 500, 2048, 13824) == qamw.OK and need.value > 0 and need.value % (500 * 2048 * 4) == 0   # the sums of parts
    assert size(2, 500, 2049, 13824, 1) == qamw.OK and need.value % (500 * 4104 * 4) == 0 and need.value > 0   # read by fours from column 2049 on: 4101 to the next four
    assert size(3, 3, 8, 17) == I and size(0, 3, 8, 131057) == I and size(0, 3, 0, 17) == I and size(0, 3, 8, 17, 2) == I
    assert L.qamw_int8_matmul_workspace_bytes(0, 3, 8, 17, 0, None) == I

    def mm(X=p, xt=2, xs=p, cs=None, m=4, ldx=8, W=p, ws=p, ldw=8, d_out=8, d_in=8, gated=0, Y=p, yt=1, ldy=8, work=None, n=0):
        return L.qamw_int8_matmul(X, xt, xs, cs, m, ldx, W, ws, ldw, d_out, d_in, gated, Y, yt, ldy, work, n, None)

    assert mm(X=None) == I and mm(W=None) == I and mm(ws=None) == I and mm(Y=None) == I and mm(xs=None) == I
    assert mm(xt=3) == I and mm(yt=2) == I and mm(gated=2) == I and mm(d_out=0) == I and mm(d_in=0) == I and mm(m=-1) == I
    assert mm(cs=p) == I                                                   # codes are not scaled again
    assert mm(xt=1, xs=p, work=p, n=1 << 20) == I                          # nor do floats come with scales
    assert mm(xt=1, xs=None, work=None, n=0) == I and mm(xt=1, xs=None, work=p, n=79) == I and mm(xt=1, xs=None, work=p + 8, n=1 << 20) == I
    assert mm(ldx=7) == S and mm(ldw=7) == S and mm(ldy=7) == S
    assert mm(Y=p + 1) == I and mm(xs=p + 2) == I and mm(ws=p + 2) == I
    assert mm(m=0, X=None, xs=None, W=None, ws=None, Y=None) == qamw.OK
    assert mm(m=1 << 22, d_out=1 << 24, ldy=1 << 24) == U                  # more tiles than a launch has

    def grouped(X=p, t=1, xs=None, xr=4, ldx=8, rows=None, W=p, ws=None, ldw=8, es=64, off=p, n=2, m=4, d_out=8, d_in=8, gated=0, Y=p, yt=1, ldy=8):
        return L.qamw_grouped_matmul(X, t, xs, xr, ldx, rows, W, ws, ldw, es, off, n, m, d_out, d_in, gated, Y, yt, ldy, None)

    assert grouped(t=0) == I and grouped(t=3) == I and grouped(yt=2) == I and grouped(n=0) == I and grouped(n=1025) == I
    assert grouped(X=None) == I and grouped(W=None) == I and grouped(off=None) == I and grouped(Y=None) == I
    assert grouped(xs=p) == I and grouped(ws=p) == I and grouped(t=2) == I and grouped(t=2, xs=p) == I
    assert grouped(X=p + 1) == I and grouped(W=p + 1) == I and grouped(rows=p + 2) == I and grouped(off=p + 1) == I
    assert grouped(ldx=7) == S and grouped(ldw=7) == S and grouped(ldy=7) == S and grouped(es=-1) == S and grouped(xr=3) == S
    assert grouped(rows=p, xr=0) == S
    assert grouped(m=0, X=None, W=None, off=None, Y=None) == qamw.OK

    assert L.qamw_route_workspace_bytes(4, 8, 2, None) == I and L.qamw_route_workspace_bytes(4, 8, 9, C.byref(need)) == I

    def route(x=p, t=0, m=4, n=8, ld=8, k=2, re=1, e=p, w=p, off=p, rows=p, pos=p, work=p, size=1 << 20):
        return L.qamw_route(x, t, m, n, ld, k, re, e, w, off, rows, pos, work, size, None)

    assert route(t=2) == I and route(k=0) == I and route(k=9) == I and route(n=64, ld=64, k=33) == I and route(n=1025, ld=1025) == I
    assert route(re=2) == I and route(x=None) == I and route(e=None) == I and route(w=None) == I and route(off=None) == I
    assert route(rows=None) == I and route(pos=None) == I and route(m=100, work=None) == I and route(m=100, size=63) == I and route(m=100, work=p + 4) == I
    assert route(ld=7) == S and route(m=-1) == I and route(off=p + 2) == I

    def comb(Y=p, t=1, yr=8, ldy=8, pos=p, w=p, m=4, k=2, d=8, out=p, ot=1, ldo=8):
        return L.qamw_combine(Y, t, yr, ldy, pos, w, m, k, d, out, ot, ldo, None)

    assert comb(Y=None) == I and comb(pos=None) == I and comb(w=None) == I and comb(out=None) == I and comb(t=2) == I and comb(ot=2) == I
    assert comb(k=0) == I and comb(k=33) == I and comb(d=0) == I and comb(yr=-1) == I and comb(ldy=7) == S and comb(ldo=7) == S
    assert comb(m=0, Y=None, pos=None, w=None, out=None) == qamw.OK


def test_refusals_of_the_binding(monkeypatch):
    monkeypatch.setattr(qamw, "_one_device", lambda *t: 0)
    x8, w8, s = torch.zeros(4, 8, dtype=torch.int8), torch.zeros(6, 8, dtype=torch.int8), torch.ones(6)
    with pytest.raises(ValueError):
        qamw.int8_matmul(x8, w8[:, :7], s, x_scales=torch.ones(4))
    with pytest.raises(ValueError):
        qamw.int8_matmul(x8, w8, s[:5], x_scales=torch.ones(4))
    with pytest.raises(ValueError):
        qamw.int8_matmul(x8, w8, s, x_scales=torch.ones(3))
    with pytest.raises(ValueError):
        qamw.int8_matmul(x8, w8[:5], s[:5], x_scales=torch.ones(4), gated=True)
    with pytest.raises(ValueError):
        qamw.int8_matmul(x8.t(), w8, s, x_scales=torch.ones(4))
    with pytest.raises(TypeError):
        qamw.int8_matmul(x8.to(torch.float16), w8, s)
    with pytest.raises(ValueError):
        qamw.int8_matmul(x8, w8, s, x_scales=torch.ones(4), out=torch.zeros(4, 5))
    off = torch.zeros(3, dtype=torch.int32)
    we = torch.zeros(2, 6, 8, dtype=torch.int8)
    with pytest.raises(TypeError):
        qamw.grouped_matmul(x8.bfloat16(), we, off)
    with pytest.raises(ValueError):
        qamw.grouped_matmul(x8, we, off[:2], x_scales=torch.ones(4), w_scales=torch.ones(2, 6))
    with pytest.raises(ValueError):
        qamw.grouped_matmul(x8, we, off.long(), x_scales=torch.ones(4), w_scales=torch.ones(2, 6))
    with pytest.raises(qamw.QamwError):
        qamw.grouped_matmul(x8, we, off, w_scales=torch.ones(2, 6), out=torch.zeros(4, 6), stream=types.SimpleNamespace(cuda_stream=0))   # codes without scales
    with pytest.raises(qamw.QamwError):
        qamw.route(torch.zeros(3, 4), 5)
    with pytest.raises(ValueError):
        qamw.combine(torch.zeros(4, 8), torch.zeros(2, 2, dtype=torch.int64), torch.zeros(2, 2))
    with pytest.raises(ValueError):
        qamw.int8_quantize(x8.float(), col_scale=torch.ones(7))


# ---------------------------------------------------------------------------------------------------------- quantisation


def quantise_ref(x, col_scale=None):
    """The steps of the definition in numpy's fp32, which rounds every one of them once."""
    v = x.float().numpy()
    if col_scale is not None:
        v = v * col_scale.numpy()
    a = np.abs(v).max(axis=1)
    some = np.isfinite(v).all(axis=1) & (a >= np.float32(2.0**-110))
    with np.errstate(all="ignore"):
        inv = np.float32(127) / a
        codes = np.where(some[:, None], np.rint(v * inv[:, None]), 0).astype(np.int8)
        scales = np.where(some, a / np.float32(127), np.where(np.isfinite(v).all(axis=1), np.float32(0), np.float32(np.nan)))
    return codes, scales.astype(np.float32)


def _strided(t, pad, skip=0):
    """The values of t [..., d] on the device in rows of d + pad elements that begin `skip` elements into an allocation; what
    lies between holds NaNs or 77."""
    flat = torch.full((t[..., 0].numel() * (t.shape[-1] + pad) + skip + pad,), float("nan") if t.is_floating_point() else 77, dtype=t.dtype, device=DEV)
    lead, st = t.shape[:-1], [1]
    ld = t.shape[-1] + pad
    for n in reversed(lead):
        st.insert(0, ld)
        ld *= n
    v = torch.as_strided(flat, t.shape, st, skip)
    v.copy_(t)
    return v


@gpu
@pytest.mark.parametrize("m,d,dtype,pad,skip,smooth", [
    (1, 1, torch.float32, 0, 0, False), (3, 5, torch.bfloat16, 0, 0, True), (1, 4096, torch.bfloat16, 0, 0, False),
    (7, 257, torch.float32, 0, 0, True), (5, 512, torch.bfloat16, 8, 0, True), (5, 512, torch.bfloat16, 3, 1, False), (300, 1024, torch.float32, 4, 4, True),
    (9, 2048, torch.bfloat16, 0, 0, True), (4, 5632, torch.float32, 0, 0, False), (6, 8208, torch.bfloat16, 0, 0, True),
    (3, 13824, torch.bfloat16, 16, 8, False), (2, 16400, torch.float32, 0, 0, True), (2, 40000, torch.bfloat16, 0, 0, True), (1, 131056, torch.float32, 0, 0, False),
    (2, 16384, torch.float32, 1, 1, True), (70000, 16, torch.bfloat16, 0, 0, False),
])
def test_quantise(m, d, dtype, pad, skip, smooth):
    say(f"[quantise] {m}x{d} {dtype} pad {pad} skip {skip} smooth {smooth}")
    g = _gen(m * 7 + d)
    x = (torch.randn(m, d, generator=g) * torch.exp(torch.randn(m, 1, generator=g))).to(dtype)
    x[m // 2, d // 2] = 9.0
    c = torch.exp(0.5 * torch.randn(d, generator=g)) if smooth else None
    codes = _strided(torch.zeros(m, d, dtype=torch.int8), pad, skip)
    scales = torch.empty(m, device=DEV)
    qamw.int8_quantize(_strided(x, pad, skip), None if c is None else c.to(DEV), out=(codes, scales))
    want, want_s = quantise_ref(x, c)
    assert np.array_equal(codes.cpu().numpy(), want)
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.abs(want).max() == 127
    if pad:
        whole = torch.as_strided(codes, (m, d + pad), codes.stride(), codes.storage_offset())
        assert (whole[:, d:] == 77).all()                      # what lies between the rows is left alone


@gpu
@pytest.mark.parametrize("d", [64, 100, 4096, 20000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantise_special_rows(d, dtype):
    say(f"[quantise] special rows {d} {dtype}")
    g = _gen(d)
    x = torch.randn(12, d, generator=g)
    x[0] = 0
    x[1] = -0.0
    x[2] *= 2.0**-112                                     # below the limit, some entries above it times 4
    x[2].clamp_(-(2.0**-111), 2.0**-111)
    x[3] *= 2.0**-112
    x[3, 1] = -(2.0**-110)
    x[4, d - 1] = math.inf
    x[5, 0] = -math.inf
    x[6, d // 2] = math.nan
    x[7, 3] = 3.0e38
    x[8] = 1.0e-41                                        # subnormal
    x[9] = 0.5                                            # every code on a tie or none: 127 and 63.5
    x[9, 0] = 1.0
    x[10, 1:] = 0
    x[11, 0], x[11, 1] = math.inf, math.nan
    x = x.to(dtype)
    codes, scales = qamw.int8_quantize(x.to(DEV))
    want, want_s = quantise_ref(x)
    assert np.array_equal(codes.cpu().numpy(), want)
    assert np.array_equal(scales.cpu().numpy(), want_s, equal_nan=True)
    assert np.isnan(want_s[[4, 5, 6, 11]]).all() and (want_s[[0, 1, 2, 8]] == 0).all() and want_s[3] > 0
    # a row that is not finite makes its product NaN and no other row's
    W = torch.randint(-127, 128, (20, d), generator=g).to(torch.int8)
    y = qamw.int8_matmul(x.to(DEV), W.to(DEV), torch.ones(20, device=DEV), out_dtype=torch.float32).cpu()
    assert torch.isnan(y[[4, 5, 6, 11]]).all() and torch.isfinite(y[[0, 1, 2, 3, 8, 9, 10]]).all() and (y[[0, 1, 2, 8]] == 0).all()


# -------------------------------------------------------------------------------------------------------------- products


def _codes(g, *shape):
    c = torch.randint(-127, 128, shape, generator=g).to(torch.int8)
    c.view(-1)[::5] = 127                                       # sums that need more than 24 bits
    return c


def int8_ref(x, xs, w, ws):
    """The exact sums, then the prescribed fp32 steps."""
    s = (x.double() @ w.double().t()).numpy()                   # below 2^53: exact
    return torch.from_numpy((s.astype(np.float32) * xs.numpy()[:, None]) * ws.numpy()[None, :])


def check(got, want, slack, what):
    """|got - want| <= slack, and half a unit of bf16 more where the result is rounded to that."""
    want, slack = want.double(), slack.double()
    if got.dtype == torch.bfloat16:
        slack = slack + (want.abs() + slack) * 2.0**-8
    off = (got.cpu().double() - want).abs()
    bad = ~(off <= slack)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float((off - slack).max())}"


def gate_ref(g, u, eg, eu):
    """silu(g) * u in 64 bits, and how far it may be off for errors eg, eu of its operands: |silu'| < 1.1; the exponential's
    argument is rounded, which its size multiplies, and a handful of roundings follow."""
    g, u = g.double(), u.double()
    s = g * torch.sigmoid(g)
    return s * u, 1.1 * eg * (u.abs() + eu) + s.abs() * eu + (s * u).abs() * (g.abs() + 16) * 2.0**-23 + 1e-37


SHAPES = [
    (1, 1, 1), (1, 17, 16), (2, 64, 100), (1, 4096, 4096), (3, 130, 1040), (8, 257, 2048), (15, 33, 5632), (16, 100, 528), (17, 31, 144), (31, 500, 272),
    (40, 2048, 1008), (64, 65, 4112), (65, 128, 64), (100, 700, 336), (129, 300, 1024), (200, 63, 15), (257, 513, 2064), (300, 260, 176), (513, 1030, 656),
    (700, 384, 128), (1000, 1600, 512), (33, 5, 13824),
]


@gpu
@pytest.mark.parametrize("m,d_out,d_in", SHAPES)
@pytest.mark.parametrize("gated", [False, True])
def test_int8_matmul_of_codes(m, d_out, d_in, gated):
    say(f"[int8] {m} x {d_out} x {d_in} gated {gated}")
    g = _gen(m * 3 + d_out * 5 + d_in)
    outs = d_out * (2 if gated else 1)
    x, w = _codes(g, m, d_in), _codes(g, outs, d_in)
    xs, ws = torch.rand(m, generator=g) / (127 * math.sqrt(d_in)) + 1e-5, (torch.rand(outs, generator=g) + 0.1) / 127
    dx, dw = x.to(DEV), w.to(DEV)
    y = qamw.int8_matmul(dx, dw, ws.to(DEV), x_scales=xs.to(DEV), gated=gated, out_dtype=torch.float32)
    b = qamw.int8_matmul(dx, dw, ws.to(DEV), x_scales=xs.to(DEV), gated=gated)
    assert y.shape == (m, d_out) and b.dtype == torch.bfloat16
    ref = int8_ref(x, xs, w, ws)
    if not gated:
        assert torch.equal(y.cpu(), ref)
        assert torch.equal(b.cpu(), ref.bfloat16())
    else:
        want, slack = gate_ref(ref[:, :d_out], ref[:, d_out:], 0.0, 0.0)
        check(y, want, slack, "fp32")
        assert torch.equal(b.cpu(), y.cpu().bfloat16())          # the same number, rounded


@gpu
@pytest.mark.parametrize("m,d_out,d_in,x_pad,w_pad,y_pad,skip", [
    (5, 100, 96, 16, 32, 3, 0), (5, 100, 96, 1, 0, 0, 0), (70, 130, 256, 16, 16, 8, 16), (70, 130, 256, 0, 5, 1, 3), (300, 270, 512, 32, 48, 2, 16), (300, 270, 512, 0, 0, 0, 1),
    (300, 270, 500, 0, 0, 1, 0), (1, 100, 4096, 0, 16, 0, 0), (600, 300, 384, 128, 0, 1, 0),
])
@pytest.mark.parametrize("x_dtype", [torch.int8, torch.float32, torch.bfloat16])
def test_int8_matmul_strides(m, d_out, d_in, x_pad, w_pad, y_pad, skip, x_dtype):
    """Leading dimensions and starts that are aligned or not; what lies between rows is neither used nor written."""
    say(f"[int8] strides {m} x {d_out} x {d_in} {x_dtype} pads {x_pad} {w_pad} {y_pad} skip {skip}")
    g = _gen(m + d_in + x_pad)
    w, ws = _codes(g, d_out, d_in), torch.rand(d_out, generator=g) / 127
    dw = _strided(w, w_pad, skip)
    out = _strided(torch.zeros(m, d_out), y_pad, skip % 4)
    if x_dtype == torch.int8:
        x, xs = _codes(g, m, d_in), torch.rand(m, generator=g)
        qamw.int8_matmul(_strided(x, x_pad, skip), dw, ws.to(DEV), x_scales=xs.to(DEV), out=out)
    else:
        f = (torch.randn(m, d_in, generator=g) * 3).to(x_dtype)
        c = torch.rand(d_in, generator=g) + 0.5
        codes, scales = quantise_ref(f, c)
        x, xs = torch.from_numpy(codes), torch.from_numpy(scales)
        qamw.int8_matmul(_strided(f, x_pad, skip), dw, ws.to(DEV), col_scale=c.to(DEV), out=out)
    assert torch.equal(out.cpu(), int8_ref(x, xs, w, ws))
    if y_pad:
        assert torch.isnan(torch.as_strided(out, (m, d_out + y_pad), out.stride(), out.storage_offset())[:, d_out:]).all()


@gpu
@pytest.mark.parametrize("m,d_out,d_in", [(1, 300, 512), (4, 300, 520), (13, 300, 5632), (50, 300, 1024), (300, 520, 768), (0, 20, 64), (16, 33, 4096), (5, 2048, 8192), (9, 1000, 528),
                                       (2, 50, 8192), (4, 70, 4096), (1, 40, 16384), (1, 40, 8208), (13, 4000, 4096), (16, 100, 8192)])
@pytest.mark.parametrize("x_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("smooth", [False, True])
def test_int8_matmul_quantises_as_the_quantiser_does(m, d_out, d_in, x_dtype, smooth):
    say(f"[int8] quantised in the call {m} x {d_out} x {d_in} {x_dtype} {smooth}")
    g = _gen(m + d_out + d_in)
    f = (torch.randn(m, d_in, generator=g) * torch.exp(torch.randn(m, 1, generator=g))).to(x_dtype)
    c = torch.rand(d_in, generator=g) + 0.5 if smooth else None
    w, ws = _codes(g, d_out, d_in), torch.rand(d_out, generator=g) / 127
    dc = None if c is None else c.to(DEV)
    y = qamw.int8_matmul(f.to(DEV), w.to(DEV), ws.to(DEV), col_scale=dc, out_dtype=torch.float32)
    codes, scales = qamw.int8_quantize(f.to(DEV), dc)
    z = qamw.int8_matmul(codes, w.to(DEV), ws.to(DEV), x_scales=scales, out_dtype=torch.float32)
    assert y.shape == (m, d_out) and torch.equal(y, z)
    if m:
        rc, rs = quantise_ref(f, c)
        assert torch.equal(y.cpu(), int8_ref(torch.from_numpy(rc), torch.from_numpy(rs), w, ws))


@gpu
@pytest.mark.parametrize("m,d_in,shift", [(1, 4096, 0), (4, 512, 0), (1, 16384, 0), (5, 512, 0), (2, 8192, 0), (3, 8192, 0), (1, 4088, 0), (1, 4096, 4)])
def test_int8_matmul_without_a_workspace(m, d_in, shift):
    """Rows that the product's own launch quantises need none; all others are refused without it, and nothing is written."""
    say(f"[int8] no workspace {m} x {d_in} shift {shift}")
    g = _gen(m + d_in)
    x = torch.randn(m * d_in + shift, generator=g).to(DEV)[shift // 4:][: m * d_in].view(m, d_in)
    w, ws = _codes(g, 100, d_in).to(DEV), (torch.rand(100, generator=g) / 127).to(DEV)
    y = torch.full((m, 100), 7.0, device=DEV)
    rc = qamw.lib().qamw_int8_matmul(x.data_ptr(), 0, None, None, m, d_in, w.data_ptr(), ws.data_ptr(), d_in, 100, d_in, 0, y.data_ptr(), 0, 100, None, 0,
                                     torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    if m * -(-d_in // 4096) <= 4 and d_in % 16 == 0 and shift == 0:
        assert rc == qamw.OK and torch.equal(y, qamw.int8_matmul(x.clone(), w, ws, out_dtype=torch.float32, workspace=torch.empty(1 << 20, dtype=torch.uint8, device=DEV)))
    else:
        assert rc == qamw.ERR_INVALID_ARG and (y == 7.0).all()
    c, s = qamw.int8_quantize(x)
    assert torch.equal(qamw.int8_matmul(x, w, ws, out_dtype=torch.float32), qamw.int8_matmul(c, w, ws, x_scales=s, out_dtype=torch.float32))


@gpu
@pytest.mark.parametrize("m,d_out,d_in", [(100, 2050, 13824), (500, 514, 13824), (129, 2049, 8192), (1000, 515, 4096), (1000, 515, 13824), (34, 8201, 12336)])
@pytest.mark.parametrize("gated", [False, True])
def test_int8_matmul_in_parts(m, d_out, d_in, gated):
    """Shapes whose columns are shared among workgroups: sums of parts, odd outputs, results in fp32 and bf16, a workspace of one's own."""
    say(f"[int8] parts {m} x {d_out} x {d_in} gated {gated}")
    g = _gen(m + d_in)
    outs = d_out * (2 if gated else 1)
    need = qamw.int8_matmul_workspace_bytes(qamw.DTYPE_I8, m, d_out, d_in, gated)
    assert need > m * outs * 4 or (need == 0 and (m, d_in) in ((129, 8192), (1000, 4096)))   # the kernel for few rows is as fast for these
    x, w, xs, ws = _codes(g, m, d_in), _codes(g, outs, d_in), torch.rand(m, generator=g) / (127 * math.sqrt(d_in)), (torch.rand(outs, generator=g) + 0.1) / 127
    guarded = torch.full((need + 256,), 77, dtype=torch.uint8, device=DEV)
    y = qamw.int8_matmul(x.to(DEV), w.to(DEV), ws.to(DEV), x_scales=xs.to(DEV), gated=gated, out_dtype=torch.float32, workspace=guarded[128:128 + need])
    b = qamw.int8_matmul(x.to(DEV), w.to(DEV), ws.to(DEV), x_scales=xs.to(DEV), gated=gated)
    assert (guarded[:128] == 77).all() and (guarded[128 + need:] == 77).all()
    ref = int8_ref(x, xs, w, ws)
    if gated:
        want, slack = gate_ref(ref[:, :d_out], ref[:, d_out:], 0.0, 0.0)
        check(y, want, slack, "fp32")
    else:
        assert torch.equal(y.cpu(), ref)
    assert torch.equal(b.cpu(), y.cpu().bfloat16())
    f = torch.randn(m, d_in, generator=g).bfloat16()              # codes and sums in one workspace
    z = qamw.int8_matmul(f.to(DEV), w.to(DEV), ws.to(DEV), gated=gated, out_dtype=torch.float32)
    c, s = qamw.int8_quantize(f.to(DEV))
    assert torch.equal(z, qamw.int8_matmul(c, w.to(DEV), ws.to(DEV), x_scales=s, gated=gated, out_dtype=torch.float32))


@gpu
def test_int8_sums_of_the_longest_rows():
    """127 * 127 * 131056 and 128 * 128 * 131056 stay within 32 bits."""
    d = 131056
    for v in (127, -127, -128):
        for m in (1, 20, 70):
            x, w = torch.full((m, d), v, dtype=torch.int8, device=DEV), torch.full((3, d), v, dtype=torch.int8, device=DEV)
            y = qamw.int8_matmul(x, w, torch.ones(3, device=DEV), x_scales=torch.ones(m, device=DEV), out_dtype=torch.float32)
            assert (y.cpu() == np.float32(v * v * d)).all()


def _offsets(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32)


def grouped_ref(x, w, offsets, rows, xs, ws, gated):
    """(result, slack) in 64 bits, for the rows that an expert has."""
    n, outs, d_in = w.shape
    m = int(offsets[-1])
    total, size = torch.zeros(m, outs, dtype=torch.float64), torch.zeros(m, outs, dtype=torch.float64)
    for e in range(n):
        a, b = int(offsets[e]), int(offsets[e + 1])
        if a == b:
            continue
        r = torch.arange(a, b) if rows is None else rows[a:b].long()
        if xs is not None:
            total[a:b] = int8_ref(x[r], xs[r], w[e], ws[e]).double()
        else:
            total[a:b] = x[r].double() @ w[e].double().t()
            size[a:b] = x[r].double().abs() @ w[e].double().abs().t()
    slack = size * d_in * 2.0**-23                              # one rounding an addition, in any order, of exact products
    if not gated:
        return total, slack
    h = outs // 2
    return gate_ref(total[:, :h], total[:, h:], slack[:, :h], slack[:, h:])


GROUPS = [
    ([1], 1, 1), ([0, 3, 0], 17, 16), ([1, 0, 2, 1, 1, 0, 0, 5], 96, 512), ([2] * 70, 33, 144), ([16, 17, 15, 0, 1], 130, 272), ([40, 0, 3, 64], 200, 1040),
    ([0] * 65 + [9] + [0] * 100 + [4], 50, 80), ([130, 0, 257, 1, 64], 300, 528), ([600, 3], 520, 384), ([0, 0, 1100], 260, 128), ([90, 80, 120, 100, 70, 110], 384, 256),
    ([0, 0], 40, 64), ([1] * 300, 20, 48), ([7, 300, 40], 77, 99), ([256, 512, 256], 512, 640), ([33] * 20, 48, 2048),
]


@gpu
@pytest.mark.parametrize("counts,d_out,d_in", GROUPS, ids=[str(i) for i in range(len(GROUPS))])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("gather", [False, True])
def test_grouped_matmul(counts, d_out, d_in, gated, i8, gather):
    say(f"[grouped] {sum(counts)} rows of {len(counts)} experts, {d_out} x {d_in} gated {gated} int8 {i8} gather {gather}")
    g = _gen(sum(counts) + d_out + d_in)
    n, m, outs = len(counts), sum(counts), d_out * (2 if gated else 1)
    spare = 5                                                   # rows that no expert has
    x_rows = m // 2 + 3 if gather else m + spare
    rows = torch.randint(0, x_rows, (m + spare,), generator=g).to(torch.int32) if gather else None
    if i8:
        x, w = _codes(g, x_rows, d_in), _codes(g, n, outs, d_in)
        xs, ws = torch.rand(x_rows, generator=g) / (127 * math.sqrt(d_in)) + 1e-5, (torch.rand(n, outs, generator=g) + 0.1) / 127
    else:
        x, w = torch.randn(x_rows, d_in, generator=g).bfloat16(), (torch.randn(n, outs, d_in, generator=g) / math.sqrt(d_in)).bfloat16()
        xs = ws = None
    off = _offsets(counts)
    want, slack = grouped_ref(x, w, off, rows, xs, ws, gated)
    to = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((m + spare, d_out), -7.0, dtype=dtype, device=DEV)
        y = qamw.grouped_matmul(x.to(DEV), w.to(DEV), off.to(DEV), rows=to(rows), x_scales=to(xs), w_scales=to(ws), gated=gated, out=out)
        assert y is out and (out[m:] == -7).all()
        check(out[:m], want, slack, dtype)
        if i8 and not gated:
            assert torch.equal(out[:m].cpu(), want.float().to(dtype))


@gpu
@pytest.mark.parametrize("m_each,d_out,d_in", [(2, 70, 96), (50, 70, 96), (300, 270, 256), (300, 270, 250)])
@pytest.mark.parametrize("pad,skip", [(0, 0), (16, 16), (8, 0), (1, 1)])
@pytest.mark.parametrize("i8", [False, True])
def test_grouped_strides_and_strangers(m_each, d_out, d_in, pad, skip, i8):
    """Padded and unaligned operands with NaNs between the rows, an expert's stride that is more than its matrix, NaNs in rows that
    are not asked for and in experts that have none: nothing of it shows."""
    say(f"[grouped] strides {m_each} {d_out} {d_in} pad {pad} skip {skip} int8 {i8}")
    g = _gen(m_each + pad)
    counts = [m_each, 0, m_each + 1]
    m = sum(counts)
    if i8:
        x, w = _codes(g, m + 4, d_in), _codes(g, 3, d_out, d_in)
        xs, ws = torch.rand(m + 4, generator=g) / 127, torch.rand(3, d_out, generator=g)
        xs[m:], ws[1] = math.nan, math.nan
    else:
        x, w = torch.randn(m + 4, d_in, generator=g).bfloat16(), torch.randn(3, d_out, d_in, generator=g).bfloat16()
        x[m:], w[1] = math.nan, math.nan
        xs = ws = None
    rows = torch.randperm(m, generator=g).to(torch.int32)
    off = _offsets(counts)
    want, slack = grouped_ref(x, w, off, rows, xs, ws, False)
    dw = _strided(torch.cat([w, torch.zeros(3, 2, d_in, dtype=w.dtype)], 1), pad, skip)[:, :d_out]
    out = _strided(torch.zeros(m, d_out), pad, skip)
    to = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    qamw.grouped_matmul(_strided(x, pad, skip), dw, off.to(DEV), rows=rows.to(DEV), x_scales=to(xs), w_scales=to(ws), out=out)
    check(out, want, slack, "strided")


@gpu
@pytest.mark.parametrize("m,d_out,d_in", [(20, 40, 256), (400, 300, 256)])
def test_grouped_infinities_stay_in_their_rows(m, d_out, d_in):
    g = _gen(m)
    x, w = torch.randn(m, d_in, generator=g).bfloat16(), torch.randn(2, d_out, d_in, generator=g).bfloat16()
    x[3, 5], x[7, 0], x[m - 1, d_in - 1] = math.inf, math.nan, -math.inf
    off = _offsets([m // 2, m - m // 2])
    y = qamw.grouped_matmul(x.to(DEV), w.to(DEV), off.to(DEV), out_dtype=torch.float32).cpu()
    odd = torch.zeros(m, dtype=torch.bool)
    odd[[3, 7, m - 1]] = True
    assert not torch.isfinite(y[odd]).any() and torch.isfinite(y[~odd]).all()
    assert torch.equal(y[3] > 0, w[0, :, 5].float() > 0) and torch.isnan(y[7]).all()
    # the largest gates and smallest: silu is the identity there, and 0
    big = torch.zeros(4, 16, dtype=torch.bfloat16)
    big[:, 0] = torch.tensor([1e30, -1e30, 200.0, -200.0]).bfloat16()
    wg = torch.zeros(1, 2, 16, dtype=torch.bfloat16)
    wg[0, 0, 0], wg[0, 1, 0] = 1.0, 1.0
    z = qamw.grouped_matmul(big.to(DEV), wg.to(DEV), _offsets([4]).to(DEV), gated=True, out_dtype=torch.float32).cpu()[:, 0]
    b = big[:, 0].float()
    assert z[0] == math.inf and z[1] == 0 and z[2] == b[2] * b[2] and abs(z[3]) < 1e-30


@gpu
def test_grouped_indices_out_of_range_stay_inside():
    """Offsets that are not ascending or beyond m, rows beyond X: unspecified results in those rows, right ones in the others."""
    g = _gen(5)
    x, w = torch.randn(64, 128, generator=g).bfloat16(), torch.randn(4, 96, 128, generator=g).bfloat16()
    rows = torch.arange(64, dtype=torch.int32)
    rows[10], rows[11] = 1 << 30, -5
    y = qamw.grouped_matmul(x.to(DEV), w.to(DEV), _offsets([16, 16, 16, 16]).to(DEV), rows=rows.to(DEV), out_dtype=torch.float32).cpu()
    want = torch.cat([x[i * 16:(i + 1) * 16].double() @ w[i].double().t() for i in range(4)])
    keep = torch.ones(64, dtype=torch.bool)
    keep[[10, 11]] = False
    assert ((y - want).abs()[keep] <= 128 * 2.0**-23 * (x.double().abs() @ w[0].double().abs().t()).max()).all()
    # the last expert's places, held within 0 .. m, are those of others too: whoever writes them, nobody writes beside them
    guarded = torch.full((64 + 64 + 64, 96), 5.0, device=DEV)
    qamw.grouped_matmul(x.to(DEV), w.to(DEV), torch.tensor([0, 16, 1 << 30, -3, 20], dtype=torch.int32, device=DEV), out=guarded[64:128])
    assert (guarded[:64] == 5).all() and (guarded[128:] == 5).all()


@gpu
def test_products_past_32_bit_offsets():
    """Rows of X, of W and of Y that begin beyond 2^32 bytes, with and without gathering."""
    d, ld = 256, 1 << 24
    m = 300
    flat = torch.empty(m * ld, dtype=torch.int8, device=DEV)
    x = torch.as_strided(flat, (m, d), (ld, 1))
    g = _gen(9)
    xc, wc = _codes(g, m, d), _codes(g, m, d)
    x.copy_(xc)
    one = torch.ones(m, device=DEV)
    want = int8_ref(xc, torch.ones(m), wc, torch.ones(m))
    dw = wc.to(DEV)
    assert torch.equal(qamw.int8_matmul(x, dw, one, x_scales=one, out_dtype=torch.float32).cpu(), want)
    assert torch.equal(qamw.int8_matmul(x[-20:], dw, one, x_scales=one[:20], out_dtype=torch.float32).cpu(), want[-20:])
    off = _offsets([5, 290, 5]).to(DEV)
    rows = torch.arange(m - 1, -1, -1, dtype=torch.int32)
    w3 = dw[None].expand(3, -1, -1)                              # one matrix for every expert: a stride of 0
    y = qamw.grouped_matmul(x, w3, off, rows=rows.to(DEV), x_scales=one, w_scales=torch.ones(3, m, device=DEV), out_dtype=torch.float32)
    assert torch.equal(y.cpu(), want.flip(0))
    few = qamw.grouped_matmul(x, w3, _offsets([2, 1, 3]).to(DEV), rows=rows[:6].to(DEV), x_scales=one, w_scales=torch.ones(3, m, device=DEV), out_dtype=torch.float32)
    assert torch.equal(few.cpu(), want.flip(0)[:6])
    x.copy_(wc)                                                  # now W is the far one
    near = xc.to(DEV)
    for k in (1, 20, m):
        assert torch.equal(qamw.int8_matmul(near[:k], x, one, x_scales=one[:k], out_dtype=torch.float32).cpu(), want[:k])
    yout = torch.as_strided(flat.view(torch.float32), (m, m), (ld // 4, 1))
    qamw.int8_matmul(near, dw, one, x_scales=one, out=yout)
    assert torch.equal(yout.cpu(), want)
    yout.zero_()
    qamw.int8_matmul(near[:20], dw, one, x_scales=one[:20], out=yout[-20:])
    assert torch.equal(yout[-20:].cpu(), want[:20])


# ------------------------------------------------------------------------------------------------------ routing, combination


def route_ref(x, k, renormalise):
    m, n = x.shape
    rows = x.double().tolist()
    experts, weights = np.full((m, k), -1, np.int32), np.zeros((m, k))
    for t in range(m):
        row = rows[t]
        ok = [e for e in range(n) if row[e] > -math.inf]
        best = sorted(ok, key=lambda e: (-row[e], e))[:k]
        if best:
            top = row[best[0]]
            p = lambda e: 1.0 if row[e] == top else math.exp(row[e] - top)  # noqa: E731
            total = math.fsum(p(e) for e in (best if renormalise else ok))
            experts[t, :len(best)] = best
            weights[t, :len(best)] = [p(e) / total for e in best]
    flat = experts.reshape(-1)
    counts = np.bincount(flat[flat >= 0], minlength=n)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    order = [s for e in range(n) for s in np.nonzero(flat == e)[0]]
    out_rows, positions = np.full(m * k, -1, np.int32), np.full(m * k, -1, np.int32)
    for p_, s in enumerate(order):
        out_rows[p_], positions[s] = s // k, p_
    return experts, weights, offsets, out_rows, positions.reshape(m, k)


@gpu
@pytest.mark.parametrize("m,n,k", [(0, 4, 2), (1, 1, 1), (1, 8, 2), (5, 8, 2), (3, 64, 6), (17, 5, 5), (63, 65, 3), (64, 128, 8), (65, 60, 8), (130, 256, 8), (200, 32, 32),
                                   (33, 1024, 17), (500, 130, 1), (1500, 16, 4), (2100, 257, 2), (4000, 3, 2), (40, 1000, 32)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route(m, n, k, dtype, renormalise):
    say(f"[route] {m} tokens, {k} of {n} experts, {dtype} renormalise {renormalise}")
    g = _gen(m + n * 3 + k)
    x = (torch.randn(m, n, generator=g) * 2).to(dtype)
    if m > 2:
        x = (x * 4).round() / 4                                # many ties
        x[torch.rand(m, n, generator=g) < 0.1] = -math.inf
        x[1] = -math.inf                                        # a token that goes nowhere
        x[2, 0] = math.nan
        x[m - 1] = math.nan
    if m > 20:
        x[3] = torch.finfo(dtype).min                           # a mask by the type's lowest value is a number like others
        x[4, 1:] = torch.finfo(dtype).min
        x[5] = -math.inf
        x[5, n - 1] = -3.0                                      # a token with one choice
        x[6, n // 2] = math.inf
        x[7, 0], x[7, n - 1] = math.inf, math.inf
        x[8] = 0.0
        x[8, ::2] = -0.0                                        # equal to 0: the lowest expert first
        x[9] = torch.finfo(dtype).max
        x[10:40] = x[10]                                        # many tokens of the same experts
    dx = _strided(x, 3, 1) if m % 2 else x.to(DEV)
    got = qamw.route(dx, k, renormalise=renormalise)
    experts, weights, offsets, rows, positions = route_ref(x, k, renormalise)
    assert np.array_equal(got.experts.cpu().numpy(), experts)
    assert np.array_equal(got.offsets.cpu().numpy(), offsets)
    assert np.array_equal(got.positions.cpu().numpy(), positions)
    assert np.array_equal(got.rows.cpu().numpy(), rows)
    # an exponential of an argument rounded to 2^-24 of at most 104 (below, it is 0), a sum of up to n terms, a division
    w = got.weights.cpu().double().numpy()
    assert (np.abs(w - weights) <= weights * (n + 120) * 2.0**-23 + 1e-37).all()
    again = qamw.route(dx, k, renormalise=renormalise)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@gpu
@pytest.mark.parametrize("m,n,k", [(1100003, 4, 2), (70001, 9, 9), (5000, 1021, 3)])
def test_route_of_many_tokens(m, n, k):
    """More workgroups than one sum of 16 bits holds the counts of, experts that all tokens like, rows of counts with an odd end."""
    say(f"[route] many {m} x {n}, {k}")
    x = torch.randn(m, n, generator=_gen(m)).bfloat16()
    x[:, 1] += 6.0
    x[100:3000] = -torch.inf
    r = qamw.route(x.to(DEV), k)
    flat = r.experts.reshape(-1).long()
    assert torch.equal(r.experts[:, 0].cpu()[3000:].long(), x[3000:].float().max(1).indices)
    assert (flat[100 * k:3000 * k] == -1).all() and (flat[:100 * k] >= 0).all() and (flat[3000 * k:] >= 0).all()
    order = torch.sort(torch.where(flat < 0, n, flat), stable=True).indices[:int((flat >= 0).sum())]
    counts = torch.bincount(flat[flat >= 0], minlength=n)
    assert torch.equal(r.offsets.long(), torch.cat([counts.new_zeros(1), counts.cumsum(0)]))
    assert torch.equal(r.rows[:len(order)].long(), order // k) and (r.rows[len(order):] == -1).all()
    positions = torch.full_like(flat, -1)
    positions[order] = torch.arange(len(order), device=DEV)
    assert torch.equal(r.positions.reshape(-1).long(), positions)


@gpu
@pytest.mark.parametrize("m,k,d,pad,skip", [(0, 2, 8, 0, 0), (1, 1, 1, 0, 0), (5, 2, 4096, 0, 0), (7, 3, 100, 0, 0), (64, 8, 839, 0, 0), (33, 6, 2048, 8, 8), (20, 32, 70, 1, 1), (300, 2, 5120, 0, 0), (9, 5, 13825, 0, 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_combine(m, k, d, pad, skip, dtype, out_dtype):
    say(f"[combine] {m} tokens, {k} of width {d}, {dtype} to {out_dtype}")
    g = _gen(m + k + d)
    n = m * k + 3
    y = torch.randn(n, d, generator=g).to(dtype)
    positions = torch.randperm(n, generator=g)[:m * k].to(torch.int32).view(m, k)
    weights = torch.rand(m, k, generator=g)
    if m > 4:
        y[positions[0, 0]] = math.nan                           # a stranger's row ...
        positions[0, 0], weights[0, 0] = -1, math.nan           # ... that is not asked for, nor is its weight
        positions[1] = -1                                       # a token that went nowhere
        positions[2, k - 1] = n + 7                             # past the end: adds nothing
        positions[3, k - 1] = positions[4, 0]                   # a row twice
    out = _strided(torch.zeros(m, d, dtype=out_dtype), pad, skip) if m else torch.zeros(m, d, dtype=out_dtype, device=DEV)
    qamw.combine(_strided(y, pad, skip), positions.to(DEV), weights.to(DEV), out=out)
    want, size = torch.zeros(m, d, dtype=torch.float64), torch.zeros(m, d, dtype=torch.float64)
    for t in range(m):
        for j in range(k):
            p = int(positions[t, j])
            if 0 <= p < n:
                want[t] += weights[t, j].double() * y[p].double()
                size[t] += (weights[t, j].double() * y[p].double()).abs()
    check(out, want, size * k * 2.0**-24, "combine")
    if pad and m:
        assert torch.isnan(torch.as_strided(out, (m, d + pad), out.stride(), out.storage_offset())[:, d:]).all()


@gpu
def test_combine_past_32_bit_offsets():
    ld, n, d = 1 << 23, 300, 200
    flat = torch.empty(n * ld, dtype=torch.bfloat16, device=DEV)
    y = torch.as_strided(flat, (n, d), (ld, 1))
    v = torch.randn(n, d, generator=_gen(1)).bfloat16()
    y.copy_(v)
    p = torch.arange(n - 1, -1, -1, dtype=torch.int32).view(-1, 2)
    got = qamw.combine(y, p.to(DEV), torch.ones(n // 2, 2, device=DEV), out_dtype=torch.float32).cpu()
    assert torch.equal(got, v[p[:, 0].long()].float() + v[p[:, 1].long()].float())


# ---------------------------------------------------------------------------------------------------------------- together


@gpu
def test_calls_on_another_stream_and_in_a_graph():
    """Results, workspaces and results' memory belong to the stream that the call names; a captured layer replays to the same."""
    say("[streams] a routed 8-bit layer on a side stream, then captured")
    g = _gen(3)
    m, n, k, d, h = 48, 8, 2, 256, 320
    x = torch.randn(m, d, generator=g).bfloat16().to(DEV)
    gate = torch.randn(m, n, generator=g).to(DEV)
    up = qamw.int8_quantize(torch.randn(n * 2 * h, d, generator=g).to(DEV))
    down = qamw.int8_quantize(torch.randn(n * d, h, generator=g).to(DEV))
    back = qamw.int8_quantize(torch.randn(d, d, generator=g).to(DEV))

    def layer(stream=None):
        r = qamw.route(gate, k, stream=stream)
        c, s = qamw.int8_quantize(x, stream=stream)
        y = qamw.grouped_matmul(c, up[0].view(n, 2 * h, d), r.offsets, rows=r.rows, x_scales=s, w_scales=up[1].view(n, 2 * h), gated=True, stream=stream)
        c, s = qamw.int8_quantize(y, stream=stream)
        z = qamw.grouped_matmul(c, down[0].view(n, d, h), r.offsets, x_scales=s, w_scales=down[1].view(n, d), stream=stream)
        z = qamw.int8_matmul(z, *back, stream=stream)
        return qamw.combine(z, r.positions, r.weights, stream=stream)

    want = layer()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = layer(side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer()
    for i in range(4):
        x.copy_(torch.randn(m, d, generator=g).bfloat16())
        gate.copy_(torch.randn(m, n, generator=g))
        eager = layer()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, eager), f"replay {i}"
