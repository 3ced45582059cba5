"""Rows in 4-bit floating point: refusals (on the CPU), codes and scales element by element against the definition, products against
exact sums, and a routed layer of them.  Where a test asks for equal numbers, every partial sum is a whole number of units below
2^24 of them, so that fp32 holds it exactly in any order."""
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
VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# ------------------------------------------------------------------------------------------------------------ refusals


def test_refusals_of_the_entry_points():
    """The pointers are never followed: every refusal comes before a launch."""
    L, I, S, U = qamw.lib(), qamw.ERR_INVALID_ARG, qamw.ERR_SHAPE, qamw.ERR_UNSUPPORTED
    p, need, more = 1 << 20, C.c_size_t(), C.c_size_t()
    assert L.qamw_mx4_row_bytes(33, C.byref(need), C.byref(more)) == qamw.OK and (need.value, more.value) == (32, 16)
    assert L.qamw_mx4_row_bytes(0, C.byref(need), C.byref(more)) == I and L.qamw_mx4_row_bytes(131073, C.byref(need), C.byref(more)) == I
    assert L.qamw_mx4_row_bytes(8, None, C.byref(more)) == I and L.qamw_mx4_row_bytes(8, C.byref(need), None) == I

    def quant(X=p, dtype=0, m=4, d=8, ldx=8, cs=None, codes=p, scales=p):
        return L.qamw_mx4_quantize(X, dtype, m, d, ldx, cs, codes, scales, None)

    assert quant(X=None) == I and quant(codes=None) == I and quant(scales=None) == I and quant(dtype=2) == I and quant(dtype=-1) == I
    assert quant(m=-1) == I and quant(m=(1 << 22) + 1) == I and quant(d=0) == I and quant(d=131073, ldx=131073) == I
    assert quant(X=p + 2) == I and quant(codes=p + 8) == I and quant(scales=p + 4) == I and quant(cs=p + 2) == I and quant(ldx=7) == S
    assert quant(m=1 << 22, d=131072, ldx=131072) == U and quant(m=0, X=None, codes=None, scales=None) == qamw.OK

    def back(codes=p, scales=p, m=4, d=8, out=p, t=1, ldo=8):
        return L.qamw_mx4_dequantize(codes, scales, m, d, out, t, ldo, None)

    assert back(codes=None) == I and back(scales=None) == I and back(out=None) == I and back(t=2) == I and back(d=0) == I and back(m=-1) == I
    assert back(codes=p + 8) == I and back(scales=p + 8) == I and back(out=p + 1) == I and back(ldo=7) == S
    assert back(m=0, codes=None, scales=None, out=None) == qamw.OK

    size = lambda t, xr, m, e, n, k, g=0: L.qamw_mx4_matmul_workspace_bytes(t, xr, m, e, n, k, g, C.byref(need))  # noqa: E731
    assert size(0, 3, 3, 0, 8, 33) == qamw.OK and need.value >= 3 * 48 and size(3, 3, 3, 0, 8, 33) == qamw.OK
    assert size(2, 3, 3, 0, 8, 33) == I and size(0, -1, 3, 0, 8, 33) == I and size(0, 3, -1, 0, 8, 33) == I and size(0, 3, 3, 1025, 8, 33) == I
    assert size(0, 3, 3, 0, 0, 33) == I and size(0, 3, 3, 0, 8, 0) == I and size(0, 3, 3, 0, 8, 131073) == I and size(0, 3, 3, 0, 8, 33, 2) == I
    assert L.qamw_mx4_matmul_workspace_bytes(0, 3, 3, 0, 8, 33, 0, None) == I

    def mm(X=p, xt=3, xs=p, cs=None, m=4, ldx=8, W=p, ws=p, d_out=8, d_in=8, gated=0, Y=p, yt=1, ldy=8, work=p, n=1 << 30):
        return L.qamw_mx4_matmul(X, xt, xs, cs, m, ldx, W, ws, d_out, d_in, gated, Y, yt, ldy, work, n, None)

    assert mm(X=None) == I and mm(W=None) == I and mm(ws=None) == I and mm(Y=None) == I and mm(xs=None) == I and mm(xt=2) == I and mm(yt=2) == I
    assert mm(gated=2) == I and mm(d_out=0) == I and mm(d_in=0) == I and mm(m=-1) == I and mm(cs=p) == I and mm(xt=1) == I
    assert mm(X=p + 8) == I and mm(xs=p + 8) == I and mm(W=p + 8) == I and mm(ws=p + 8) == I and mm(Y=p + 1) == I
    five = dict(xt=1, xs=None, m=5)                                        # up to four rows of 4096 are quantised in the product's own launch
    assert mm(**five, work=None, n=0) == I and mm(**five, n=64) == I and mm(**five, work=p + 8) == I
    assert mm(xt=1, xs=None, ldx=7) == S and mm(ldy=7) == S
    assert mm(m=1 << 22, d_out=1 << 24, ldy=1 << 24) == U                  # more tiles than a launch has
    assert mm(d_out=1 << 16, d_in=131072, ldy=1 << 16) == U                # more than 2 GiB of codes
    assert mm(**five, d_out=1 << 16, d_in=131072, ldx=131072, ldy=1 << 16) == U
    assert mm(m=0, X=None, xs=None, W=None, ws=None, Y=None, work=None, n=0) == qamw.OK

    def grouped(X=p, t=3, xs=p, cs=None, xr=4, ldx=8, rows=None, W=p, ws=p, off=p, n=2, m=4, d_out=8, d_in=8, gated=0, Y=p, yt=1, ldy=8, work=p, size=1 << 30):
        return L.qamw_mx4_grouped_matmul(X, t, xs, cs, xr, ldx, rows, W, ws, off, n, m, d_out, d_in, gated, Y, yt, ldy, work, size, None)

    assert grouped(n=0) == I and grouped(n=-1) == I and grouped(n=1025) == I and grouped(off=None) == I and grouped(off=p + 2) == I and grouped(rows=p + 1) == I
    assert grouped(xr=3) == S and grouped(rows=p, xr=0) == S and grouped(ldy=7) == S and grouped(t=0) == I and grouped(t=0, xs=None, size=0) == I
    assert grouped(rows=p, xr=1 << 20, d_in=131072) == U                   # gathered from more than 2 GiB
    assert grouped(m=0, X=None, xs=None, W=None, ws=None, off=None, Y=None, work=None, size=0) == qamw.OK


def test_refusals_of_the_binding(monkeypatch):
    monkeypatch.setattr(qamw, "_one_device", lambda *t: 0)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    w = qamw.Mx4(u8(6, 16), u8(6, 16), 8)
    x = torch.zeros(4, 8)
    for bad in (qamw.Mx4(u8(6, 32), u8(6, 16), 8), qamw.Mx4(u8(6, 16), u8(5, 16), 8), qamw.Mx4(u8(6, 16), u8(6, 16), 33),
                qamw.Mx4(u8(6, 32)[:, :16], u8(6, 16), 8), qamw.Mx4(u8(6, 16).to(torch.int8), u8(6, 16), 8), qamw.Mx4(u8(2, 6, 16), u8(2, 6, 16), 8)):
        with pytest.raises(ValueError):
            qamw.mx4_matmul(x, bad)
        with pytest.raises(ValueError):
            qamw.mx4_dequantize(bad)
    with pytest.raises(qamw.QamwError):
        qamw.mx4_matmul(x, qamw.Mx4(u8(6, 16), u8(6, 16), 0))
    with pytest.raises(ValueError):
        qamw.mx4_matmul(x[:, :7], w)
    with pytest.raises(ValueError):
        qamw.mx4_matmul(x.t(), w)
    with pytest.raises(ValueError):
        qamw.mx4_matmul(x, w, col_scale=torch.ones(7))
    with pytest.raises(TypeError):
        qamw.mx4_matmul(x.half(), w)
    with pytest.raises(ValueError):
        qamw.mx4_matmul(x, qamw.Mx4(u8(5, 16), u8(5, 16), 8), gated=True)
    with pytest.raises(ValueError):
        qamw.mx4_matmul(x, w, out=torch.zeros(4, 5))
    e = qamw.Mx4(u8(2, 6, 16), u8(2, 6, 16), 8)
    off = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        qamw.mx4_grouped_matmul(x, w, off)
    with pytest.raises(ValueError):
        qamw.mx4_grouped_matmul(x, e, off[:2])
    with pytest.raises(ValueError):
        qamw.mx4_grouped_matmul(x, e, off.long())
    with pytest.raises(ValueError):
        qamw.mx4_grouped_matmul(x, e, off, rows=torch.zeros(4))
    with pytest.raises(ValueError):
        qamw.mx4_quantize(x, col_scale=torch.ones(9))
    with pytest.raises(ValueError):
        qamw.mx4_quantize(x, out=qamw.Mx4(u8(5, 16), u8(5, 16), 8))
    with pytest.raises(TypeError):
        qamw.mx4_dequantize(w, out_dtype=torch.float16)


# ---------------------------------------------------------------------------------------------------------- quantisation


def quantise_ref(x, col_scale=None):
    """(codes, scale bytes by block, in their order) by the definition: fp32 product, then exact steps in 64 bits; borders between values go to the
    even code."""
    v = x.float().numpy()
    if col_scale is not None:
        v = v * col_scale.float().numpy()
    m, d = v.shape
    nb = -(-d // 32)
    b = np.zeros((m, nb * 32))
    b[:, :d] = v
    b = b.reshape(m, nb, 32)
    with np.errstate(all="ignore"):
        a = np.abs(b).max(axis=2)
        fine = np.isfinite(a)
        e = np.where(fine & (a > 0), np.maximum(np.frexp(np.where(fine, a, 1))[1] - 3, -127), -127)
        t = np.abs(b) * np.exp2(-e.astype(np.float64))[:, :, None]
        c = np.zeros(t.shape, np.uint8)
        for k, border in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
            c += (t >= border) if k % 2 else (t > border)
        c += 8 * np.signbit(b).astype(np.uint8)
    c = np.where(fine[:, :, None], c, 0).reshape(m, nb * 32)
    return c, np.where(fine, e + 127, 255).astype(np.uint8)


def pack(codes, scales, d):
    """Codes [m][32 blocks] and scale bytes [m][blocks] in the library's layout, by its definition."""
    m, nb = scales.shape
    packed = codes[:, 0::2] | codes[:, 1::2] << 4
    s = np.zeros((m, -(-d // 512) * 16), np.uint8)
    for b in range(nb):
        s[:, 16 * (b // 16) + 4 * (b % 4) + (b % 16) // 4] = scales[:, b]
    assert packed.shape[1] == 16 * -(-d // 32)
    return packed, s


def values(codes, scales, d):
    """What codes stand for, in 64 bits."""
    with np.errstate(invalid="ignore"):
        power = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
        return (VALUES[codes].reshape(codes.shape[0], -1, 32) * power[:, :, None]).reshape(codes.shape[0], -1)[:, :d]


def to_device(codes, scales, d):
    p, s = pack(codes, scales, d)
    return qamw.Mx4(torch.from_numpy(p).to(DEV), torch.from_numpy(s).to(DEV), d)


def _strided(t, pad, skip):
    """The same matrix on the device, with rows `pad` elements longer and a start `skip` elements into its memory."""
    m, d = t.shape
    flat = torch.full((skip + m * (d + pad) + 8,), 77, dtype=t.dtype, device=DEV)
    v = torch.as_strided(flat, t.shape, (d + pad, 1), skip)
    v.copy_(t)
    return v


@gpu
@pytest.mark.parametrize("m,d,dtype,pad,skip,smooth", [
    (1, 1, torch.float32, 0, 0, False), (3, 5, torch.bfloat16, 0, 0, True), (1, 4096, torch.bfloat16, 0, 0, False), (7, 257, torch.float32, 0, 0, True),
    (5, 512, torch.bfloat16, 8, 0, True), (5, 513, torch.bfloat16, 3, 1, False), (300, 1024, torch.float32, 4, 4, True), (9, 31, torch.bfloat16, 0, 0, True),
    (9, 32, torch.float32, 1, 0, False), (9, 33, torch.bfloat16, 0, 1, False), (4, 5632, torch.float32, 0, 0, False), (3, 13824, torch.bfloat16, 16, 8, False),
    (2, 4095, torch.float32, 1, 1, True), (1, 131072, torch.float32, 0, 0, False), (2, 131071, torch.bfloat16, 0, 0, True), (70000, 16, torch.bfloat16, 0, 0, False),
    (33, 11008, torch.bfloat16, 0, 0, True), (16400, 5, torch.bfloat16, 2, 1, True), (17001, 33, torch.float32, 0, 0, False), (5601, 1029, torch.bfloat16, 3, 1, True),
])
def test_quantise(m, d, dtype, pad, skip, smooth):
    say(f"[mx4] quantise {m}x{d} {dtype} pad {pad} skip {skip} smooth {smooth}")
    g = _gen(m * 7 + d)
    x = (torch.randn(m, d, generator=g) * torch.exp(2 * torch.randn(m, 1, generator=g))).to(dtype)
    c = torch.exp(0.5 * torch.randn(d, generator=g)) if smooth else None
    cb, sb = qamw.mx4_row_bytes(d)
    whole = torch.full((m * cb + 64,), 77, dtype=torch.uint8, device=DEV), torch.full((m * sb + 64,), 77, dtype=torch.uint8, device=DEV)
    out = qamw.Mx4(whole[0][:m * cb].view(m, cb), whole[1][:m * sb].view(m, sb), d)
    q = qamw.mx4_quantize(_strided(x, pad, skip), None if c is None else c.to(DEV), out=out)
    codes, scales = quantise_ref(x, c)
    want_c, want_s = pack(codes, scales, d)
    assert np.array_equal(q.scales.cpu().numpy(), want_s)
    assert np.array_equal(q.codes.cpu().numpy(), want_c)
    assert (whole[0][m * cb:] == 77).all() and (whole[1][m * sb:] == 77).all()
    # and back, to rows of any stride
    for t in (torch.float32, torch.bfloat16):
        to = _strided(torch.zeros(m, d, dtype=t), pad, skip)
        assert qamw.mx4_dequantize(q, out=to) is to
        assert torch.equal(to.cpu(), torch.from_numpy(values(codes, scales, d)).to(t))
        if pad:
            assert (torch.as_strided(to, (m, d + pad), to.stride(), to.storage_offset())[:, d:] == 77).all()
    assert torch.equal(qamw.mx4_dequantize(q).cpu(), to.cpu())


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantise_special_blocks(dtype):
    say(f"[mx4] special blocks {dtype}")
    g = _gen(3)
    x = torch.randn(14, 32, generator=g)
    x[0] = 0
    x[1] = -0.0
    x[2, 5] = math.inf
    x[3, 31] = -math.inf
    x[4, 0] = math.nan
    x[5] = 3.0e38 * torch.sign(x[5])
    x[6] *= 2.0**-126                                      # the scale is the smallest: e = -127
    x[7] *= 2.0**-130                                      # subnormal values: codes of what is left at e = -127
    x[8] = 1e-45
    x[9] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4) * torch.tensor([1.0, -1.0] * 16)   # the borders
    x[10] = torch.tensor([7.9, 7.0, 6.99, 4.0] * 8)        # beyond 6
    x[11] = 0
    x[11, 3] = 4.0
    x[12] = torch.nextafter(torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4), torch.tensor([0.0, 9.0] * 16))
    x[13, 1:] = 2.0**-100
    x = x.to(dtype)
    q = qamw.mx4_quantize(x.to(DEV))
    codes, scales = quantise_ref(x)
    want_c, want_s = pack(codes, scales, 32)
    assert np.array_equal(q.scales.cpu().numpy(), want_s) and np.array_equal(q.codes.cpu().numpy(), want_c)
    assert (want_s[2:5, 0] == 255).all() and want_s[0, 0] == 0
    y = qamw.mx4_dequantize(q, out_dtype=torch.float32).cpu().numpy().astype(np.float64)
    assert np.array_equal(y, values(codes, scales, 32), equal_nan=True)


def test_layout_is_what_the_definition_says():
    """A row of one block in each place: on the CPU, the packer of these tests against the formula's inverse."""
    for b in range(48):
        scales = np.zeros((1, 48), np.uint8)
        scales[0, b] = 200
        _, s = pack(np.zeros((1, 48 * 32), np.uint8), scales, 48 * 32)
        at = int(np.flatnonzero(s[0])[0])
        assert at // 16 * 16 + at % 4 * 4 + at % 16 // 4 == b


# -------------------------------------------------------------------------------------------------------------- products


def _rows(g, m, d, spread):
    """Random codes of all values with scales of `spread` neighbouring powers of two: (codes, scales by block), zero past column d."""
    nb = -(-d // 32)
    codes = torch.randint(0, 16, (m, nb * 32), generator=g).to(torch.uint8).numpy()
    codes[:, d:] = 0
    return codes, (120 + torch.randint(0, spread, (m, nb), generator=g)).to(torch.uint8).numpy()


def product_ref(xc, xs, wc, ws, d):
    """In 64 bits: exact, since all terms are whole numbers of 2^-16 and far below 2^53 of them."""
    return torch.from_numpy(values(xc, xs, d) @ values(wc, ws, d).T)


def gate_ref(g, u):
    """silu(g) * u in 64 bits, and how far it may be off: the exponential's argument is rounded, which its size multiplies, and a handful of
    roundings follow."""
    s = g * torch.sigmoid(g)
    return s * u, (s * u).abs() * (g.abs() + 16) * 2.0**-23 + 1e-37


def check(got, want, slack):
    if got.dtype == torch.bfloat16:
        slack = slack + (want.abs() + slack) * 2.0**-8
    off = (got.cpu().double() - want).abs()
    bad = ~(off <= slack)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}, worst {float((off - slack).max())}"


SHAPES = [
    (1, 1, 1), (1, 17, 32), (2, 64, 100), (1, 4096, 4096), (3, 130, 1040), (8, 257, 2048), (13, 2047, 5632), (15, 33, 511), (16, 100, 512), (17, 31, 513),
    (31, 500, 272), (40, 2048, 1008), (64, 65, 4112), (65, 128, 64), (100, 700, 336), (129, 300, 1024), (200, 63, 15), (257, 513, 2065), (300, 260, 176),
    (513, 1030, 656), (700, 384, 128), (1000, 1600, 512), (33, 5, 13824), (5, 1000, 767), (300, 520, 769), (260, 256, 1280),
    (1, 13837, 300), (8, 9001, 1100), (16, 8193, 2048), (20, 9001, 1100), (32, 5120, 3333), (45, 5130, 3333), (128, 2047, 5632),   # many outputs of few rows
]


@gpu
@pytest.mark.parametrize("m,d_out,d_in", SHAPES)
@pytest.mark.parametrize("gated", [False, True])
def test_matmul_of_codes(m, d_out, d_in, gated):
    """Scales of 4 and 2 neighbouring powers of two: a term is at most 4 * 36 * 2^4 = 2304 units of a quarter at the smallest scales, so that up to 7281
    columns no sum passes 2^24 units; at 13824 columns sums of random signs are some 2^17, a hundredth of that."""
    say(f"[mx4] product {m} x {d_out} x {d_in} gated {gated}")
    g = _gen(m * 3 + d_out * 5 + d_in)
    outs = d_out * (2 if gated else 1)
    (xc, xs), (wc, ws) = _rows(g, m, d_in, 2), _rows(g, outs, d_in, 4)
    x, w = to_device(xc, xs, d_in), to_device(wc, ws, d_in)
    y = qamw.mx4_matmul(x, w, gated=gated, out_dtype=torch.float32)
    b = qamw.mx4_matmul(x, w, gated=gated)
    assert y.shape == (m, d_out) and b.dtype == torch.bfloat16
    ref = product_ref(xc, xs, wc, ws, d_in)
    if not gated:
        assert torch.equal(y.cpu(), ref.float())
    else:
        want, slack = gate_ref(ref[:, :d_out], ref[:, d_out:])
        check(y, want, slack)
    assert torch.equal(b.cpu(), y.cpu().bfloat16())            # the same number, rounded


@gpu
@pytest.mark.parametrize("m,d_out,d_in", [(1, 5, 7), (300, 700, 100), (77, 260, 4100), (513, 513, 513), (256, 512, 1024), (600, 300, 769), (2000, 300, 256)])
@pytest.mark.parametrize("tile", [64, 128, 256])
@pytest.mark.parametrize("gated", [False, True])
def test_matmul_by_tiles(m, d_out, d_in, tile, gated):
    """The kernel for many rows by every size of tile, whatever the estimate would choose: the same exact sums."""
    say(f"[mx4] tiles of {tile}: {m} x {d_out} x {d_in} gated {gated}")
    g = _gen(m + d_out * 5 + d_in)
    (xc, xs), (wc, ws) = _rows(g, m, d_in, 2), _rows(g, d_out * (2 if gated else 1), d_in, 4)
    x, w = to_device(xc, xs, d_in), to_device(wc, ws, d_in)
    before = qamw.set_kernel_path(tile)
    try:
        y = qamw.mx4_matmul(x, w, gated=gated, out_dtype=torch.float32)
        b = qamw.mx4_matmul(x, w, gated=gated)
        e = qamw.Mx4(w.codes.view(1, *w.codes.shape), w.scales.view(1, *w.scales.shape), d_in)
        rows = torch.randint(0, m, (m,), generator=g).to(torch.int32)
        grouped = qamw.mx4_grouped_matmul(x, e, torch.tensor([0, m], dtype=torch.int32, device=DEV), rows=rows.to(DEV), gated=gated, out_dtype=torch.float32)
    finally:
        qamw.set_kernel_path(before)
    ref = product_ref(xc, xs, wc, ws, d_in)
    if gated:
        want, slack = gate_ref(ref[:, :d_out], ref[:, d_out:])
        check(y, want, slack)
    else:
        assert torch.equal(y.cpu(), ref.float())
    assert torch.equal(b, y.bfloat16()) and torch.equal(grouped, y[rows.long().to(DEV)])


@gpu
@pytest.mark.parametrize("m,d_out,d_in", [(1, 300, 4096), (12, 64, 5632), (100, 333, 2048), (600, 300, 4100)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("smooth", [False, True])
def test_matmul_of_floats(m, d_out, d_in, dtype, smooth):
    """Quantised in the call as by mx4_quantize; any two orders of a sum of d terms, each addition off by at most 2^-23 of it, are within
    2 d 2^-23 of the sum of the terms' sizes: the bound that holds for scales of all sizes."""
    say(f"[mx4] floats {m} x {d_out} x {d_in} {dtype} smooth {smooth}")
    g = _gen(m + d_out + d_in)
    x = (torch.randn(m, d_in, generator=g) * torch.exp(torch.randn(m, 1, generator=g))).to(dtype)
    w = torch.randn(d_out, d_in, generator=g) / math.sqrt(d_in)
    c = torch.exp(0.5 * torch.randn(d_in, generator=g)) if smooth else None
    dw = qamw.mx4_quantize(w.to(DEV))
    dx = _strided(x, 5, 3)
    y = qamw.mx4_matmul(dx, dw, col_scale=None if c is None else c.to(DEV), out_dtype=torch.float32)
    q = qamw.mx4_quantize(dx, None if c is None else c.to(DEV))
    assert torch.equal(y, qamw.mx4_matmul(q, dw, out_dtype=torch.float32))
    xv, wv = torch.from_numpy(values(*quantise_ref(x, c), d_in)), torch.from_numpy(values(*quantise_ref(w), d_in))
    check(y, xv @ wv.T, d_in * 2.0**-23 * (xv.abs() @ wv.abs().T))
    assert float((y.cpu().double() - xv @ wv.T).norm() / (xv @ wv.T).norm()) < 1e-6     # and far less in the mean


@gpu
def test_matmul_output_rows_and_what_lies_between():
    say("[mx4] strided outputs")
    g = _gen(5)
    for m, d_out, d_in, pad, skip in ((5, 100, 96, 3, 1), (300, 270, 512, 2, 3), (300, 272, 512, 0, 4), (70, 131, 256, 5, 0), (1000, 512, 640, 8, 8)):
        for t in (torch.float32, torch.bfloat16):
            for gated in (False, True):
                (xc, xs), (wc, ws) = _rows(g, m, d_in, 2), _rows(g, d_out * (2 if gated else 1), d_in, 4)
                out = _strided(torch.zeros(m, d_out, dtype=t), pad, skip)
                x, w = to_device(xc, xs, d_in), to_device(wc, ws, d_in)
                assert qamw.mx4_matmul(x, w, gated=gated, out=out) is out
                assert torch.equal(out, qamw.mx4_matmul(x, w, gated=gated, out_dtype=t))
                flat = torch.as_strided(out, (m, d_out + pad), out.stride(), skip)
                assert (flat[:, d_out:] == 77).all() and (torch.as_strided(out, (skip + 1,), (1,), 0)[:skip] == 77).all()


@gpu
@pytest.mark.parametrize("m", [1, 20, 300])
def test_rows_that_are_no_numbers(m):
    """A block with an infinity or a NaN makes its row's products NaN and no others'; as a row of W, its output's."""
    say(f"[mx4] not numbers, {m} rows")
    g = _gen(m)
    x, w = torch.randn(m, 1000, generator=g), torch.randn(70, 1000, generator=g)
    x[m // 2, 999], w[69, 3] = math.inf, math.nan
    y = qamw.mx4_matmul(x.to(DEV), qamw.mx4_quantize(w.to(DEV)), out_dtype=torch.float32).cpu()
    nan = torch.zeros(m, 70, dtype=torch.bool)
    nan[m // 2], nan[:, 69] = True, True
    assert torch.equal(torch.isnan(y), nan) and torch.isfinite(y[~nan]).all()


@gpu
def test_no_rows():
    w = qamw.mx4_quantize(torch.randn(8, 64, device=DEV))
    assert qamw.mx4_matmul(torch.randn(0, 64, device=DEV), w).shape == (0, 8)
    q = qamw.mx4_quantize(torch.randn(0, 64, device=DEV))
    assert q.codes.shape == (0, 32) and qamw.mx4_dequantize(q).shape == (0, 64)
    e = qamw.Mx4(w.codes.view(2, 4, -1), w.scales.view(2, 4, -1), 64)
    off = torch.zeros(3, dtype=torch.int32, device=DEV)
    assert qamw.mx4_grouped_matmul(torch.randn(5, 64, device=DEV), e, off, rows=torch.empty(0, dtype=torch.int32, device=DEV)).shape == (0, 4)
    out = torch.full((5, 4), 7.0, device=DEV)
    qamw.mx4_grouped_matmul(torch.randn(5, 64, device=DEV), e, off, out=out)      # experts without rows
    assert (out == 7.0).all()


def _offsets(sizes, m, g):
    off = np.concatenate([[0], np.cumsum(sizes)])
    assert off[-1] <= m
    return torch.from_numpy(off.astype(np.int32))


@gpu
@pytest.mark.parametrize("sizes,tokens,d_out,d_in", [
    ([1, 0, 3, 0], 5, 33, 96), ([0, 0, 0, 7], 7, 130, 512), ([2, 2, 2, 2, 2], 3, 5632, 2048), ([70, 0, 1, 64, 65], 100, 100, 333), ([300, 17, 0, 257, 1], 200, 270, 1024),
    ([16] * 40, 64, 48, 640), ([1] * 100, 30, 64, 100), ([1000, 24], 600, 300, 1500), ([5] * 16, 30, 5643, 300), ([20, 31, 32, 33, 0, 1], 40, 5650, 640),
])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("gather", [False, True])
def test_grouped_matmul(sizes, tokens, d_out, d_in, gated, gather):
    say(f"[mx4] grouped {len(sizes)} experts, {sum(sizes)} rows x {d_out} x {d_in} gated {gated} gather {gather}")
    g = _gen(sum(sizes) + d_out)
    n, outs, used = len(sizes), d_out * (2 if gated else 1), sum(sizes)
    m = used + 3                                              # three rows that no expert has
    x_rows = tokens if gather else m
    xc, xs = _rows(g, x_rows, d_in, 2)
    ws = [_rows(g, outs, d_in, 4) for _ in range(n)]
    parts = [pack(c, s, d_in) for c, s in ws]
    w = qamw.Mx4(torch.from_numpy(np.stack([p[0] for p in parts])).to(DEV), torch.from_numpy(np.stack([p[1] for p in parts])).to(DEV), d_in)
    off = _offsets(sizes, m, g)
    rows = torch.randint(0, x_rows, (m,), generator=g).to(torch.int32) if gather else None
    out = torch.full((m, d_out), 77.0, device=DEV)
    x = to_device(xc, xs, d_in)
    qamw.mx4_grouped_matmul(x, w, off.to(DEV), rows=None if rows is None else rows.to(DEV), gated=gated, out=out)
    b = qamw.mx4_grouped_matmul(x, w, off.to(DEV), rows=None if rows is None else rows.to(DEV), gated=gated)
    got = out.cpu()
    assert (got[used:] == 77).all()
    for e in range(n):
        lo, hi = int(off[e]), int(off[e + 1])
        if lo == hi:
            continue
        idx = rows[lo:hi].long().numpy() if gather else np.arange(lo, hi)
        ref = product_ref(xc[idx], xs[idx], *ws[e], d_in)
        if gated:
            want, slack = gate_ref(ref[:, :d_out], ref[:, d_out:])
            check(got[lo:hi], want, slack)
        else:
            assert torch.equal(got[lo:hi], ref.float())
    assert torch.equal(b[:used].cpu(), got[:used].bfloat16())


@gpu
def test_grouped_matmul_of_floats_and_bad_indices():
    """Tokens quantised in the call, smoothed or not; rows and offsets out of range touch nothing beyond the arrays."""
    say("[mx4] grouped, floats, bad indices")
    g = _gen(8)
    n, d_out, d_in, tokens = 4, 96, 700, 50
    w = qamw.mx4_quantize(torch.randn(n * d_out, d_in, generator=g).to(DEV))
    w = qamw.Mx4(w.codes.view(n, d_out, -1), w.scales.view(n, d_out, -1), d_in)
    off = torch.tensor([0, 30, 31, 31, 100], dtype=torch.int32, device=DEV)
    rows = torch.randint(0, tokens, (100,), generator=g).to(torch.int32).to(DEV)
    c = torch.rand(d_in, generator=g).to(DEV) + 0.5
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn(tokens, d_in, generator=g).to(dtype).to(DEV)
        y = qamw.mx4_grouped_matmul(x, w, off, rows=rows, col_scale=c, out_dtype=torch.float32)
        q = qamw.mx4_quantize(x, c)
        assert torch.equal(y, qamw.mx4_grouped_matmul(q, w, off, rows=rows, out_dtype=torch.float32))
        one = qamw.mx4_matmul(qamw.Mx4(q.codes[rows[:30].long()], q.scales[rows[:30].long()], d_in), qamw.Mx4(w.codes[0], w.scales[0], d_in), out_dtype=torch.float32)
        assert float((y[:30] - one).abs().max()) <= d_in * 2.0**-22 * float(one.abs().max() + 40)
    bad_rows = rows.clone()
    bad_rows[::3], bad_rows[1::3] = -5, 1 << 30
    for bad_off in ([0, 30, 31, 31, 1 << 30], [-7, 30, 20, 31, 100], [100, 50, 0, 100, 0]):
        out = torch.full((104, d_out), 77.0, device=DEV)
        qamw.mx4_grouped_matmul(q, w, torch.tensor(bad_off, dtype=torch.int32, device=DEV), rows=bad_rows, out=out[:100])
        assert (out[100:] == 77).all()
    torch.cuda.synchronize()


@gpu
def test_two_products_at_once_and_in_a_graph():
    """Two streams with workspaces of their own, and a captured call that is replayed with new inputs in place, eager calls between."""
    say("[mx4] streams, graph")
    g = _gen(9)
    w = qamw.mx4_quantize(torch.randn(512, 1024, generator=g).to(DEV))
    for m in (3, 400):
        xs = [torch.randn(m, 1024, generator=g).to(DEV) for _ in range(4)]
        want = [qamw.mx4_matmul(x, w) for x in xs]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = [qamw.mx4_matmul(x, w, stream=side if i % 2 else None) for i, x in enumerate(xs)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        held = xs[0].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = qamw.mx4_matmul(held, w)
        for x, e in zip(xs, want):
            held.copy_(x)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, e)
            assert torch.equal(qamw.mx4_matmul(xs[1], w), want[1])


@gpu
@pytest.mark.parametrize("m", [3, 300])
def test_experts_beyond_4_gib(m):
    """The last of many experts, whose matrix begins beyond 2^32 bytes of codes, and no rows for the others."""
    say(f"[mx4] {m} rows of the last of 104 experts")
    n, outs, d = 104, 22016, 4096
    cb, sb = qamw.mx4_row_bytes(d)
    W = qamw.Mx4(torch.zeros(n, outs, cb, dtype=torch.uint8, device=DEV), torch.zeros(n, outs, sb, dtype=torch.uint8, device=DEV), d)
    assert (n - 1) * outs * cb > 2**32
    last = qamw.Mx4(W.codes[-1], W.scales[-1], d)
    g = torch.Generator(device=DEV).manual_seed(3)
    qamw.mx4_quantize(torch.randn(outs, d, generator=g, device=DEV, dtype=torch.bfloat16), out=last)
    x = qamw.mx4_quantize(torch.randn(m, d, generator=g, device=DEV))
    offsets = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
    offsets[-1] = m
    for gated in (False, True):
        try:
            qamw.set_kernel_path(0 if m == 3 else 128)        # the same tiles, and so the same sums
            got, want = qamw.mx4_grouped_matmul(x, W, offsets, gated=gated), qamw.mx4_matmul(x, last, gated=gated)
        finally:
            qamw.set_kernel_path(0)
        assert torch.isfinite(want).all() and want.abs().max() > 10
        err = (got.double() - want.double()).abs().max() / want.double().abs().max()
        assert err <= 2.0**-8 if m == 3 else torch.equal(got, want)
