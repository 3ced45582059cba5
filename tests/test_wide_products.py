"""The products of many rows, whose workgroups go from tile to tile: bit for bit against sums in 64 bits in int8, within the bound of the
roundings in bf16.  Sums of whole numbers below 2^53 are exact in 64 bits, on the device as on the CPU."""
import numpy as np
import pytest
import torch

from paper_2605_26339_amd import qamw

from .test_served_layers import _strided, gate_ref, say

gpu = pytest.mark.gpu
DEV = "cuda"
TYPES = (torch.float32, torch.bfloat16)


def _gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def _codes(g, *shape):
    return torch.randint(-127, 128, shape, generator=g, device=DEV, dtype=torch.int32).to(torch.int8)


def _scales(g, *shape):
    """Of different sizes, so that another row's or another output's is not taken for its own; a gate stays below 80 in size with them."""
    return torch.exp(torch.randn(*shape, generator=g, device=DEV).clamp(-1.5, 1.5)) / 127


def _offsets(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)


def _sums(x, w):
    return torch.mm(x.double(), w.double().t().contiguous())


def _scaled(x, xs, w, ws):
    """The exact sums, then the two prescribed fp32 products."""
    return _sums(x, w).float() * xs[:, None] * ws[None, :]


def expect(got, ref, gated, slack, what):
    """got [m][d_out] against ref [m][outs], the sums with their scales: the same bits where nothing but prescribed steps lies between
    (slack None and no gate), otherwise within slack, what the gate makes of it, and half a unit of bf16 where the result is one."""
    if not gated and slack is None:
        assert torch.equal(got, ref.to(got.dtype)), f"{what}: {int((got != ref.to(got.dtype)).sum())} of {got.numel()}"
        return
    want, off = ref.double(), torch.zeros_like(ref, dtype=torch.float64) if slack is None else slack
    if gated:
        h = ref.shape[1] // 2
        want, off = gate_ref(want[:, :h], want[:, h:], off[:, :h], off[:, h:])
    if got.dtype == torch.bfloat16:
        off = off + (want.abs() + off) * 2.0**-8
    bad = ~((got.double() - want).abs() <= off)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, rows {bad.any(1).nonzero()[:4, 0].tolist()}, outputs {bad.any(0).nonzero()[:4, 0].tolist()}"


# ---- few columns: a tile is one or two stages, and its scales follow the last one's at once -------------------------------------------


@gpu
@pytest.mark.parametrize("d_in", [16, 128, 144, 256, 272])
@pytest.mark.parametrize("m,d_out,gated", [(8192, 4096, False), (5000, 9001, False), (4100, 4100, False), (4096, 11008, True), (2040, 8184, True)])
def test_int8_of_few_columns(m, d_out, d_in, gated):
    """Two, three and five tiles a workgroup."""
    say(f"[wide] {m} x {d_out} x {d_in} gated {gated}")
    g = _gen(m + d_out + d_in)
    outs = d_out * (2 if gated else 1)
    x, w, xs, ws = _codes(g, m, d_in), _codes(g, outs, d_in), _scales(g, m), _scales(g, outs) / d_in**0.5
    ref = _scaled(x, xs, w, ws)
    for dtype in TYPES:
        y = qamw.int8_matmul(x, w, ws, x_scales=xs, gated=gated, out_dtype=dtype)
        expect(y, ref, gated, None, dtype)


@gpu
@pytest.mark.parametrize("d_in", [16, 144, 256])
@pytest.mark.parametrize("counts,d_out,gated", [([0, 700, 1301, 5, 256, 900, 511, 328], 4112, True), ([0, 700, 1301, 5, 256, 900, 511, 328], 8203, False),
                                                ([150, 90, 129, 231], 16400, False), ([300, 255, 257, 388], 16400, True)])
def test_int8_groups_of_few_columns(counts, d_out, d_in, gated):
    """Experts of uneven numbers of rows, gathered ones."""
    say(f"[wide] {counts} x {d_out} x {d_in} gated {gated}")
    n, m, outs = len(counts), sum(counts), d_out * (2 if gated else 1)
    g = _gen(m + d_out + d_in)
    x, w, xs, ws = _codes(g, m // 2, d_in), _codes(g, n, outs, d_in), _scales(g, m // 2), _scales(g, n, outs) / d_in**0.5
    rows = torch.randint(0, m // 2, (m,), generator=g, device=DEV, dtype=torch.int32)
    off = _offsets(counts)
    for dtype in TYPES:
        y = qamw.grouped_matmul(x, w, off, rows=rows, x_scales=xs, w_scales=ws, gated=gated, out_dtype=dtype)
        for e in range(n):
            a, b = int(off[e]), int(off[e + 1])
            if a < b:
                r = rows[a:b].long()
                expect(y[a:b], _scaled(x[r], xs[r], w[e], ws[e]), gated, None, (dtype, e))


# ---- which kernel ---------------------------------------------------------------------------------------------------------------------


@pytest.fixture
def by_tiles(request):
    """The kernel for many rows, by tiles of so many, whatever the estimate says."""
    rows = request.param
    before = qamw.set_kernel_path(rows)
    yield rows
    qamw.set_kernel_path(before)


def test_the_kernels_that_these_tests_are_for():
    """What the tests above multiply goes to the kernel for many rows, and so do prompts; one row does not."""
    plan, i8, bf16 = qamw.product_plan, qamw.DTYPE_I8, qamw.DTYPE_BF16
    for d_in in (16, 128, 144, 256, 272):
        for m, d_out, gated in ((8192, 4096, False), (5000, 9001, False), (4100, 4100, False), (4096, 11008, True), (2040, 8184, True)):
            p = plan(i8, m, d_out, d_in, gated=gated)
            assert p.many_rows and p.parts == 1
            assert -(-m // p.tile_rows) * -(-d_out // (128 if gated else 256)) > 256 + 8      # more than a tile a workgroup
    for d_in in (16, 144, 256):
        for m, n, d_out, gated in ((4001, 8, 4112, True), (4001, 8, 8203, False), (600, 4, 16400, False)):
            assert plan(i8, m, d_out, d_in, n, gated).many_rows
    for p in (plan(i8, 8192, 11008, 4096, gated=True), plan(i8, 8002, 11008, 4096, 8, True), plan(bf16, 32768, 2816, 2048, 64, True)):
        assert p == (True, 256, 1)
    assert not plan(i8, 1, 4096, 4096).many_rows and plan(i8, 500, 514, 13824).parts > 1


def test_the_switch_and_its_refusals():
    I = qamw.ERR_INVALID_ARG
    before = qamw.set_kernel_path(0)
    try:
        for rows in (64, 128, 256):
            qamw.set_kernel_path(rows)
            assert qamw.set_kernel_path(96) == rows and qamw.set_kernel_path(512) == rows and qamw.set_kernel_path(3) == rows
            assert qamw.product_plan(qamw.DTYPE_I8, 1, 48, 16) == (True, rows, 1) and qamw.product_plan(qamw.DTYPE_BF16, 500, 514, 13824, 3) == (True, rows, 1)
            need = qamw.int8_matmul_workspace_bytes.__wrapped__(qamw.DTYPE_I8, 500, 514, 13824)
            assert need > 0                                     # as much as without the switch
            qamw.set_kernel_path(0)
            assert need == qamw.int8_matmul_workspace_bytes.__wrapped__(qamw.DTYPE_I8, 500, 514, 13824)
    finally:
        qamw.set_kernel_path(before)
    out = (qamw.C.c_int * 3)()
    ask = lambda t=2, m=4, n=0, o=8, k=16, g=0, to=out: qamw.lib().qamw_product_plan(t, m, n, o, k, g, to)  # noqa: E731
    assert ask() == qamw.OK and ask(t=1, n=4) == qamw.OK and ask(t=1) == I and ask(t=0, n=4) == I and ask(t=3, n=4) == I
    assert ask(m=0) == I and ask(m=(1 << 22) + 1) == I and ask(n=-1) == I and ask(n=1025) == I and ask(o=0) == I and ask(o=(1 << 24) + 1) == I
    assert ask(k=0) == I and ask(k=131057) == I and ask(g=2) == I and ask(to=None) == I


# ---- from tile to tile, every tile, type and kind of result ------------------------------------------------------------------------------


def _operands(g, i8, n, outs, x_rows, d_in):
    """X, W, their scales in int8."""
    if i8:
        return _codes(g, x_rows, d_in), _codes(g, n, outs, d_in), _scales(g, x_rows), _scales(g, n, outs) / d_in**0.5
    return (torch.randn(x_rows, d_in, generator=g, device=DEV).bfloat16(), (torch.randn(n, outs, d_in, generator=g, device=DEV) / d_in**0.5).bfloat16(), None, None)


def _reference(x, xs, w, ws):
    """(sums with their scales, what fp32 sums of exact products in any order may be off: one rounding an addition)"""
    if xs is not None:
        return _scaled(x, xs, w, ws), None
    return _sums(x, w), _sums(x.abs(), w.abs()) * x.shape[1] * 2.0**-23


@gpu
@pytest.mark.parametrize("by_tiles", [64, 128, 256], indirect=True)
@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("whole", [False, True])
def test_one_matrix_from_tile_to_tile(by_tiles, i8, gated, whole):
    """2 to 3.4 tiles a workgroup, ends of rows and outputs inside a tile; `whole`: results stored by whole pieces of 16 bytes."""
    m = {64: 21, 128: 20, 256: 13}[by_tiles] * by_tiles - by_tiles // 2 - 3
    d_out = {False: 10245, True: 10248}[whole] // (2 if gated else 1)
    if whole:
        d_out -= d_out % 8
    outs = d_out * (2 if gated else 1)
    for d_bytes in (16, 400, 1040):
        d_in = d_bytes if i8 else d_bytes // 2
        say(f"[wide] by {by_tiles}: {m} x {d_out} x {d_in} int8 {i8} gated {gated}")
        g = _gen(m + outs + d_in)
        x, w, xs, ws = _operands(g, i8, 1, outs, m, d_in)
        assert qamw.product_plan(qamw.DTYPE_I8 if i8 else qamw.DTYPE_BF16, m, d_out, d_in, 1, gated) == (True, by_tiles, 1)
        ref, slack = _reference(x, xs, w[0], None if ws is None else ws[0])
        for dtype in TYPES:
            if i8:
                y = qamw.int8_matmul(x, w[0], ws[0], x_scales=xs, gated=gated, out_dtype=dtype)
            else:
                y = qamw.grouped_matmul(x, w, _offsets([m]), gated=gated, out_dtype=dtype)
            expect(y, ref, gated, slack, dtype)


@gpu
@pytest.mark.parametrize("by_tiles", [64, 128, 256], indirect=True)
@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("gather", [False, True])
def test_experts_from_tile_to_tile(by_tiles, i8, gated, gather):
    """Experts without rows, with one, with whole tiles and ragged ends, more than a workgroup's turn of them; rows that nobody has keep
    what they held, padding between rows too."""
    t = by_tiles
    counts = [0, 1, t, 2 * t - 1, 0, 0, t + 1, t // 2, 3 * t + 5, 7, 0] + [t // 4 + 1] * 6
    d_out, pad = (9001, 3) if gather else (9008, 0)
    if gated:
        d_out = d_out // 2 + (0 if pad else 4)
    n, m, outs = len(counts), sum(counts), d_out * (2 if gated else 1)
    for d_in in (128, 272):
        say(f"[wide] by {t}: {m} rows of {n} experts x {d_out} x {d_in} int8 {i8} gated {gated} gathered {gather}")
        g = _gen(m + outs + d_in)
        spare = 5
        x_rows = m // 2 + 3 if gather else m + spare
        x, w, xs, ws = _operands(g, i8, n, outs, x_rows, d_in)
        rows = torch.randint(0, x_rows, (m + spare,), generator=g, device=DEV, dtype=torch.int32) if gather else None
        assert qamw.product_plan(qamw.DTYPE_I8 if i8 else qamw.DTYPE_BF16, m + spare, d_out, d_in, n, gated) == (True, t, 1)
        off = _offsets(counts)
        for dtype in TYPES:
            y = _strided(torch.full((m + spare, d_out), -7.0, dtype=dtype), pad)
            qamw.grouped_matmul(x, w, off, rows=rows, x_scales=xs, w_scales=ws, gated=gated, out=y)
            assert (y[m:] == -7).all()
            if pad:
                assert torch.isnan(torch.as_strided(y, (m + spare, d_out + pad), y.stride(), y.storage_offset())[:, d_out:]).all()
            for e in range(n):
                a, b = int(off[e]), int(off[e + 1])
                if a < b:
                    r = torch.arange(a, b, device=DEV) if rows is None else rows[a:b].long()
                    ref, slack = _reference(x[r], None if xs is None else xs[r], w[e], None if ws is None else ws[e])
                    expect(y[a:b], ref, gated, slack, (dtype, e))


@gpu
@pytest.mark.parametrize("by_tiles", [64, 128, 256], indirect=True)
@pytest.mark.parametrize("i8", [False, True])
def test_offsets_that_do_not_ascend(by_tiles, i8):
    """Every other expert claims all places, so that there are many times the tiles that rows have room for: the call ends, and nothing is
    written beside Y.  Where every expert has the same matrix its claims agree, and what is written is right."""
    n, m, d_out, d_in = 40, 3 * by_tiles + 9, 515, 256
    say(f"[wide] by {by_tiles}: offsets up and down, {m} rows of {n} experts, int8 {i8}")
    g = _gen(m)
    x, w, xs, ws = _operands(g, i8, 1, d_out, m, d_in)
    off = torch.tensor([0, m] * (n // 2) + [0], dtype=torch.int32, device=DEV)
    guarded = torch.full((3 * m, d_out), 5.0, device=DEV)
    qamw.grouped_matmul(x, w.expand(n, -1, -1), off, x_scales=xs, w_scales=None if ws is None else ws.repeat(n, 1), out=guarded[m:2 * m])
    assert (guarded[:m] == 5).all() and (guarded[2 * m:] == 5).all()
    ref, slack = _reference(x, xs, w[0], None if ws is None else ws[0])
    expect(guarded[m:2 * m], ref, False, slack, "all places claimed")
