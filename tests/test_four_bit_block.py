"""The example's block in 4 bits: norms, scored routing, the experts' products, combination and the norm after it, each step against plain
operations in 64 bits on what the step before it gave, and the whole captured and replayed."""
import importlib.util
import os

import pytest
import torch

from paper_2605_26339_amd import qamw

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def _example():
    spec = importlib.util.spec_from_file_location("routed_layer_example", os.path.join(ROOT, "examples", "routed_layer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _values(q):
    """What an Mx4 stands for, in 64 bits, on the CPU, from its layout."""
    codes, scales, d = q.codes.cpu().reshape(-1, q.codes.shape[-1]), q.scales.cpu().reshape(-1, q.scales.shape[-1]), q.columns
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)
    v = table[torch.stack([codes & 15, codes >> 4], 2).long()].reshape(codes.shape[0], -1, 32)
    blocks = torch.arange(v.shape[1])
    e = scales[:, 16 * (blocks // 16) + 4 * (blocks % 4) + blocks % 16 // 4].double() - 127
    return (v * torch.exp2(e)[:, :, None]).flatten(1)[:, :d].reshape(*q.codes.shape[:-1], d)


def _norm(h, w):
    return h / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-6) * w


@pytest.mark.parametrize("tokens,experts,k,groups,top,width,hidden", [(1, 8, 2, 2, 1, 256, 128), (5, 16, 3, 4, 2, 288, 160), (150, 12, 4, 3, 2, 512, 320)])
def test_block_step_by_step(tokens, experts, k, groups, top, width, hidden):
    print(f"[4-bit block] {tokens} tokens, {k} of {experts} experts in {groups} groups, {width} x {hidden}", flush=True)
    ex = _example()
    gen = torch.Generator().manual_seed(tokens)
    rand = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    up, down = rand(experts, 2 * hidden, width) / width**0.5, rand(experts, width, hidden) / hidden**0.5
    up, down = (ex.in_4_bits(ex.Experts(e.bfloat16().cuda(), None)) for e in (up, down))
    h, router = rand(tokens, width).bfloat16(), (rand(experts, width) / width**0.5).bfloat16()
    w, w2, bias, gate = 1 + 0.1 * rand(width), 1 + 0.1 * rand(width), 0.1 * rand(experts), torch.rand(width, generator=gen).bfloat16()
    dev = [t.cuda() for t in (h, w, router, bias, w2, gate)]
    run = lambda s: ex.routed_block(s, dev[1], dev[2], dev[3], up, down, k, groups, top, dev[4], gate=dev[5])  # noqa: E731
    stream, q = run(dev[0])

    _, x = qamw.block_norm(dev[0], dev[1])
    want = _norm(h.double(), w.double())
    assert ((x.cpu().double() - want).abs() <= want.abs() * (2.0**-8 + 2.0**-19)).all()
    logits = x @ dev[2].t()
    r = qamw.route_scored(logits, k, bias=dev[3], groups=groups, top_groups=top)
    c = torch.sigmoid(logits.cpu().double()) + bias.double()
    each = experts // groups
    of_group = c.view(tokens, groups, each).topk(2, dim=2).values.sum(2)
    stays = torch.zeros(tokens, groups, dtype=torch.bool).scatter_(1, torch.sort(of_group, dim=1, descending=True, stable=True).indices[:, :top], True)
    chosen = torch.sort(c.masked_fill(~stays.repeat_interleave(each, 1), -torch.inf), dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(r.experts.cpu().long(), chosen)
    weights = torch.sigmoid(logits.cpu().double()).gather(1, chosen)
    weights = weights / weights.sum(1, keepdim=True)
    # the experts, in 64 bits on the rows' 4 bits; hidden values as the kernel rounded them, since the next 4 bits go by them
    xv, wu, wd = _values(qamw.mx4_quantize(x)), _values(up), _values(down)
    hid = qamw.mx4_grouped_matmul(x, up, r.offsets, rows=r.rows, gated=True)
    hv = _values(qamw.mx4_quantize(hid))
    y = torch.zeros(tokens, width, dtype=torch.float64)
    for t in range(tokens):
        for j in range(k):
            e, at = int(chosen[t, j]), int(r.positions[t, j])
            g, u = (wu[e] @ xv[t]).chunk(2)
            s = g * torch.sigmoid(g) * u
            # two sums of `width` terms, each addition off by 2^-23 of the terms' sizes at most, and bf16
            size = (wu[e].abs() @ xv[t].abs()).chunk(2)
            slack = s.abs() * 2.0**-8 + (1 + 2.0**-8) * width * 2.0**-23 * (1.1 * size[0] * (u.abs() + 1) + (g.abs() + 1) * size[1]) + s.abs() * (g.abs() + 16) * 2.0**-22
            assert ((hid[at].cpu().double() - s).abs() <= slack).all()
            y[t] += weights[t, j] * (wd[e] @ hv[at])
    got = qamw.combine(qamw.mx4_grouped_matmul(hid, down, r.offsets), r.positions, r.weights)
    # products and their weighted sum are rounded to bf16, 2^-8 each and at most
    bound = sum(weights[:, j:j + 1] * torch.stack([(wd[int(e)] @ hv[int(p)]).abs() for e, p in zip(chosen[:, j], r.positions[:, j])]) for j in range(k))
    assert ((got.cpu().double() - y).abs() <= (bound + y.abs()) * 2.0**-8 * 1.01 + 1e-4).all()
    after = h.double() + gate.double() * got.cpu().double()
    assert ((stream.cpu().double() - after).abs() <= after.abs() * 2.0**-8 + (h.double().abs() + after.abs()) * 2.0**-22).all()
    _, wanted = qamw.block_norm(stream, dev[4], quantize="mx4")
    assert torch.equal(q.codes, wanted.codes) and torch.equal(q.scales, wanted.scales)

    held = dev[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s2, q2 = run(held)
    for shift in range(3):
        held.copy_(dev[0].roll(shift, 0))
        graph.replay()
        torch.cuda.synchronize()
        s3, q3 = run(held)
        assert torch.equal(s2, s3) and torch.equal(q2.codes, q3.codes) and torch.equal(q2.scales, q3.scales)


def test_layers_of_all_widths_agree():
    """The example's layer in 4 bits, 8 bits and bf16: an error of 4 bits is a step of a sixth to a third of a value, rounded by half of it, some 8 % of a value in the
    mean square with two significant bits; four such operands meet (inputs, hidden values, both weights, gate and up), so that below half the size is left."""
    ex = _example()
    router, up, down = ex.build(8, 512, 384)
    x = torch.randn(90, 512, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    logits = x @ router.t()
    want = ex.routed_layer(x, logits, up, down, 2).double()
    four = ex.routed_layer(x, logits, ex.in_4_bits(up), ex.in_4_bits(down), 2).double()
    assert float((four - want).norm() / want.norm()) < 0.5
