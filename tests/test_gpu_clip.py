"""Norms and clipping (sigtrain_grad_norm, sigtrain_clip) against 64-bit sums.

Tolerances: the norm is a root of a sum of n squares in double, (n + 2) 2^-53 relative at worst, half of that after the root; a scaled value is
rounded once (eps / 2 of its type) after a product in double, or in float for 16-bit inputs (with a float factor: 2 * 2^-24)."""
import math

import pytest
import torch

from paper_2509_10613_amd import autograd as ska
from paper_2509_10613_amd import binding as sk

pytestmark = pytest.mark.gpu

TYPES = [torch.float64, torch.float32, torch.bfloat16, torch.float16]


def make(seed, sizes, dtypes, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=gen, dtype=torch.float64) * scale).to(dtypes[i % len(dtypes)]) for i, n in enumerate(sizes)]


def norm_of(grads):
    return math.sqrt(math.fsum((g.double() ** 2).sum().item() for g in grads))


def check(grads, bound, norm, outs):
    want = norm_of(grads)
    n = sum(g.numel() for g in grads)
    assert norm.dtype == torch.float64 and norm.shape == ()
    assert abs(norm.item() - want) <= (n + 4) * 2.0 ** -53 * want
    f = min(1.0, bound / want) if want > 0 else 1.0
    for g, o in zip(grads, outs):
        fin = torch.finfo(o.dtype)
        if f == 1.0:
            assert torch.equal(o.cpu(), g.to(o.dtype))
            continue
        u = 2.0 ** -23 if g.dtype in (torch.bfloat16, torch.float16) else 0.0
        ref = g.double() * f
        err = (o.double().cpu() - ref).abs()
        assert torch.all(err <= (fin.eps / 2 * (1 + u) + u + (n + 6) * 2.0 ** -53) * ref.abs() + fin.smallest_normal * fin.eps / 2)


SIZES = [[1], [7], [0, 3, 0], [8] * 5, [255, 256, 257], [16383, 16384, 16385], [100000, 1, 31], [70001] * 9, [5] * 95, [5] * 96, [5] * 97, list(range(300)),
         [3000001]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%dx%d" % (len(s), max(s)))
def test_norm_and_clipping(sizes, dtype):
    print("clip", len(sizes), max(sizes), dtype, flush=True)
    grads = make(len(sizes), sizes, [dtype])
    dev = [g.cuda() for g in grads]
    norm = ska.grad_norm(dev)
    check(grads, math.inf, norm, dev)
    for part in (0.3, 2.0):
        bound = part * norm.item()
        outs = [torch.full_like(d, 9.0) for d in dev]
        check(grads, bound, ska.clip_grad_norm(dev, bound, out=outs), outs)
        assert all(torch.equal(d.cpu(), g) for d, g in zip(dev, grads))
        same = [d.clone() for d in dev]
        check(grads, bound, ska.clip_grad_norm(same, bound), same)
        assert all(torch.equal(a, b) for a, b in zip(same, outs))


def test_types_together_and_into_each_other():
    grads = make(1, [1000, 33, 5000, 129, 64, 7, 2000, 4, 90, 91, 92, 93, 94, 95, 96, 97], TYPES, 0.1)
    dev = [g.cuda() for g in grads]
    for shift in range(4):
        outs = [torch.empty_like(d, dtype=TYPES[(i // 4 + i + shift) % 4]) for i, d in enumerate(dev)]
        check(grads, 0.5, ska.clip_grad_norm(dev, 0.5, out=outs), outs)


def test_arrays_one_behind_the_other_at_any_alignment():
    for dtype in TYPES:
        grads = make(2, [1, 5, 17000, 3, 40001], [dtype])
        flat = torch.cat(grads).cuda()
        at, dev = 0, []
        for g in grads:
            dev.append(flat[at:at + g.numel()])
            at += g.numel()
        check(grads, 1.0, ska.clip_grad_norm(dev, 1.0), dev)


def test_squares_beyond_the_types_range():
    for dtype, scale in ((torch.float32, 1e30), (torch.bfloat16, 1e30), (torch.float16, 2e4), (torch.float32, 1e-30)):
        grads = make(3, [1000, 77], [dtype], scale)
        dev = [g.cuda() for g in grads]
        check(grads, 1.0, ska.clip_grad_norm(dev, 1.0), dev)


def test_infinite_and_undefined_norms_pass_everything_on():
    for bad, dtype in ((math.inf, torch.float32), (math.nan, torch.bfloat16), (-math.inf, torch.float64)):
        grads = make(4, [50, 20000], [dtype])
        grads[1][19999] = bad
        dev = [g.cuda() for g in grads]
        norm = ska.clip_grad_norm(dev, 0.1)
        assert (math.isnan if math.isnan(bad) else math.isinf)(norm.item())
        assert all(torch.equal(d.cpu().nan_to_num(nan=7.0), g.nan_to_num(nan=7.0)) for d, g in zip(dev, grads))


def test_bounds_at_the_ends():
    grads = make(5, [300], [torch.float32])
    dev = [grads[0].cuda()]
    ska.clip_grad_norm(dev, 0.0)
    assert torch.all(dev[0] == 0)
    assert ska.clip_grad_norm(dev, 0.0).item() == 0 and torch.all(dev[0] == 0)
    assert ska.grad_norm([]).item() == 0 and ska.clip_grad_norm([], 1.0).item() == 0
    assert ska.grad_norm(torch.zeros(0, device="cuda")).item() == 0
    dev = [grads[0].cuda()]
    assert abs(ska.clip_grad_norm(dev, math.inf).item() - norm_of(grads)) <= 1e-13 * norm_of(grads) and torch.equal(dev[0].cpu(), grads[0])


def test_a_single_tensor_and_other_layouts():
    gen = torch.Generator().manual_seed(6)
    g = torch.randn((40, 30), generator=gen)
    d = g.cuda()
    for view in (d.clone().T, d.clone()[::2], d.clone()[:, 3:9]):
        before = view.double().cpu()
        norm = ska.clip_grad_norm(view, 2.0)
        assert abs(norm.item() - before.norm().item()) <= 1e-12 * norm.item()
        assert torch.all((view.double().cpu() - before * (2.0 / norm.item())).abs() <= 2.0 ** -24 * before.abs())
        out = torch.empty((view.shape[1], view.shape[0]), device="cuda").T
        view.copy_(before)
        ska.clip_grad_norm(view, 2.0, out=out)
        assert torch.all((out.double().cpu() - before * (2.0 / norm.item())).abs() <= 2.0 ** -24 * before.abs())


def test_another_stream_and_a_captured_graph():
    grads = make(7, [1000, 30000, 5] * 40, [torch.float32, torch.bfloat16])
    dev = [g.cuda() for g in grads]
    outs = [torch.empty_like(d) for d in dev]
    norm = sk.clip(dev, 3.0, out=outs)
    want = [o.clone() for o in outs]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for o in outs:
            o.zero_()
        again = sk.clip(dev, 3.0, out=outs)
    stream.synchronize()
    assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n = sk.clip(dev, 3.0, out=outs)
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(n, norm) and all(torch.equal(a, b) for a, b in zip(outs, want))


def test_in_place_scaling_is_seen_by_autograd():
    x = torch.randn(5, device="cuda")
    w = torch.ones(5, device="cuda", requires_grad=True)
    y = (w * x).sum()
    ska.clip_grad_norm(x, 1e-3)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_refusals():
    a, b = torch.randn(8, device="cuda"), torch.randn(4, device="cuda")
    with pytest.raises(sk.SigKernelError, match="overlaps"):
        ska.clip_grad_norm([a, a], 1.0)
    with pytest.raises(sk.SigKernelError, match="overlaps"):
        ska.clip_grad_norm([a[:6], a[4:]], 1.0)
    with pytest.raises(sk.SigKernelError, match="negative or NaN"):
        ska.clip_grad_norm([a], -1.0)
    with pytest.raises(ValueError, match="outputs"):
        ska.clip_grad_norm([a, b], 1.0, out=[a])
    with pytest.raises(ValueError, match="shape"):
        ska.clip_grad_norm([a], 1.0, out=[b])
    with pytest.raises(TypeError):
        ska.grad_norm([a.int()])
    before = a.clone()
    with pytest.raises(TypeError):
        ska.clip_grad_norm([a, b.long()], 1e-3)
    assert torch.equal(a, before)
