"""Cross entropy of a read-out (sigtrain_entropy_*) against the definition in 64 bits.

Tolerances, with u = 2^-23 for float sums (2^-52 for double; a step, not half: a matrix instruction may cut off) and R the largest |z - lse|:
 - a logit is a sum of D products: off by at most dz = (D + 1) u sum |h| |w| (its row's largest);
 - exp and log of the instruction set: (2 R + 4) u relative; sums of exponentials in a tree of at most 80 + V / 128 additions after another;
   so a probability is off by p e, e = 2 dz + (2 R + 90 + V / 128) u, and a loss by e + 4 u |lse|;
 - a logit's gradient G is u_t (p - 1[target]), off by |u_t| (p e + 2 u) and rounded to the arrays' type: half a step, eps / 2 |G| (float16
   is scaled before: 2^-25 of 2^-13 of the largest |u_t| at worst);
 - grad_h and grad_w add K such products by float: (K + 2) u times the sum of their magnitudes; and are rounded once."""
import pytest
import torch

from paper_2509_10613_amd import autograd as ska
from paper_2509_10613_amd import binding as sk

pytestmark = pytest.mark.gpu

TYPES = [torch.float64, torch.float32, torch.bfloat16, torch.float16]


def make(seed, T, V, D, dtype, spread=3.0, outside=0.15):
    gen = torch.Generator().manual_seed(seed)
    h = torch.randn((T, D), generator=gen, dtype=torch.float64).to(dtype)
    w = (torch.randn((V, D), generator=gen, dtype=torch.float64) * (spread / D ** 0.5)).to(dtype)
    targets = torch.randint(0, V, (T,), generator=gen)
    targets = torch.where(torch.rand((T,), generator=gen) < outside, torch.where(torch.rand((T,), generator=gen) < 0.5, -100, V), targets)
    return h, w, targets


def check(h, w, targets, reduction, up, loss, gh, gw):
    dtype, (T, D), V = h.dtype, h.shape, w.shape[0]
    u = 2.0 ** -52 if dtype == torch.float64 else 2.0 ** -23
    fin = torch.finfo(dtype)
    half, tiny = fin.eps / 2, fin.smallest_normal * fin.eps
    H, W = h.double(), w.double()
    there = (targets >= 0) & (targets < V)
    at = torch.where(there, targets, 0).long()
    H = torch.where(there.unsqueeze(1), H, 0.0)
    z = H @ W.T
    lse = torch.logsumexp(z, 1)
    losses = torch.where(there, lse - z.gather(1, at.unsqueeze(1)).squeeze(1), 0.0)
    R = (z - lse.unsqueeze(1)).abs().max().item() if T else 0.0
    dz = (D + 1) * u * (H.abs() @ W.abs().T).max().item() if T else 0.0
    e = 2 * dz + (2 * R + 90 + V / 128) * u
    count = int(there.sum())
    want = {"none": losses, "sum": losses.sum(), "mean": losses.sum() / max(count, 1)}[reduction]
    each = e + 4 * u * lse.abs().max().item() if T else 0.0
    slack = {"none": each, "sum": each * T, "mean": each}[reduction]
    assert torch.all((loss.double().cpu() - want).abs() <= slack + u * want.abs()), (loss, want)
    if reduction == "none":
        assert torch.all(loss.cpu()[~there] == 0)
    if gh is None and gw is None:
        return
    ut = up.double() if reduction == "none" else up.double().expand(T) / (max(count, 1) if reduction == "mean" else 1)
    ut = torch.where(there, ut, 0.0)
    p = torch.exp(z - lse.unsqueeze(1))
    hot = torch.zeros_like(z).scatter_(1, at.unsqueeze(1), 1.0)
    G = ut.unsqueeze(1) * (p - hot)
    most = ut.abs().max().item() if T else 0.0
    floor = most * 2.0 ** -38 if dtype == torch.float16 else tiny / 2
    dG = ut.abs().unsqueeze(1) * (p * e + 2 * u) + half * G.abs() + floor
    dG = torch.where(there.unsqueeze(1), dG, 0.0)
    if gh is not None:
        want = G @ W
        bound = dG @ W.abs() + (V + 2) * u * (G.abs() @ W.abs())
        assert torch.all((gh.double().cpu() - want).abs() <= bound * (1 + 2 * half) + half * want.abs() + tiny / 2)
        assert torch.all(gh.cpu()[~there] == 0)
    if gw is not None:
        want = G.T @ H
        bound = dG.T @ H.abs() + (T + 2) * u * (G.abs().T @ H.abs())
        assert torch.all((gw.double().cpu() - want).abs() <= bound * (1 + 2 * half) + half * want.abs() + tiny / 2)


def run(h, w, targets, reduction="mean", up=None):
    a, b = h.cuda().requires_grad_(), w.cuda().requires_grad_()
    loss = ska.linear_cross_entropy(a, b, targets.cuda(), reduction)
    if up is None:
        gen = torch.Generator().manual_seed(11)
        up = torch.randn(loss.shape, generator=gen, dtype=torch.float64).to(loss.dtype)
    gh, gw = torch.autograd.grad(loss, [a, b], up.cuda())
    return up, loss.detach(), gh, gw


# one row, one class, one column; sizes around the tiles' 128 (and 256), steps of 128 bytes and their multiples, odd columns that go through
# copies, more rows than classes and fewer, features as wide as a signature
SIZES = [(1, 1, 1), (1, 2, 3), (2, 1, 64), (1, 1000, 64), (3, 700, 128), (17, 33, 65), (63, 64, 64), (64, 65, 127), (127, 129, 128),
         (128, 128, 256), (129, 127, 60), (130, 1000, 341), (255, 257, 32), (256, 256, 64), (257, 511, 96), (300, 77, 1024), (5, 3000, 192), (1000, 10, 16),
         (40, 130, 5461)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D", SIZES)
def test_loss_and_gradients(T, V, D, dtype):
    h, w, targets = make(T + V + D, T, V, D, dtype)
    if T <= 3:
        targets[0] = V - 1
    print("entropy T=%d V=%d D=%d %s" % (T, V, D, dtype), flush=True)
    for reduction in ("mean", "none", "sum") if T in (17, 130, 257) else ("mean",) if T % 2 else ("none",):
        check(h, w, targets, reduction, *run(h, w, targets, reduction))


@pytest.mark.parametrize("dtype", TYPES)
def test_pieces_of_the_classes(dtype):
    """Workspaces from the least up: several pieces, and the same results as with one."""
    T, V, D = 70, 1500, 72
    h, w, targets = make(1, T, V, D, dtype)
    hd, wd, td = h.cuda(), w.cuda(), targets.cuda()
    dt = sk._ST_TYPES[dtype]
    size = sk.load().sigtrain_entropy_workspace_bytes
    for part in (0.0, 0.3, 1.0):
        sizes = [int(size(b, T, V, D, dt, 1) + part * (size(b, T, V, D, dt, 0) - size(b, T, V, D, dt, 1))) for b in (0, 1)]
        ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
        loss, lse, rows = sk.entropy_fwd(hd, wd, td, "mean", ws=ws[0])
        up = torch.tensor(0.7, dtype=loss.dtype)
        gh, gw = sk.entropy_bwd(hd, wd, td, lse, rows, up.cuda(), "mean", ws=ws[1])
        check(h, w, targets, "mean", up, loss, gh, gw)
        assert rows.item() == int(((targets >= 0) & (targets < V)).sum())


def test_one_side_alone():
    h, w, targets = make(3, 50, 300, 40, torch.bfloat16)
    up, loss, gh, gw = run(h, w, targets)
    a = h.cuda().requires_grad_()
    (only,) = torch.autograd.grad(ska.linear_cross_entropy(a, w.cuda(), targets.cuda()), [a], up.cuda())
    assert torch.equal(only, gh)
    b = w.cuda().requires_grad_()
    (only,) = torch.autograd.grad(ska.linear_cross_entropy(h.cuda(), b, targets.cuda()), [b], up.cuda())
    assert torch.equal(only, gw)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_without_a_target_reach_nothing(dtype):
    h, w, targets = make(4, 200, 90, 24, dtype, outside=0.4)
    clean = run(h, w, targets)
    dirty = h.clone()
    out = (targets < 0) | (targets >= 90)
    dirty[out] = float("nan")
    dirty[out.nonzero()[::2, 0]] = float("inf")
    got = run(dirty, w, targets)
    for a, b in zip(clean, got):
        assert torch.equal(a.cpu(), b.cpu())


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_no_row_has_a_target(reduction):
    for T in (0, 1, 130):
        h, w, _ = make(5, T, 60, 20, torch.float32)
        up, loss, gh, gw = run(h, w, torch.full((T,), -1), reduction)
        assert loss.shape == ((T,) if reduction == "none" else ()) and torch.all(loss == 0)
        assert gh.shape == h.shape and torch.all(gh == 0) and torch.all(gw == 0)


def test_large_and_masked_logits():
    """Logits of +-1e4 beside each other, and classes whose logits are minus infinity (as a vector of the read-out that masks them has them)."""
    h, w, targets = make(6, 40, 200, 16, torch.float32)
    w[::7] *= 1e4
    w[100:150, 0], h[:, 0] = float("-inf"), h[:, 0].abs() + 0.1
    targets = torch.where((targets >= 100) & (targets < 150), 3, targets)
    a = h.cuda()
    loss = ska.linear_cross_entropy(a, w.cuda(), targets.cuda(), "none").double().cpu()
    z = h.double() @ w.double().T
    assert torch.isneginf(z[:, 100:150]).all()
    there = (targets >= 0) & (targets < 200)
    want = torch.where(there, torch.logsumexp(z, 1) - z.gather(1, targets.clamp(0, 199).unsqueeze(1)).squeeze(1), 0.0)
    slack = 4 * 17 * 2.0 ** -23 * (h.double().abs() @ w.double().abs().nan_to_num(posinf=0.0).T).max(1).values + 1e-4
    assert torch.all((loss - want).abs() <= slack)


def test_gradients_of_halves_that_would_be_subnormal():
    """A mean over many rows: unscaled, the logits' gradients (about 1e-8) would be float16's smallest numbers."""
    T, V, D = 4096, 300, 64
    h, w, targets = make(7, T, V, D, torch.float16)
    check(h, w, targets, "mean", *run(h, w, targets, "mean", torch.tensor(1.0)))


def test_shapes_with_more_axes_and_other_layouts():
    h, w, targets = make(8, 60, 50, 30, torch.float32)
    want = run(h, w, targets, "none")
    a = h.view(5, 12, 30).transpose(0, 1).contiguous().cuda().transpose(0, 1).requires_grad_()
    b = w.T.contiguous().cuda().T.requires_grad_()
    y = targets.view(5, 12).int().cuda()
    loss = ska.linear_cross_entropy(a, b, y, "none")
    gh, gw = torch.autograd.grad(loss, [a, b], want[0].view(5, 12).cuda())
    assert loss.shape == (5, 12) and torch.equal(loss.flatten(), want[1])
    assert torch.equal(gh.reshape(60, 30), want[2]) and torch.equal(gw, want[3])
    # a read-out that begins one element behind a 16-byte boundary
    for dtype in TYPES:
        h, w, targets = make(9, 33, 40, 128, dtype)
        want = run(h, w, targets)
        big = torch.empty(w.numel() + 1, dtype=dtype, device="cuda")[1:].view(w.shape)
        big.copy_(w)
        high = torch.empty(h.numel() + 1, dtype=dtype, device="cuda")[1:].view(h.shape)
        high.copy_(h)
        big.requires_grad_(), high.requires_grad_()
        loss = ska.linear_cross_entropy(high, big, targets.cuda())
        gh, gw = torch.autograd.grad(loss, [high, big], want[0].cuda())
        assert torch.equal(loss, want[1]) and torch.equal(gh, want[2]) and torch.equal(gw, want[3])


def test_the_same_call_gives_the_same_bits():
    h, w, targets = make(10, 300, 2000, 200, torch.bfloat16)
    for a, b in zip(run(h, w, targets), run(h, w, targets)):
        assert torch.equal(a, b)


def test_another_stream_and_a_captured_graph():
    h, w, targets = make(12, 100, 600, 64, torch.float16)
    up, *want = run(h, w, targets)
    h, w, targets, up = h.cuda(), w.cuda(), targets.cuda(), up.cuda()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        loss, lse, rows = sk.entropy_fwd(h, w, targets)
        gh, gw = sk.entropy_bwd(h, w, targets, lse, rows, up)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((loss, gh, gw), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, lse, rows = sk.entropy_fwd(h, w, targets)
        gh, gw = sk.entropy_bwd(h, w, targets, lse, rows, up)
    for _ in range(3):
        for t in (loss, gh, gw):
            t.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((loss, gh, gw), want))
        h.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        l2, lse2, rows2 = sk.entropy_fwd(h, w, targets)
        again = (l2, *sk.entropy_bwd(h, w, targets, lse2, rows2, up))
        assert all(torch.equal(a, b) for a, b in zip((loss, gh, gw), again))
        h.mul_(2.0)


def test_gradients_against_differences():
    h, w, targets = make(13, 6, 5, 4, torch.float64)
    h, w = h.cuda().requires_grad_(), w.cuda().requires_grad_()
    for reduction in ("mean", "sum", "none"):
        assert torch.autograd.gradcheck(lambda a, b: ska.linear_cross_entropy(a, b, targets.cuda(), reduction), (h, w))


def test_many_classes():
    """More classes than one piece takes with the default workspace."""
    T, V, D = 64, 200001, 1024
    h, w, targets = make(14, T, V, D, torch.bfloat16, outside=0.0)
    check(h, w, targets, "mean", *run(h, w, targets))


# several pieces of few rows, of logits in parts (few tiles of many steps), of rows in steps of their own; between the least workspace and the best
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D", [(9, 1300, 50), (16, 700, 128), (40, 900, 9000), (300, 1100, 136)])
def test_pieces_of_other_shapes(T, V, D, dtype):
    h, w, targets = make(T + D, T, V, D, dtype)
    hd, wd, td = h.cuda(), w.cuda(), targets.cuda()
    dt = sk._ST_TYPES[dtype]
    size = sk.load().sigtrain_entropy_workspace_bytes
    for part in (0.0, 0.5, 1.0):
        sizes = [int(size(b, T, V, D, dt, 1) + part * (size(b, T, V, D, dt, 0) - size(b, T, V, D, dt, 1))) for b in (0, 1)]
        ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
        loss, lse, rows = sk.entropy_fwd(hd, wd, td, "sum", ws=ws[0])
        up = torch.tensor(-1.3, dtype=loss.dtype)
        gh, gw = sk.entropy_bwd(hd, wd, td, lse, rows, up.cuda(), "sum", ws=ws[1])
        check(h, w, targets, "sum", up, loss, gh, gw)


def test_what_lies_behind_a_workspace_stays():
    """Nothing is written past the bytes that were given, nor past the last row of an output."""
    for dtype in TYPES:
        for T, V, D in ((7, 300, 33), (130, 500, 64), (40, 300, 9000)):
            h, w, targets = make(T, T, V, D, dtype)
            hd, wd, td = h.cuda(), w.cuda(), targets.cuda()
            size = sk.load().sigtrain_entropy_workspace_bytes
            for least in (0, 1):
                sizes = [int(size(b, T, V, D, sk._ST_TYPES[dtype], least)) for b in (0, 1)]
                bufs = [torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda") for n in sizes]
                loss, lse, rows = sk.entropy_fwd(hd, wd, td, "sum", ws=bufs[0][:sizes[0]])
                sk.entropy_bwd(hd, wd, td, lse, rows, torch.ones_like(loss), "sum", ws=bufs[1][:sizes[1]])
                assert all(torch.all(b[n:] == 77) for b, n in zip(bufs, sizes))


def test_large_tiles_in_a_captured_graph():
    """Tiles of 256 (more LDS than a kernel has without asking) recorded and replayed."""
    T, V, D = 2100, 9000, 256
    h, w, targets = make(21, T, V, D, torch.bfloat16)
    hd, wd, td = h.cuda(), w.cuda(), targets.cuda()
    up = torch.tensor(1.0, device="cuda")
    l, lse, rows = sk.entropy_fwd(hd, wd, td)
    want = (l, *sk.entropy_bwd(hd, wd, td, lse, rows, up))
    check(h, w, targets, "mean", up.cpu(), *want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l2, lse2, rows2 = sk.entropy_fwd(hd, wd, td)
        got = (l2, *sk.entropy_bwd(hd, wd, td, lse2, rows2, up))
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        sk.entropy_fwd(hd, wd, td)


def test_restored_and_changed_inputs():
    """Saved tensors that come back from the host give the same gradients; inputs that have changed since are an error."""
    h, w, targets = make(22, 50, 70, 40, torch.float32)
    want = run(h, w, targets)
    a, b, y = h.cuda().requires_grad_(), w.cuda().requires_grad_(), targets.cuda()
    with torch.autograd.graph.save_on_cpu():
        loss = ska.linear_cross_entropy(a, b, y)
    for x, g in zip(torch.autograd.grad(loss, [a, b], want[0].cuda()), want[2:]):
        assert torch.equal(x, g)
    for changed in (0, 1, 2):
        a, b, y = h.cuda().requires_grad_(), w.cuda().requires_grad_(), targets.cuda()
        loss = ska.linear_cross_entropy(a * 1.0, b * 1.0 if changed != 1 else b, y)
        hd, wd = a.view(5, 10, 40) * 1.0, b * 1.0
        loss = ska.linear_cross_entropy(hd, wd, y.view(5, 10))
        (hd, wd, y)[changed].mul_(1)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            torch.autograd.grad(loss, [a, b])


def test_a_second_derivative_is_refused():
    h, w, targets = make(23, 10, 12, 8, torch.float64)
    a, b = h.cuda().requires_grad_(), w.cuda().requires_grad_()
    ga, gb = torch.autograd.grad(ska.linear_cross_entropy(a, b, targets.cuda()) ** 2, [a, b], create_graph=True)
    with pytest.raises(RuntimeError, match="twice"):
        (ga.sum() + gb.sum()).backward()
    t = torch.randn(6, 3, device="cuda", requires_grad=True)
    (gt,) = torch.autograd.grad((ska.embed(torch.tensor([1, 4], device="cuda"), t) ** 2).sum(), [t], create_graph=True)
    with pytest.raises(RuntimeError, match="twice"):
        gt.sum().backward()


def test_two_threads_at_once():
    """Calls from two threads on streams of their own."""
    import threading
    sets = [make(30 + i, 90, 400, 64, torch.bfloat16) for i in range(2)]
    want = [run(*s) for s in sets]
    got, torch_sync = [None, None], torch.cuda.synchronize
    torch_sync()

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got[i] = run(*sets[i])
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for a, b in zip(want, got):
        assert all(torch.equal(x.cpu(), y.cpu()) for x, y in zip(a, b))


def test_a_row_alone_and_no_axes():
    h, w, targets = make(24, 1, 30, 20, torch.float32)
    targets[0] = 3
    want = run(h, w, targets, "none")
    a = h.view(20).cuda().requires_grad_()
    loss = ska.linear_cross_entropy(a, w.cuda(), targets.view(()).cuda(), "none")
    (g,) = torch.autograd.grad(loss, [a], want[0].view(()).cuda())
    assert loss.shape == () and torch.equal(loss, want[1][0]) and torch.equal(g, want[2][0])


@pytest.mark.parametrize("dtype", TYPES)
def test_few_classes_and_wide_rows(dtype):
    """Products divided into parts on either side; one piece that takes less than two (several pieces need sums of grad_h)."""
    for T, V, D in ((1500, 40, 1100), (500, 300, 1030)):
        h, w, targets = make(T, T, V, D, dtype)
        check(h, w, targets, "mean", *run(h, w, targets))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D", [(70, 90, 8), (70, 90, 72), (130, 300, 200), (40, 257, 1992), (600, 700, 136)])
def test_rows_that_end_within_a_step(T, V, D, dtype):
    """Rows of whole 16 bytes that are read as they lie: what is behind a row's end, here a class that is masked by minus infinity, stays out of it."""
    h, w, targets = make(T + D, T, V, D, dtype)
    h[:, 0] = h[:, 0].abs() + 0.5
    masked = torch.arange(5, V, 7)
    keep = torch.ones(V, dtype=torch.bool)
    keep[masked] = False
    targets = torch.where((targets >= 0) & (targets < V) & ~keep[targets.clamp(0, V - 1)], 0, targets)
    clean = torch.cumsum(keep, 0) - 1                       # the classes that are left, by number
    few = torch.where((targets >= 0) & (targets < V), clean[targets.clamp(0, V - 1)], targets.clamp(max=-1))
    w[masked, 0] = float("-inf")
    wd = w.cuda()
    loss, lse, rows = sk.entropy_fwd(h.cuda(), wd, targets.cuda(), "none")
    check(h, w[keep], few, "none", None, loss, None, None)
    up = torch.randn((T,), generator=torch.Generator().manual_seed(1), dtype=torch.float64).to(loss.dtype)
    _, gw = sk.entropy_bwd(h.cuda(), wd, targets.cuda(), lse, rows, up.cuda(), "none", want_h=False)
    assert torch.all(gw[masked.cuda()] == 0)
    check(h, w[keep], few, "none", up, loss, None, gw[keep.cuda()])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_tiles_of_rows_that_end_within_a_step(dtype):
    T, V, D = 2100, 5001, 200
    h, w, targets = make(25, T, V, D, dtype)
    check(h, w, targets, "mean", *run(h, w, targets))


# at most 16 classes and wide rows: one class and all 16, columns of parts and of one, rows of one wave and of several ranges
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D", [(1, 3, 600), (17, 1, 512), (30, 2, 1001), (130, 10, 5461), (3000, 16, 515), (700, 7, 2048), (64, 16, 20000)])
def test_few_classes_of_wide_rows(T, V, D, dtype):
    h, w, targets = make(T + V + D, T, V, D, dtype, outside=0.2 if T > 1 else 0.0)
    for reduction in ("mean", "none"):
        check(h, w, targets, reduction, *run(h, w, targets, reduction))
    clean = run(h, w, targets)
    dirty = h.clone()
    dirty[(targets < 0) | (targets >= V)] = float("nan")
    assert all(torch.equal(a.cpu(), b.cpu()) for a, b in zip(clean, run(dirty, w, targets)))
    hd, wd, td = h.cuda(), w.cuda(), targets.cuda()
    size = sk.load().sigtrain_entropy_workspace_bytes
    for least in (0, 1):   # a workspace of the least bytes, and nothing written behind it
        sizes = [int(size(b, T, V, D, sk._ST_TYPES[dtype], least)) for b in (0, 1)]
        bufs = [torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda") for n in sizes]
        loss, lse, rows = sk.entropy_fwd(hd, wd, td, "sum", ws=bufs[0][:sizes[0]])
        gh, gw = sk.entropy_bwd(hd, wd, td, lse, rows, torch.ones_like(loss), "sum", ws=bufs[1][:sizes[1]])
        check(h, w, targets, "sum", torch.ones((), dtype=loss.dtype), loss, gh, gw)
        assert all(torch.all(b[n:] == 77) for b, n in zip(bufs, sizes))
        only_h = sk.entropy_bwd(hd, wd, td, lse, rows, torch.ones_like(loss), "sum", want_w=False)[0]
        only_w = sk.entropy_bwd(hd, wd, td, lse, rows, torch.ones_like(loss), "sum", want_h=False)[1]
        assert torch.equal(only_h, sk.entropy_bwd(hd, wd, td, lse, rows, torch.ones_like(loss), "sum")[0])
        assert torch.equal(only_w, sk.entropy_bwd(hd, wd, td, lse, rows, torch.ones_like(loss), "sum")[1])
