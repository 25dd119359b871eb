"""Upstream gradients of the rows' own (reduction "none") that lie far apart: a row's gradient of h is as good as if it were alone.

Tolerances are those of test_gpu_entropy, each row's by its own |u_t|.  With u = 2^-23 (2^-52 for double) and e a probability's error relative to it:
 - G_tv = u_t (p - hot) is rounded to the arrays' type after the power of two nearest to u_t is taken out (the quotient of mantissas that is left is in
   (1/2, 2)); float16 holds it times 2^14, so where it is subnormal the half step of 2^-25 is at most 2^-25 / (2^14 / 2) |u_t| = 2^-38 |u_t|; other types'
   smallest numbers are below any of these sizes;
 - grad_w multiplies G by h with the powers of two put back.  They are exact unless h becomes subnormal: float16's copy of h has its largest entry at 2^14
   or more, so half a step of 2^-25 is at most 2^-39 of that one, and beside quotients of at least 1/4 of each other at most 2^-37 B |p - hot| for B = max |u h|
   (over rows whose upstream is finite); other types': the smallest normal number times the largest |u|."""
import pytest
import torch

from paper_2509_10613_amd import binding as sk
from tests.test_gpu_entropy import TYPES, make

pytestmark = pytest.mark.gpu


def check(h, w, targets, up, gh, gw, rows):
    """gh in the rows `rows`; gw, if given, of all rows."""
    dtype, (T, D), V = h.dtype, h.shape, w.shape[0]
    u = 2.0 ** -52 if dtype == torch.float64 else 2.0 ** -23
    fin = torch.finfo(dtype)
    half, tiny = fin.eps / 2, fin.smallest_normal * fin.eps
    H, W = h.double(), w.double()
    z = H @ W.T
    lse = torch.logsumexp(z, 1, keepdim=True)
    R = (z - lse).abs().max().item()
    e = 2 * (D + 1) * u * (H.abs() @ W.abs().T).max().item() + (2 * R + 90 + V / 128) * u
    there = (targets >= 0) & (targets < V)
    ut = torch.where(there, up.double(), 0.0).unsqueeze(1)
    p = torch.exp(z - lse)
    off = p - torch.zeros_like(z).scatter_(1, targets.clamp(0, V - 1).unsqueeze(1), 1.0)
    floor = 2.0 ** -38 if dtype == torch.float16 else tiny / 2
    G, dG = ut * off, ut.abs() * (p * e + 2 * u + half * off.abs() + floor)
    want = (G @ W)[rows]
    bound = (dG @ W.abs() + (V + 2) * u * (G.abs() @ W.abs()))[rows]
    got = gh.double().cpu()[rows]
    assert torch.all((got - want).abs() <= bound * (1 + 2 * half) + half * want.abs() + tiny / 2)
    if gw is None:
        return
    most = (ut.abs() * H.abs()).max().item() * 2.0 ** -37 if dtype == torch.float16 else ut.abs().max().item() * fin.smallest_normal
    want = G.T @ H
    bound = dG.T @ H.abs() + (T + 2) * u * (G.abs().T @ H.abs()) + most * off.abs().sum(0).unsqueeze(1)
    assert torch.all((gw.double().cpu() - want).abs() <= bound * (1 + 2 * half) + half * want.abs() + tiny / 2)


def gradients(h, w, targets, up, **kw):
    hd, wd, td = h.cuda(), w.cuda(), targets.cuda()
    _, lse, rows = sk.entropy_fwd(hd, wd, td, "none")
    return sk.entropy_bwd(hd, wd, td, lse, rows, up.cuda(), "none", **kw)


# tiles of three sizes, logits and products in parts, pieces (the least workspace), one row, few classes of wide rows
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D,least", [(64, 5000, 80, False), (40, 300, 5461, False), (2100, 9000, 64, False), (70, 1500, 72, True), (1, 3000, 33, False),
                                         (130, 10, 1000, False)])
@pytest.mark.parametrize("decades", [0, 8])
def test_upstreams_decades_apart(T, V, D, least, decades, dtype):
    h, w, targets = make(T + V + D, T, V, D, dtype, spread=0.5, outside=0.1 if T > 1 else 0.0)
    gen = torch.Generator().manual_seed(2)
    up = torch.randn((T,), generator=gen, dtype=torch.float64) * 10.0 ** -(torch.rand((T,), generator=gen, dtype=torch.float64) * decades).round()
    if dtype == torch.float16:
        up *= 64.0   # (losses are scaled so that small gradients stay in the type's range)
    up = up.to(torch.float64 if dtype == torch.float64 else torch.float32)
    ws = None
    if least:
        ws = torch.empty(int(sk.load().sigtrain_entropy_workspace_bytes(1, T, V, D, sk._ST_TYPES[dtype], 1)), dtype=torch.uint8, device="cuda")
    gh, gw = gradients(h, w, targets, up, ws=ws)
    check(h, w, targets, up, gh, gw, torch.arange(T))
    again = gradients(h, w, targets, up, ws=ws)
    assert torch.equal(gh, again[0]) and torch.equal(gw, again[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D", [(64, 700, 80), (33, 9, 600)])
def test_one_infinite_upstream(T, V, D, dtype):
    """It makes its own row's gradients infinite or NaN, and those of the read-out; the other rows' are theirs."""
    h, w, targets = make(T + V, T, V, D, dtype, outside=0.0)
    up = torch.randn((T,), generator=torch.Generator().manual_seed(3), dtype=torch.float64) * 100
    up[5], up[9] = float("inf"), float("nan")
    up = up.to(torch.float64 if dtype == torch.float64 else torch.float32)
    gh, gw = gradients(h, w, targets, up)
    fine = torch.isfinite(up)
    check(h, w, targets, torch.where(fine, up, 0.0), gh, None, fine)
    assert not torch.isfinite(gh[5]).any() and torch.isnan(gh[9]).all() and not torch.isfinite(gw).any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.float64])
def test_upstreams_at_the_ends_of_the_range(dtype):
    T, V, D = 40, 500, 48
    h, w, targets = make(4, T, V, D, dtype, outside=0.0)
    up = torch.ones(T, dtype=torch.float64)
    up[::4], up[1::4], up[2::4] = 1e30, 1e-28, -1e-20
    up = up.to(torch.float64 if dtype == torch.float64 else torch.float32)
    gh, gw = gradients(h, w, targets, up)
    check(h, w, targets, up, gh, gw, torch.arange(T))


def test_the_largest_upstream_at_a_row_of_zeros():
    T, V, D = 20, 300, 64
    h, w, targets = make(6, T, V, D, torch.float16, outside=0.0)
    up = torch.full((T,), 1e-4)
    h[3], up[3] = 0.0, 1e4
    gh, gw = gradients(h, w, targets, up)
    check(h, w, targets, up, gh, gw, torch.arange(T))
    h[:] = 0.0
    gh, gw = gradients(h, w, targets, up)
    check(h, w, targets, up, gh, gw, torch.arange(T))
    assert torch.all(gw == 0)


def test_a_captured_graph_with_other_upstreams_at_every_replay():
    T, V, D = 50, 700, 40
    h, w, targets = (t.cuda() for t in make(7, T, V, D, torch.float16))
    up = torch.randn((T,), generator=torch.Generator().manual_seed(8)).cuda()
    _, lse, rows = sk.entropy_fwd(h, w, targets, "none")
    sk.entropy_bwd(h, w, targets, lse, rows, up, "none")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = sk.entropy_bwd(h, w, targets, lse, rows, up, "none")
    for factor in (1.0, 1e-3, 1e-3, 1e5):
        up.mul_(factor)
        for t in got:
            t.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        want = sk.entropy_bwd(h, w, targets, lse, rows, up, "none")
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and got[1].any()
