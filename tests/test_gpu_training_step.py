"""Embedding, signatures, read-out, loss, gradients and clipping in one step, against the same step in 64 bits on the CPU."""
import numpy as np
import pytest
import torch

from oracle import signature as osig
from paper_2509_10613_amd import autograd as ska

pytestmark = pytest.mark.gpu


def step(tokens, table, w, targets, N, bound):
    x = ska.embed(tokens, table, 0.5)
    S = ska.signature(x, N)
    loss = ska.linear_cross_entropy(S, w, targets)
    grads = list(torch.autograd.grad(loss, [table, w]))
    raw = [g.clone() for g in grads]
    norm = ska.clip_grad_norm(grads, bound)
    return loss.detach(), raw, norm, grads


def inputs(seed, B=12, L=20, d=3, N=3, V=40, C=25, dtype=torch.float64):
    gen = torch.Generator().manual_seed(seed)
    n = sum(d ** k for k in range(N + 1))
    tokens = torch.randint(0, V, (B, L), generator=gen)
    table = torch.randn((V, d), generator=gen, dtype=torch.float64).to(dtype)
    w = (torch.randn((C, n), generator=gen, dtype=torch.float64) * 0.3).to(dtype)
    targets = torch.randint(0, C, (B,), generator=gen)
    targets[3] = -1
    return tokens, table, w, targets


def loss_of(tokens, table, w, targets, N):
    S = torch.tensor(osig.signature((0.5 * table[tokens]).numpy().astype(np.float64), N))
    z = S @ w.T
    there = targets >= 0
    return (torch.logsumexp(z, 1) - z.gather(1, targets.clamp(min=0).unsqueeze(1)).squeeze(1))[there].mean()


@pytest.mark.parametrize("dtype", [torch.float64, torch.float32])
def test_a_step_and_its_gradients(dtype):
    tokens, table, w, targets = inputs(1, dtype=dtype)
    got = step(tokens.cuda(), table.cuda().requires_grad_(), w.cuda().requires_grad_(), targets.cuda(), 3, 1e-2)
    table, w = table.double(), w.double()
    ref = loss_of(tokens, table, w, targets, 3)
    tol = 1e-10 if dtype == torch.float64 else 2e-4   # (the signatures' own tolerances, 1e-10 and 1e-5, through a read-out of 40 entries of 0.3)
    assert abs(got[0].item() - ref.item()) <= tol
    # gradients against central differences of the step's own arithmetic in 64 bits: off by eps^2 / 6 third derivatives and 1e-16 / eps
    eps, gen = 1e-5, torch.Generator().manual_seed(2)
    for i, p in enumerate((table, w)):
        for _ in range(4):
            v = torch.randn(p.shape, generator=gen, dtype=torch.float64)
            ends = [loss_of(tokens, *(q + s * eps * v if q is p else q for q in (table, w)), targets, 3).item() for s in (1, -1)]
            slope = (got[1][i].double().cpu() * v).sum().item()
            assert abs(slope - (ends[0] - ends[1]) / (2 * eps)) <= (1e-6 if dtype == torch.float64 else 2e-3) * (1 + abs(slope))
    total = sum((g.double() ** 2).sum().item() for g in got[1]) ** 0.5
    assert abs(got[2].item() - total) <= 1e-12 * total and total > 1e-2
    for raw, g in zip(got[1], got[3]):
        ref = raw.double() * (1e-2 / total)
        assert torch.all((g.double() - ref).abs() <= (torch.finfo(dtype).eps / 2 + 1e-12) * ref.abs())


def test_a_step_as_a_captured_graph():
    tokens, table, w, targets = (t.cuda() for t in inputs(3))
    table.requires_grad_(), w.requires_grad_()
    want = step(tokens, table, w, targets, 3, 1e-2)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(tokens, table, w, targets, 3, 1e-2)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(tokens, table, w, targets, 3, 1e-2)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0])
        assert torch.equal(got[1][1], want[1][1])   # (the signatures' gradients are sums by atomics: to rounding)
        assert torch.allclose(got[1][0], want[1][0], rtol=1e-10, atol=1e-13) and torch.allclose(got[2], want[2], rtol=1e-10)
        step(tokens, table, w, targets, 3, 1e-2)


def test_the_squared_mmd_of_symbols():
    """A table trained on the squared MMD of two sets of symbol sequences: gradients against differences."""
    tokens, table, _, _ = inputs(4, B=6, L=8, V=9)
    other = tokens.flip(1).contiguous().cuda()
    tokens = tokens.cuda()
    f = lambda t: ska.sig_mmd2(ska.embed(tokens, t, 0.3), ska.embed(other, t, 0.3))  # noqa: E731
    assert torch.autograd.gradcheck(f, (table.cuda().requires_grad_(),), eps=1e-5, atol=1e-7)
