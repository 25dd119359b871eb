"""Which tensors clip_grad_norm refuses to write because they share entries, for layouts that are not contiguous (addresses only; no GPU)."""
import random

import pytest
import torch

from paper_2509_10613_amd import autograd as ska
from paper_2509_10613_amd import binding as sk

X = torch.zeros(8, 8)
FLAT = torch.zeros(100)


@pytest.mark.parametrize("outs", [
    [X[:, ::2], X[:, ::2]], [X.T, X], [X.T, X.T], [X[:, :3], X], [X, X[:, 2:4]], [X[::2], X[2:6].T], [X.T, X[3:5]], [X[:, 1:3], X[:, 1:4]],
    [X[:, :4], X[:, 2:6]],     [FLAT[::2], FLAT[:7]], [FLAT[0:9:2], FLAT[8:20]], [torch.ones(3), X.T, torch.ones(2), X[7, 7:].expand(1)],
], ids=range(12))
def test_shared_entries(outs):
    with pytest.raises(sk.SigKernelError, match="overlaps"):
        ska._refuse_shared(outs)
    with pytest.raises(sk.SigKernelError, match="overlaps"):
        ska._refuse_shared(outs[::-1])


@pytest.mark.parametrize("outs", [
    [X[:, :4], X[:, 4:]], [X[::2], X[1::2]], [X[:4].T, X[4:].T], [X[:, 0], X[:, 1], X[:, 7]], [FLAT[::2], FLAT[1::2]], [X.T, torch.zeros(3, 4).T],
    [X[:0], X.T], [X[2:2].T, X[2:3, :0], X], [FLAT[0:9:2], FLAT[9:20]], [torch.zeros(1, 5).expand(1, 5).T, torch.zeros(())],
], ids=range(10))
def test_no_shared_entries(outs):
    ska._refuse_shared(outs)
    ska._refuse_shared(outs[::-1])


def test_a_tensor_that_shares_entries_with_itself():
    for t in (torch.zeros(4).expand(3, 4), torch.zeros(3, 1).expand(3, 2).T):
        with pytest.raises(ValueError, match="share memory"):
            ska._refuse_shared([torch.zeros(2), t])


def test_against_the_sets_of_bytes():
    rng, base = random.Random(3), torch.zeros(4096, dtype=torch.uint8)

    def view():
        flat = base.view(rng.choice([torch.float32, torch.float64, torch.bfloat16]))
        axes = rng.randrange(0, 4)
        return flat.as_strided([rng.randrange(1, 6) for _ in range(axes)], [rng.randrange(1, 20) for _ in range(axes)], rng.randrange(0, 60))

    def memory(t):
        at = torch.full(t.shape, t.data_ptr() - base.data_ptr())
        for k, (n, s) in enumerate(zip(t.shape, t.stride())):
            at = at + (torch.arange(n) * s * t.element_size()).view([n if i == k else 1 for i in range(t.dim())])
        return {a + j for a in at.flatten().tolist() for j in range(t.element_size())}

    seen = [0, 0]
    for _ in range(3000):
        a, b = view(), view()
        shared = bool(memory(a) & memory(b))
        seen[shared] += 1
        if shared:
            with pytest.raises(sk.SigKernelError, match="overlaps"):
                ska._refuse_shared([a, b])
        else:
            ska._refuse_shared([a, b])
    assert min(seen) > 300
