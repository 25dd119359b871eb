"""clip_grad_norm of tensors that share entries and are not contiguous: an error, and nothing written."""
import pytest
import torch

from paper_2509_10613_amd import autograd as ska
from paper_2509_10613_amd import binding as sk

pytestmark = pytest.mark.gpu


def test_a_strided_tensor_given_twice():
    x = torch.randn(40, 30, generator=torch.Generator().manual_seed(1)).cuda()
    before = x.clone()
    for grads in ([x[:, ::2], x[:, ::2]], [x.T, x], [x[:, :7], x[:, :9]], [torch.ones(3, device="cuda"), x.T, x.T]):
        with pytest.raises(sk.SigKernelError, match="overlaps"):
            ska.clip_grad_norm(grads, 1e-3)
        with pytest.raises(sk.SigKernelError, match="overlaps"):
            ska.clip_grad_norm([g.clone() for g in grads], 1e-3, out=grads)
        assert torch.equal(x, before)


def test_an_expanded_tensor_is_refused_before_others_are_scaled():
    x, row = torch.randn(9, device="cuda"), torch.randn(4, device="cuda")
    before, kept = x.clone(), row.clone()
    with pytest.raises(ValueError, match="share memory"):
        ska.clip_grad_norm([x, row.expand(3, 4)], 1e-3)
    assert torch.equal(x, before) and torch.equal(row, kept)
    assert abs(ska.grad_norm([x, row.expand(3, 4)]).item() ** 2 - (x.double().norm() ** 2 + 3 * row.double().norm() ** 2).item()) <= 1e-12 * 100


def test_parts_of_one_matrix_side_by_side():
    x = torch.randn(40, 30, generator=torch.Generator().manual_seed(2)).cuda()
    before = x.double()
    norm = ska.clip_grad_norm([x[:, :10], x[:, 10:25], x[:, 25:]], 0.5)
    assert abs(norm.item() - before.norm().item()) <= 1e-12 * norm.item()
    assert torch.all((x.double() - before * (0.5 / norm)).abs() <= 2.0 ** -24 * before.abs())
