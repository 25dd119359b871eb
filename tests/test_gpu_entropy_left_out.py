"""Rows that take no part in the gradients of the cross entropy: without a target, or with an upstream gradient of 0.  Infinities and NaN in the read-out
reach no row of grad_h that is left out, and what a row that is left out holds does not reach grad_w, whichever kernels the sizes select."""
import pytest
import torch

from paper_2509_10613_amd import binding as sk
from tests.test_gpu_entropy import TYPES, check, make

pytestmark = pytest.mark.gpu

# one piece as a whole, logits and products in parts, 256 x 256 tiles, few rows, a single one, few classes of wide rows
SIZES = [(130, 300, 200), (40, 130, 5461), (1500, 40, 1100), (2100, 5001, 200), (9, 1300, 50), (1, 70, 33), (130, 10, 5461), (12, 16, 515)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("bad", [float("-inf"), float("nan")])
def test_rows_without_a_target_beside_infinities_of_the_read_out(T, V, D, dtype, bad):
    h, w, targets = make(T + V, T, V, D, dtype, outside=0.3)
    if T == 1:
        targets[0] = -1
    w[V // 2, D // 3] = bad
    out = (targets < 0) | (targets >= V)
    assert out.any()
    hd, wd, td = h.cuda(), w.cuda(), targets.cuda()
    for reduction in ("mean", "none"):
        loss, lse, rows = sk.entropy_fwd(hd, wd, td, reduction)
        gh, _ = sk.entropy_bwd(hd, wd, td, lse, rows, torch.ones_like(loss), reduction)
        assert torch.all(gh[out.cuda()] == 0)
        only = sk.entropy_bwd(hd, wd, td, lse, rows, torch.ones_like(loss), reduction, want_w=False)[0]
        assert torch.all(only[out.cuda()] == 0)


@pytest.mark.parametrize("dtype", TYPES)
def test_pieces_of_the_classes(dtype):
    T, V, D = 70, 1500, 72
    h, w, targets = make(1, T, V, D, dtype, outside=0.3)
    w[1499, 0], w[3, 1] = float("inf"), float("nan")
    out = ((targets < 0) | (targets >= V)).cuda()
    hd, wd, td = h.cuda(), w.cuda(), targets.cuda()
    least = int(sk.load().sigtrain_entropy_workspace_bytes(1, T, V, D, sk._ST_TYPES[dtype], 1))
    loss, lse, rows = sk.entropy_fwd(hd, wd, td, "sum")
    gh, _ = sk.entropy_bwd(hd, wd, td, lse, rows, torch.ones_like(loss), "sum", ws=torch.empty(least, dtype=torch.uint8, device="cuda"))
    assert torch.all(gh[out] == 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D", SIZES)
def test_rows_whose_upstream_is_zero(T, V, D, dtype):
    """The gradients are those of the rows that are left; the others may hold anything."""
    h, w, targets = make(T + D, T, V, D, dtype, outside=0.0)
    up = torch.randn((T,), generator=torch.Generator().manual_seed(5), dtype=torch.float64)
    up[::3] = 0.0
    up = up.to(torch.float64 if dtype == torch.float64 else torch.float32)
    hd, wd, td = h.cuda(), w.cuda(), targets.cuda()
    loss, lse, rows = sk.entropy_fwd(hd, wd, td, "none")
    gh, gw = sk.entropy_bwd(hd, wd, td, lse, rows, up.cuda(), "none")
    check(h, w, targets, "none", up, loss, gh, gw)
    assert torch.all(gh[::3] == 0)
    hd[::3] = float("nan")
    loss, lse, rows = sk.entropy_fwd(hd, wd, td, "none")
    assert all(torch.equal(a, b) for a, b in zip((gh, gw), sk.entropy_bwd(hd, wd, td, lse, rows, up.cuda(), "none")))
