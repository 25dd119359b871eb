"""Tables scaled by numbers that a float does not hold.

Tolerances: products with such a scale are formed in double, 2^-53, and rounded once (eps / 2 of the type, or half its smallest subnormal); the sums of the
gradient before them are in float for 16-bit types: (c + 2) 2^-24 of the terms' magnitudes for c terms."""
import pytest
import torch

from paper_2509_10613_amd import autograd as ska

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1e39, -3e60, 1e300, 1e-39, -1e-45, 1e-60, 1e-310])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("n,V,D", [(50, 12, 7), (9000, 5, 33), (300, 400, 1)])
def test_scales_beyond_a_float(n, V, D, dtype, scale):
    gen = torch.Generator().manual_seed(n)
    fin = torch.finfo(dtype)
    tokens = torch.randint(-1, V, (n,), generator=gen)
    # entries that the scale brings back into the type's range, as far as the type has them, and zeros
    size = min(max(1.0 / abs(scale), fin.smallest_normal), fin.max / 1e5)
    table = (torch.randn((V, D), generator=gen, dtype=torch.float64) * size).to(dtype)
    up = (torch.randn((n, D), generator=gen, dtype=torch.float64) * size).to(dtype)
    table[::3], up[::5] = 0.0, 0.0
    up[tokens == 1] = 0.0   # (a row of sums that are 0)
    t = table.cuda().requires_grad_()
    out = ska.embed(tokens.cuda(), t, scale)
    (grad,) = torch.autograd.grad(out, [t], up.cuda())
    there, tiny = tokens >= 0, fin.smallest_normal * fin.eps
    ref = torch.zeros((n, D), dtype=torch.float64)
    ref[there] = table.double()[tokens[there]] * scale
    largest = fin.max * (1 + fin.eps / 4)   # (beyond this a result may be infinite, and beyond half a step more it is)

    def same(got, ref, slack):
        got = got.double().cpu()
        inside = ref.abs() + slack < largest
        assert not torch.isnan(got).any() and torch.all(got[ref == 0] == 0)
        assert torch.all((got - ref).abs()[inside] <= slack[inside])
        beyond = ref.abs() - slack > largest
        assert torch.all(got[beyond] == ref[beyond].sign() * float("inf"))

    same(out.detach(), ref, (fin.eps / 2 + 2.0 ** -52) * ref.abs() + tiny / 2)
    rows = up.double()[there]
    total = torch.zeros((V, D), dtype=torch.float64).index_add_(0, tokens[there], rows)
    each = torch.zeros((V, D), dtype=torch.float64).index_add_(0, tokens[there], rows.abs())
    count = torch.bincount(tokens[there], minlength=V).double().unsqueeze(1)
    u = 2.0 ** -24 if dtype != torch.float32 else 2.0 ** -53
    ref = torch.where(each == 0, 0.0, total * scale)
    same(grad, ref, (count + 2) * u * (each * abs(scale)) * (1 + fin.eps) + fin.eps / 2 * ref.abs() + tiny / 2)


@pytest.mark.parametrize("scale", [2.0 ** -126, 3.4e38, 0.0, -0.0])
def test_the_ends_of_a_floats_range(scale):
    table = torch.tensor([[0.0, 1.0, -0.5, 2.0 ** -7]], dtype=torch.bfloat16, device="cuda").requires_grad_()
    out = ska.embed(torch.zeros(2, dtype=torch.long, device="cuda"), table, scale)
    (grad,) = torch.autograd.grad(out, [table], torch.full((2, 4), 0.25, dtype=torch.bfloat16, device="cuda"))
    want = (table.detach().double() * scale).to(torch.bfloat16)
    assert torch.equal(out.detach(), want.expand(2, 4))
    assert torch.equal(grad, torch.full((1, 4), 0.5 * scale, dtype=torch.float64, device="cuda").to(torch.bfloat16))
