"""Factors of clipping that a float does not hold, and 16-bit tensors that become doubles.

Tolerances, with n entries: the norm in double is off by (n + 4) 2^-53 relative; the factor by two roundings more; the product by one, in double, or
for 16-bit inputs whose factor is a normal float in float (2^-24 for the factor, 2^-24 for the product); the result is rounded once."""
import math

import pytest
import torch

from paper_2509_10613_amd import autograd as ska

pytestmark = pytest.mark.gpu


def check(given, outs, bound, norm, product):
    n = sum(g.numel() for g in given)
    want = math.sqrt(math.fsum((g.double() ** 2).sum().item() for g in given))
    assert abs(norm.item() - want) <= (n + 4) * 2.0 ** -53 * want
    f = bound / want
    for g, o in zip(given, outs):
        fin = torch.finfo(o.dtype)
        ref = g.double() * f
        slack = (fin.eps / 2 * (1 + product) + product + (n + 8) * 2.0 ** -53) * ref.abs() + fin.smallest_normal * fin.eps / 2
        assert torch.all((o.double().cpu() - ref).abs() <= slack)
        assert ref.abs().max() > 100 * slack.max()   # (the slack says something: bfloat16's half step alone is 2^-8, a 256th)


# factors of about 1e-41, 1e-44 and 1e-48
@pytest.mark.parametrize("bound", [1.0, 1e-3, 1e-7])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32, torch.float64])
def test_a_factor_below_the_normal_floats(bound, out):
    gen = torch.Generator().manual_seed(1)
    given = [(torch.randn(k, generator=gen, dtype=torch.float64) * 5e37).clamp(-3e38, 3e38).to(torch.bfloat16) for k in (300001, 5, 700000)]
    dev = [g.cuda() for g in given]
    outs = [torch.full_like(d, 9.0, dtype=out) for d in dev]
    norm = ska.clip_grad_norm(dev, bound, out=outs)
    check(given, outs, bound, norm, 0.0)
    if out == torch.bfloat16:
        assert torch.equal(ska.clip_grad_norm(dev, bound), norm) and all(torch.equal(a, b) for a, b in zip(dev, outs))


@pytest.mark.parametrize("dtype,scale,bound", [(torch.bfloat16, 1.0, 0.1), (torch.float16, 1.0, 0.1), (torch.bfloat16, 1e-30, 1e-35), (torch.bfloat16, 1e30, 1.0)])
def test_16_bits_into_doubles_are_rounded_once(dtype, scale, bound):
    gen = torch.Generator().manual_seed(2)
    given = [(torch.randn(k, generator=gen, dtype=torch.float64) * scale).to(dtype) for k in (1003, 70000)]
    dev = [g.cuda() for g in given]
    outs = [torch.empty_like(d, dtype=torch.float64) for d in dev]
    check(given, outs, bound, ska.clip_grad_norm(dev, bound, out=outs), 0.0)


def test_a_product_below_the_normal_floats_from_a_factor_that_is_one():
    gen = torch.Generator().manual_seed(3)
    given = [torch.cat([torch.tensor([1e30], dtype=torch.float64), torch.randn(5000, generator=gen, dtype=torch.float64)]).to(torch.bfloat16)]
    dev = [g.cuda() for g in given]
    outs = [torch.empty_like(d, dtype=torch.float64) for d in dev]
    check(given, outs, 1e-5, ska.clip_grad_norm(dev, 1e-5, out=outs), 0.0)
    outs = [torch.empty_like(d, dtype=torch.float32) for d in dev]
    check(given, outs, 1e-5, ska.clip_grad_norm(dev, 1e-5, out=outs), 2.0 ** -23)
