"""Tables of vectors (sigtrain_embed_*) against the definition in 64 bits.

Tolerances: a value is rounded once, by at most half a step (eps / 2 relative, or half the smallest subnormal); the product before it is in
float for 16-bit types, with a float factor (2 * 2^-24 relative), in double otherwise.  A gradient row of c terms is summed in the
same precision u: at most (c + 2) u times the sum of the terms' magnitudes, wherever the additions are grouped."""
import itertools

import pytest
import torch

from paper_2509_10613_amd import autograd as ska
from paper_2509_10613_amd import binding as sk

pytestmark = pytest.mark.gpu

TYPES = [torch.float64, torch.float32, torch.bfloat16, torch.float16]


def unit(dtype):
    """Of the sums and products."""
    return 2.0 ** -24 if dtype in (torch.bfloat16, torch.float16) else 2.0 ** -53


def tiny(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def make(seed, shape, V, D, dtype, skew=False):
    gen = torch.Generator().manual_seed(seed)
    if skew:
        tokens = (torch.rand(shape, generator=gen, dtype=torch.float64) ** 6 * V).long().clamp_(0, max(V - 1, 0))
    else:
        tokens = torch.randint(0, V, shape, generator=gen)
    outside = torch.rand(shape, generator=gen) < 0.1
    tokens = torch.where(outside, torch.where(torch.rand(shape, generator=gen) < 0.5, -1, V), tokens)
    table = torch.randn((V, D), generator=gen, dtype=torch.float64).to(dtype)
    up = torch.randn((*shape, D), generator=gen, dtype=torch.float64).to(dtype)
    return tokens, table, up


def check(tokens, table, up, scale, out, grad):
    V, D = table.shape
    dtype = table.dtype
    flat = tokens.reshape(-1).long()
    there = (flat >= 0) & (flat < V)
    half, u = torch.finfo(dtype).eps / 2, unit(dtype)
    ref = torch.zeros((flat.numel(), D), dtype=torch.float64)
    ref[there] = table.double()[flat[there]] * scale
    got = out.double().cpu().reshape(-1, D)
    assert torch.all((got - ref).abs() <= (half + 2 * u) * ref.abs() * (1 + half) + tiny(dtype) / 2)
    assert torch.all(got[~there] == 0)
    if grad is None:
        return
    rows = up.double().reshape(-1, D)[there]
    want = torch.zeros((V, D), dtype=torch.float64).index_add_(0, flat[there], rows) * scale
    size = torch.zeros((V, D), dtype=torch.float64).index_add_(0, flat[there], rows.abs()) * abs(scale)
    count = torch.bincount(flat[there], minlength=V).double().unsqueeze(1)
    assert torch.all((grad.double().cpu() - want).abs() <= (count + 2) * u * size * (1 + half) + half * want.abs() + tiny(dtype) / 2)


def both(tokens, table, up, scale):
    t = table.cuda().requires_grad_()
    out = ska.embed(tokens.cuda(), t, scale)
    (grad,) = torch.autograd.grad(out, [t], up.cuda())
    return out.detach(), grad


# one token, odd and even columns, columns of more than one workgroup's width, one row, more rows than tokens and fewer, tokens around the
# 8192 that one workgroup sorts, more than one digit's rows (511, 512, 513) and more than two digits' (300000)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,D", [
    (1, 1, 1), (1, 7, 5), (3, 1, 16), (5, 40000, 3), (64, 2, 8), (257, 100, 7), (1000, 511, 24), (1001, 512, 33), (999, 513, 1),
    (300, 300, 2048), (65, 17, 4100), (40, 9, 9001), (8191, 1000, 4), (8192, 1000, 5), (8193, 1000, 6), (20000, 300000, 2), (50000, 3, 2),
])
def test_rows_and_gradients(n, V, D, dtype):
    tokens, table, up = make(n + V + D, (n,), V, D, dtype)
    print("embed n=%d V=%d D=%d %s: %s" % (n, V, D, dtype, describe(n, V, D, dtype)), flush=True)
    scale = 1.75 if n % 2 else -0.3
    check(tokens, table, up, scale, *both(tokens, table, up, scale))


def describe(n, V, D, dtype):
    import ctypes as C
    buf = C.create_string_buffer(256)
    sk._check(sk.load().sigtrain_describe(1, n, V, D, sk._ST_TYPES[dtype], 0, buf, len(buf)))
    return buf.value.decode()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape,V,D", [((128, 256), 1000, 5), ((7, 3001), 50257, 64), ((2, 4096), 12, 512), ((40000,), 70000, 9)])
def test_frequent_symbols(shape, V, D, dtype):
    tokens, table, up = make(V, shape, V, D, dtype, skew=True)
    check(tokens, table, up, 2.0, *both(tokens, table, up, 2.0))


@pytest.mark.parametrize("n,V,D", [(100, 5, 3), (30000, 1, 40), (9000, 4, 300)])
def test_every_token_the_same(n, V, D):
    for symbol in (0, V - 1):
        tokens, table, up = make(3, (n,), V, D, torch.float32)
        tokens = torch.full((n,), symbol)
        check(tokens, table, up, 1.0, *both(tokens, table, up, 1.0))


def test_no_token_stands_for_a_row():
    for n in (0, 1, 10000):
        tokens, table, up = make(n, (n,), 50, 6, torch.bfloat16)
        tokens = torch.full((n,), -7)
        out, grad = both(tokens, table, up, 3.0)
        assert out.shape == (n, 6) and torch.all(out == 0) and torch.all(grad == 0)


def test_tokens_far_outside_and_of_32_bits():
    tokens, table, up = make(5, (4, 50), 30, 9, torch.float32)
    tokens[0, 0], tokens[0, 1], tokens[1, 0] = 2 ** 40 + 3, -2 ** 63, 2 ** 32 + 1   # (the last two words of which are symbols)
    check(tokens, table, up, 1.0, *both(tokens, table, up, 1.0))
    tokens = tokens.clamp(-5, 40).int()
    check(tokens, table, up, 1.0, *both(tokens, table, up, 1.0))


def test_absent_upstream_infinities_stay_out_of_other_rows():
    """What padded positions hold upstream reaches no row; what a symbol's positions hold reaches its row alone."""
    tokens = torch.tensor([0, 1, -1, 2, 3, 1])
    _, table, up = make(1, (6,), 4, 11, torch.float32)
    up[2] = float("nan")
    up[4] = float("inf")
    out, grad = both(tokens, table, up, 1.0)
    assert torch.isfinite(grad[:3]).all() and torch.isinf(grad[3]).all()


def test_views_at_any_alignment():
    """Tables and upstream gradients that begin one element behind a 16-byte boundary, tokens with strides."""
    for dtype, D in itertools.product(TYPES, (5, 16)):
        tokens, table, up = make(9, (33, 4), 21, D, dtype)
        big = torch.empty(table.numel() + 1, dtype=dtype, device="cuda")
        t = big[1:].view(table.shape)
        t.copy_(table)
        t.requires_grad_()
        spread = torch.stack([tokens, tokens * 0], 0).permute(1, 2, 0).contiguous().cuda()[..., 0]
        assert not spread.is_contiguous()
        out = ska.embed(spread, t, 0.5)
        g = torch.empty(up.numel() + 1, dtype=dtype, device="cuda")[1:].view(up.shape)
        g.copy_(up)
        (grad,) = torch.autograd.grad(out, [t], g)
        check(tokens, table, up, 0.5, out.detach(), grad)
        (grad,) = torch.autograd.grad(ska.embed(spread, t, 0.5), [t], up.cuda().transpose(0, 1).contiguous().transpose(0, 1))
        check(tokens, table, up, 0.5, out.detach(), grad)


def test_the_same_call_gives_the_same_bits():
    tokens, table, up = make(2, (30000,), 500, 24, torch.float32, skew=True)
    a, b = both(tokens, table, up, 1.0), both(tokens, table, up, 1.0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_offsets_that_pass_32_bits():
    """2^31 entries and more in the output and the table; checked where they end."""
    V, D, n = 140000, 16384, 140000
    table = torch.zeros((V, D), dtype=torch.float16, device="cuda")
    table[-1] = 2.0
    table[131072] = 3.0
    tokens = torch.arange(n, device="cuda")
    out = sk.embed_fwd(tokens, table, 1.5)
    assert torch.all(out[-1] == 3.0) and torch.all(out[131072] == 4.5) and torch.all(out[131071] == 0)
    grad = sk.embed_bwd(tokens.flip(0).contiguous(), out, V, 2.0)
    assert torch.all(grad[0] == 6.0) and torch.all(grad[n - 1 - 131072] == 9.0) and torch.all(grad[-1] == 0)
    assert grad.sum(dtype=torch.float64).item() == (6.0 + 9.0) * D


def test_another_stream_and_a_captured_graph():
    tokens, table, up = make(4, (64, 50), 300, 20, torch.float32)
    want = both(tokens, table, up, 1.0)
    tokens, up = tokens.cuda(), up.cuda()
    t = table.cuda().requires_grad_()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        out = ska.embed(tokens, t, 1.0)
        (grad,) = torch.autograd.grad(out, [t], up)
    stream.synchronize()
    assert torch.equal(out.detach(), want[0]) and torch.equal(grad, want[1])
    del out, grad
    graph = torch.cuda.CUDAGraph()
    t2 = table.cuda()
    with torch.cuda.graph(graph):
        o = sk.embed_fwd(tokens, t2, 1.0)
        g = sk.embed_bwd(tokens, up, 300, 1.0)
    for i in range(3):
        o.zero_(), g.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(g, want[1])
        tokens.copy_(tokens.flip(0)), up.copy_(up.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        again = sk.embed_fwd(tokens, t2, 1.0), sk.embed_bwd(tokens, up, 300, 1.0)
        assert torch.equal(o, again[0]) and torch.equal(g, again[1])
        tokens.copy_(tokens.flip(0)), up.copy_(up.flip(0))


def test_gradient_against_differences():
    tokens, table, _ = make(6, (5, 4), 6, 3, torch.float64)
    assert torch.autograd.gradcheck(lambda t: ska.embed(tokens.cuda(), t, 1.3), (table.cuda().requires_grad_(),))


def test_more_tokens_than_the_last_launch_of_a_digit_adds_up():
    """More than 128 tiles of 8192 symbols: three launches per digit."""
    for V in (700, 40000):
        tokens, table, up = make(V, (1100000,), V, 3, torch.float32, skew=True)
        check(tokens, table, up, 1.5, *both(tokens, table, up, 1.5))


def test_what_lies_behind_a_workspace_stays():
    for dtype in TYPES:
        for n, V, D in ((100, 30, 7), (9000, 50, 5), (300, 4, 600)):
            tokens, table, up = make(n, (n,), V, D, dtype, skew=True)
            size = int(sk.load().sigtrain_embed_bwd_workspace_bytes(n, V, D, sk._ST_TYPES[dtype]))
            ws = torch.full((size + 4096,), 77, dtype=torch.uint8, device="cuda")
            out = torch.full((V * D + 64,), 7.0, dtype=dtype, device="cuda")
            sk.embed_bwd(tokens.cuda(), up.cuda(), V, 1.0, grad_table=out[:V * D].view(V, D), ws=ws[:size])
            assert torch.all(ws[size:] == 77) and torch.all(out[V * D:] == 7.0)
            rows = torch.full((n * D + 64,), 7.0, dtype=dtype, device="cuda")
            sk.embed_fwd(tokens.cuda(), table.cuda(), 1.0, out=rows[:n * D].view(n, D))
            assert torch.all(rows[n * D:] == 7.0)


def test_a_table_without_rows():
    out = sk.embed_fwd(torch.arange(5, device="cuda"), torch.empty((0, 3), device="cuda"))
    assert out.shape == (5, 3) and torch.all(out == 0)


def test_restored_tokens_and_shapes():
    tokens, table, up = make(31, (4, 6), 9, 5, torch.float64)
    want = both(tokens, table, up, 1.0)
    t = table.cuda().requires_grad_()
    with torch.autograd.graph.save_on_cpu():
        out = ska.embed(tokens.cuda(), t)
    (grad,) = torch.autograd.grad(out, [t], up.cuda())
    assert torch.equal(out.detach(), want[0]) and torch.equal(grad, want[1])
    out = ska.embed(tokens[0, 0].cuda(), t)
    assert out.shape == (5,)
    assert ska.embed(tokens[:0].cuda(), t).shape == (0, 6, 5)
