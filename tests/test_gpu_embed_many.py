"""More vectors than one launch of the look-up takes (2^31)."""
import pytest
import torch

from paper_2509_10613_amd import binding as sk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [1, 2, 3])
def test_more_vectors_than_a_launch_takes(D):
    """Columns of one vector (1, 2) and of two (3); checked where one launch ends and the next begins, and where the last ends."""
    per_row = {1: 1, 2: 1, 3: 2}[D]
    border = (2 ** 31 - 1) // per_row
    n = border + 1000
    table = torch.tensor([[float(D * v + d) for d in range(D)] for v in range(7)], dtype=torch.bfloat16, device="cuda")
    tokens = torch.zeros(n, dtype=torch.int32, device="cuda")
    ends = [(0, 50), (border - 60, border + 60), (n - 40, n)]
    gen = torch.Generator().manual_seed(D)
    for a, b in ends:
        tokens[a:b] = torch.randint(-1, 8, (b - a,), generator=gen, dtype=torch.int32).cuda()
    out = torch.full((n * D + 64,), 9.0, dtype=torch.bfloat16, device="cuda")
    sk.embed_fwd(tokens, table, 0.5, out=out[:n * D].view(n, D))
    assert torch.all(out[n * D:] == 9.0)
    rows = torch.cat([table * 0.5, torch.zeros((2, D), dtype=torch.bfloat16, device="cuda")])
    for a, b in ends:
        t = tokens[a:b].long()
        assert torch.equal(out[a * D:b * D].view(-1, D), rows[torch.where((t >= 0) & (t < 7), t, 7)])
    for a in range(50, n - 40, 1 << 28):
        b = min(a + (1 << 28), n - 40)
        some = (out[a * D:b * D].view(-1, D) != rows[0]).any(1).nonzero().flatten() + a
        assert torch.all((some >= border - 60) & (some < border + 60))
