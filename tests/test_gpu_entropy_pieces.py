"""Cross entropy in pieces of the classes whose last has fewer steps than the others' products are divided among.  Tolerances: those of test_gpu_entropy."""
import ctypes as C
import re

import pytest
import torch

from paper_2509_10613_amd import binding as sk
from tests.test_gpu_entropy import check, make

pytestmark = pytest.mark.gpu

BF16, F16, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64


# the workspace's bytes decide the pieces; rows of w that are copied and (856 channels) rows that are read as they lie, up to the last class and no further
@pytest.mark.parametrize("T,V,D,dtype,size", [(94, 260, 16, F64, 622262), (7, 527, 39, F64, 669824), (75, 1035, 5, F32, 515440), (435, 539, 56, F32, 3093774),
                                              (36, 5178, 856, BF16, 3453237), (36, 5178, 856, F16, 3453237), (2, 6451, 976, BF16, 3306115),
                                              (978, 39956, 529, BF16, 20513728)])
@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_a_last_piece_of_few_steps(T, V, D, dtype, size, reduction):
    print("entropy T=%d V=%d D=%d %s %s in %d bytes" % (T, V, D, dtype, reduction, size), flush=True)
    buf = C.create_string_buffer(512)
    sk._check(sk.load().sigtrain_describe(3, T, V, D, sk._ST_TYPES[dtype], size, buf, len(buf)))
    plan = {k: int(v) for k, v in re.findall(r"(\w+)=(\d+)", buf.value.decode())}
    assert plan["last_parts"] < plan["parts"] and plan["pieces"] > 1
    h, w, targets = make(T + V, T, V, D, dtype)
    targets[0] = V - 1
    hd, wd, td = h.cuda(), w.cuda(), targets.cuda()
    loss, lse, rows = sk.entropy_fwd(hd, wd, td, reduction)
    up = torch.randn(loss.shape, generator=torch.Generator().manual_seed(3), dtype=torch.float64).to(loss.dtype)
    ws = torch.full((size + 4096,), 77, dtype=torch.uint8, device="cuda")
    gh, gw = sk.entropy_bwd(hd, wd, td, lse, rows, up.cuda(), reduction, ws=ws[:size])
    check(h, w, targets, reduction, up, loss, gh, gw)
    assert torch.all(ws[size:] == 77)
