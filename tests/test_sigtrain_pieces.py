"""Plans of the cross entropy's backward call: no workgroup of a divided product may be left without a step, in the last piece of the classes either."""
import ctypes as C
import random
import re

import pytest

from paper_2509_10613_amd import binding as sk


@pytest.fixture(scope="module")
def describe():
    import os
    if not os.path.exists(sk.LIB_PATH):
        from paper_2509_10613_amd import build
        build.build()
    lib, buf = sk.load(), C.create_string_buffer(512)

    def plan(T, V, D, dt, ws):
        assert lib.sigtrain_describe(3, T, V, D, dt, ws, buf, len(buf)) == 0
        return {k: int(v) for k, v in re.findall(r"(\w+)=(\d+)", buf.value.decode())}

    return plan


def check(p, V):
    if "parts" not in p:   # (few classes of wide rows: no such product)
        return False
    assert 1 <= p["parts"] <= p["grad_h_steps"] and 1 <= p["last_parts"] <= p["last_steps"] and p["last_parts"] <= p["parts"]
    return p["last_parts"] < p["parts"]


# default workspaces (0), and some that hold smaller pieces: the last piece has one to seven steps where the others are divided among more
@pytest.mark.parametrize("T,V,D,dt,ws", [(8689, 537712, 11, 1, 0), (2995, 4358224, 7, 0, 0), (2, 278537, 8154, 1, 0), (978, 39956, 529, 2, 20513728),
                                         (94, 260, 16, 1, 622262), (36, 5178, 856, 2, 3453237), (36, 5178, 856, 3, 3453237), (75, 1035, 5, 0, 515440)])
def test_a_last_piece_of_few_steps(describe, T, V, D, dt, ws):
    assert check(describe(T, V, D, dt, ws), V)


def test_every_part_of_every_piece_has_a_step(describe):
    rng, q, fewer = random.Random(7), sk.load().sigtrain_entropy_workspace_bytes, 0
    for _ in range(20000):
        T, V, D, dt = int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 19)), int(2 ** rng.uniform(0, 13)), rng.randrange(4)
        least, best = q(1, T, V, D, dt, 1), q(1, T, V, D, dt, 0)
        fewer += check(describe(T, V, D, dt, rng.choice([0, least, int(least + (best - least) * rng.random())])), V)
    assert fewer > 0
