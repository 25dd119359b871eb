"""The entry points of include/sigtrain.h without a GPU: exports, argument checks, workspace queries, and the wrappers' refusals."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2509_10613_amd import autograd as ska
from paper_2509_10613_amd import binding as sk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ONE, OTHER, BIG = C.c_void_p(256), C.c_void_p(1 << 20), 1 << 40
NULL, SHAPE, DTYPE, WORKSPACE = -1, -2, -4, -5


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sk.LIB_PATH):
        from paper_2509_10613_amd import build
        build.build()
    return sk.load()


def test_exports_every_declared_symbol(lib):
    header = open(os.path.join(ROOT, "include", "sigtrain.h")).read()
    assert set(re.findall(r"\b(sigtrain_[a-z0-9_]+)\s*\(", header)) == set(sk.TRAIN_EXPORTS)
    for name in sk.TRAIN_EXPORTS:
        assert getattr(lib, name) is not None


def test_the_types_are_those_of_the_header():
    header = open(os.path.join(ROOT, "include", "sigtrain.h")).read()
    assert "ST_F32 = SK_F32, ST_F64 = SK_F64, ST_BF16 = 2, ST_F16 = 3" in header
    assert (sk.ST_F32, sk.ST_F64, sk.ST_BF16, sk.ST_F16) == (sk.SK_F32, sk.SK_F64, 2, 3)


def test_embed_arguments(lib):
    f, b = lib.sigtrain_embed_fwd, lib.sigtrain_embed_bwd
    assert f(ONE, ONE, OTHER, 4, 8, 3, 1.0, 1, 4, None) == DTYPE
    assert f(ONE, ONE, OTHER, 4, 8, 3, 1.0, 2, 0, None) == DTYPE
    for count, V, D in ((-1, 8, 3), (4, -1, 3), (4, 8, 0), (4, 8, (1 << 24) + 1), (4, (1 << 31) - 1, 3), ((1 << 40) + 1, 8, 3)):
        assert f(ONE, ONE, OTHER, count, V, D, 1.0, 1, 0, None) == SHAPE
        assert b(ONE, ONE, OTHER, count, V, D, 1.0, 1, 0, ONE, BIG, None) == SHAPE
        assert lib.sigtrain_embed_bwd_workspace_bytes(count, V, D, 0) == 0
    for scale in (float("nan"), float("inf")):
        assert f(ONE, ONE, OTHER, 4, 8, 3, scale, 1, 0, None) == SHAPE
    assert b(ONE, ONE, OTHER, (1 << 31) - 1, 8, 3, 1.0, 1, 0, ONE, BIG, None) == SHAPE   # (the sort's places are 32-bit numbers)
    assert f(None, ONE, OTHER, 4, 8, 3, 1.0, 1, 0, None) == NULL
    assert f(ONE, None, OTHER, 4, 8, 3, 1.0, 1, 0, None) == NULL
    assert f(ONE, C.c_void_p(257), OTHER, 4, 8, 3, 1.0, 1, 2, None) == NULL
    assert b(ONE, None, OTHER, 4, 8, 3, 1.0, 1, 0, ONE, BIG, None) == NULL
    need = lib.sigtrain_embed_bwd_workspace_bytes(4, 8, 3, 0)
    assert need > 0 and need % 256 == 0
    assert b(ONE, ONE, OTHER, 4, 8, 3, 1.0, 1, 0, ONE, need - 1, None) == WORKSPACE
    assert b(ONE, ONE, OTHER, 4, 8, 3, 1.0, 1, 0, C.c_void_p(128), need, None) == WORKSPACE
    assert b(ONE, ONE, OTHER, 4, 8, 3, 1.0, 1, 0, None, need, None) == WORKSPACE
    # no token, and no row: nothing to do
    assert f(None, None, None, 0, 8, 3, 1.0, 1, 0, None) == 0
    assert b(None, None, None, 4, 0, 3, 1.0, 1, 0, None, 0, None) == 0


def test_entropy_arguments(lib):
    f, b, q = lib.sigtrain_entropy_fwd, lib.sigtrain_entropy_bwd, lib.sigtrain_entropy_workspace_bytes
    fwd = lambda T=4, V=8, D=3, red=1, it=1, dt=0, ws=ONE, n=BIG, h=ONE, w=ONE, t=ONE, loss=ONE, lse=ONE, rows=ONE: f(  # noqa: E731
        h, w, t, loss, lse, rows, T, V, D, red, it, dt, ws, n, None)
    bwd = lambda T=4, V=8, D=3, red=1, it=1, dt=0, ws=ONE, n=BIG, h=ONE, g=ONE, gh=ONE, gw=ONE: b(  # noqa: E731
        h, ONE, ONE, ONE, ONE, g, gh, gw, T, V, D, red, it, dt, ws, n, None)
    for call in (fwd, bwd):
        assert call(dt=4) == DTYPE and call(dt=-1) == DTYPE and call(it=2) == DTYPE
        assert call(red=3) == SHAPE and call(T=-1) == SHAPE and call(V=0) == SHAPE and call(D=0) == SHAPE
        assert call(T=4000001) == SHAPE and call(D=4000001) == SHAPE and call(V=(1 << 31) - 1) == SHAPE
        assert call(h=None) == NULL and call(h=C.c_void_p(258)) == NULL
        assert call(ws=None) == WORKSPACE and call(ws=C.c_void_p(64)) == WORKSPACE and call(n=255) == WORKSPACE
    assert b"needed" in lib.sigkernel_last_error()
    for name in ("w", "t", "loss", "lse", "rows"):
        assert fwd(**{name: None}) == NULL
    assert bwd(g=None) == NULL
    assert bwd(gh=None, gw=None) == 0
    for back in (0, 1):
        for T, V, D, dt in ((1, 1, 1, 0), (8192, 131072, 4096, 2), (128, 1000, 5461, 1), (0, 5, 5, 3)):
            least, best = q(back, T, V, D, dt, 1), q(back, T, V, D, dt, 0)
            assert 0 < least <= best and least % 256 == 0
            call = fwd if back == 0 else bwd
            if T:
                assert call(T=T, V=V, D=D, dt=dt, n=least - 1) == WORKSPACE
    assert q(0, 4, 0, 3, 0, 0) == 0 and q(1, 4, 8, 3, 9, 0) == 0
    # the logits of all classes never exist at once: far less than them even at its fastest
    assert q(1, 8192, 262144, 1024, 2, 0) < 8192 * 262144 * 2


def test_a_piece_fits_every_workspace_from_the_least_on(lib):
    buf = C.create_string_buffer(256)
    for op, T, V, D, dt in ((2, 700, 50257, 100, 0), (3, 700, 50257, 128, 2), (3, 33, 9000, 5461, 1)):
        least, best = (lib.sigtrain_entropy_workspace_bytes(op - 2, T, V, D, dt, n) for n in (1, 0))
        for i in range(9):
            have = least + (best - least) * i // 8
            assert lib.sigtrain_describe(op, T, V, D, dt, have, buf, len(buf)) == 0
            piece, pieces, ws = (int(re.search(r" %s=(\d+)" % k, buf.value.decode()).group(1)) for k in ("piece", "pieces", "ws"))
            assert ws <= have and piece * pieces >= V and piece * (pieces - 1) < V


def test_the_least_workspace_is_never_more_than_the_best(lib):
    import random
    rng = random.Random(5)
    q = lib.sigtrain_entropy_workspace_bytes
    for _ in range(400):
        T, V, D = (int(2 ** rng.uniform(0, 14)) for _ in range(3))
        for back in (0, 1):
            for dt in range(4):
                assert 0 < q(back, T, V, D, dt, 1) <= q(back, T, V, D, dt, 0), (back, T, V, D, dt)
    assert q(1, 2000, 300, 5461, 1, 1) <= q(1, 2000, 300, 5461, 1, 0)


def test_describe(lib):
    buf = C.create_string_buffer(256)
    for op in range(4):
        assert lib.sigtrain_describe(op, 10, 20, 30, 0, 0, buf, len(buf)) == 0 and buf.value
    assert lib.sigtrain_describe(4, 10, 20, 30, 0, 0, buf, len(buf)) == SHAPE
    assert lib.sigtrain_describe(0, 10, 20, 30, 0, 0, None, 0) == NULL
    assert lib.sigtrain_describe(1, 10, 20, 0, 0, 0, buf, len(buf)) == SHAPE


def arrays(*ranges):
    n = len(ranges)
    return (C.c_void_p * n)(*[r[0] for r in ranges]), (C.c_int64 * n)(*[r[1] for r in ranges]), (C.c_int * n)(*[r[2] for r in ranges])


def test_clip_arguments(lib):
    f, g = lib.sigtrain_clip, lib.sigtrain_grad_norm
    need = lib.sigtrain_clip_workspace_bytes(2)
    assert need > 0 and lib.sigtrain_clip_workspace_bytes(-1) == 0
    at, counts, dts = arrays((4096, 8, 0), (8192, 8, 2))
    ok = dict(n=2, bound=1.0, norm=ONE, ws=ONE, size=need)

    def clip(at=at, to=at, counts=counts, dts=dts, out_dts=dts, **kw):
        a = dict(ok, **kw)
        return f(at, to, counts, dts, out_dts, a["n"], a["bound"], a["norm"], a["ws"], a["size"], None)

    assert clip(n=-1) == SHAPE and clip(bound=-1.0) == SHAPE and clip(bound=float("nan")) == SHAPE
    assert clip(at=None) == NULL and clip(to=None) == NULL and clip(counts=None) == NULL and clip(norm=None) == NULL and clip(out_dts=None) == NULL
    assert clip(ws=None) == WORKSPACE and clip(size=need - 1) == WORKSPACE and clip(ws=C.c_void_p(8)) == WORKSPACE
    assert clip(dts=(C.c_int * 2)(0, 7)) == DTYPE and clip(out_dts=(C.c_int * 2)(0, 7)) == DTYPE
    assert clip(out_dts=(C.c_int * 2)(0, 3)) == DTYPE                    # in place with another type
    assert clip(counts=(C.c_int64 * 2)(8, -1)) == SHAPE
    assert clip(at=(C.c_void_p * 2)(4096, None)) == NULL and clip(at=(C.c_void_p * 2)(4098, 8192)) == NULL
    # outputs that overlap: one array twice in place, an output on another input, two outputs, an output beside its input
    twice = arrays((4096, 8, 0), (4096, 8, 0))
    assert clip(at=twice[0], to=twice[0], dts=twice[2], out_dts=twice[2]) == SHAPE
    for to in ((8192, 65536), (65536, 65540), (4100, 65536), (65536, 8190), (8192, 4096)):
        assert clip(to=(C.c_void_p * 2)(*to), out_dts=(C.c_int * 2)(0, 2)) == SHAPE, to
    assert b"overlaps" in lib.sigkernel_last_error()
    assert g(at, counts, dts, -1, ONE, ONE, need, None) == SHAPE
    assert g(at, counts, dts, 2, None, ONE, need, None) == NULL
    assert g(at, counts, dts, 2, ONE, ONE, need - 1, None) == WORKSPACE
    assert g(at, counts, (C.c_int * 2)(0, -1), 2, ONE, ONE, need, None) == DTYPE


def test_wrappers_refuse_host_tensors_and_wrong_types():
    tokens, table = torch.zeros(3, dtype=torch.long), torch.zeros(4, 2)
    with pytest.raises(ValueError, match="device tensor"):
        ska.embed(tokens, table)
    with pytest.raises(ValueError, match="device tensor"):
        sk.embed_bwd(tokens, torch.zeros(3, 2), 4)
    with pytest.raises(ValueError, match="device tensor"):
        ska.linear_cross_entropy(torch.zeros(3, 2), table, tokens)
    with pytest.raises(ValueError, match="expected, got"):
        ska.linear_cross_entropy(torch.zeros(3, 2), table, tokens[:2])
    with pytest.raises(ValueError, match="device tensors"):
        ska.clip_grad_norm([table], 1.0)
    with pytest.raises(ValueError, match="device tensors"):
        ska.grad_norm(table)
    with pytest.raises(TypeError, match="float64, float32, bfloat16 or float16"):
        sk._st_dt(torch.zeros(1, dtype=torch.int32))
    with pytest.raises(TypeError, match="int32 or int64"):
        sk._st_it(torch.zeros(1))
