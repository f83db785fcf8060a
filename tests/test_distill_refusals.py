"""The distillation loss without a GPU: every bad argument is reported by the host before a device is touched (the addresses
are made up), and an empty call is fine."""
import ctypes
import math
import os

import pytest

INVALID, OK = 1, 0
A = 0x10000  # an address that nothing reads


@pytest.fixture(scope="module")
def gp():
    from paper_1811_06965_amd import build, gp as g
    if not os.path.exists(g.LIB_PATH):
        build.build()
    g.load()
    return g


def forward(gp, **kw):
    a = dict(dtype=gp.GP_BF16, logits=A, rows=4, vocab=10, ld=10, ids=A, teacher=A, top=3, scale=1.0, clip=0.0, rest=1, loss=A,
             lse=A, rest_lse=A, ws=None, ws_bytes=0, stream=None)
    a.update(kw)
    return gp.load().gp_distill(*a.values())


def backward(gp, **kw):
    a = dict(dtype=gp.GP_F32, logits=A, rows=4, vocab=10, ld=12, ids=A, teacher=A, top=3, scale=1.0, clip=0.0, rest=1, lse=A,
             rest_lse=A, dloss=A, dlogits=A + 4096, ldd=10, stream=None)
    a.update(kw)
    return gp.load().gp_distill_backward(*a.values())


BOTH = [dict(dtype=2), dict(dtype=-1), dict(logits=None), dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=(1 << 30) + 1),
        dict(ld=9), dict(ld=1 << 41), dict(ids=None), dict(teacher=None), dict(top=0), dict(top=257), dict(top=-1), dict(scale=0.0),
        dict(scale=-1.0), dict(scale=math.nan), dict(scale=1e7), dict(clip=-1.0), dict(clip=math.nan), dict(clip=math.inf),
        dict(logits=A + 1), dict(ids=A + 2), dict(teacher=A + 2), dict(lse=None), dict(rest_lse=None), dict(lse=A + 2), dict(rest_lse=A + 2)]


@pytest.mark.parametrize("kw", BOTH + [dict(loss=None), dict(loss=A + 1), dict(ws=A + 8, ws_bytes=64)])
def test_forward_refuses(gp, kw):
    assert forward(gp, **kw) == INVALID
    assert "distill" in gp.gp_last_error()


@pytest.mark.parametrize("kw", BOTH + [
    dict(dloss=None), dict(dloss=A + 1), dict(dlogits=None), dict(dlogits=A + 4098), dict(ldd=9), dict(ldd=1 << 41),
    # an output that overlaps the logits without being them
    dict(dlogits=A), dict(dlogits=A + 4, ldd=12), dict(dlogits=A + (3 * 12 + 9) * 4), dict(dlogits=A - 3 * 10 * 4)])
def test_backward_refuses(gp, kw):
    assert backward(gp, **kw) == INVALID
    assert "distill" in gp.gp_last_error()


def test_no_rows(gp):
    none = dict(rows=0, logits=None, ids=None, teacher=None, lse=None, rest_lse=None)
    assert forward(gp, loss=None, **none) == OK
    assert backward(gp, dloss=None, dlogits=None, **none) == OK


def test_workspace(gp):
    n = ctypes.c_size_t()
    f = gp.load().gp_distill_workspace
    for args in ((2, 1, 10), (0, -1, 10), (0, 1, 0), (0, 1, (1 << 30) + 1)):
        assert f(*args, ctypes.byref(n)) == INVALID
    assert f(0, 1, 10, None) == INVALID
    assert gp.gp_distill_workspace(gp.GP_BF16, 0, 10) == 0 and gp.gp_distill_workspace(gp.GP_BF16, 1, 1 << 20) > 0


def test_header(gp):
    import re
    h = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gp.h")).read()
    assert int(re.search(r"#define GP_DISTILL_MAX (\d+)", h).group(1)) == gp.GP_DISTILL_MAX


def test_wrappers_refuse_without_a_device(gp):
    torch = pytest.importorskip("torch")
    from paper_1811_06965_amd import ops
    z, ids, t, v = torch.zeros(3, 5), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2), torch.zeros(3)
    for f in (lambda: ops.distill(z, ids, t), lambda: ops.distill(z.double(), ids, t), lambda: ops.distill(z[0], ids, t),
              lambda: ops.distill_backward(z, ids, t, v, v, rest_lse=v)):
        with pytest.raises(ValueError):
            f()
