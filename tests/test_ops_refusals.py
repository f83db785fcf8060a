"""Refusals of the operators on the caller's own tensors: every bad argument is
reported by the host before a device is touched (no GPU here, and the addresses
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


def lp(gp, **kw):
    a = dict(dtype=gp.GP_BF16, logits=A, rows=4, vocab=10, ld=10, tokens=A, scale=1.0, clip=0.0, logp=A, lse=A,
             entropy=A, top=2, top_ids=A, top_logp=A, ws=None, ws_bytes=0, stream=None)
    a.update(kw)
    return gp.load().gp_token_logprobs(*a.values())


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(dtype=-1), dict(logits=None), dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(ld=9),
    dict(tokens=None), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(clip=-1.0),
    dict(clip=math.nan), dict(clip=math.inf), dict(top=-1), dict(top=33, vocab=40, ld=40), dict(top=11),
    dict(top_ids=None), dict(top_logp=None), dict(logits=A + 1), dict(logits=A + 2, dtype=0), dict(tokens=A + 2),
    dict(logp=A + 1), dict(lse=A + 2), dict(entropy=A + 3), dict(top_ids=A + 2), dict(top_logp=A + 2),
    dict(ws=A + 8, ws_bytes=64)])
def test_token_logprobs_refuses(gp, kw):
    assert lp(gp, **kw) == INVALID
    assert "token_logprobs" in gp.gp_last_error()


def test_token_logprobs_of_no_rows(gp):
    assert lp(gp, rows=0) == OK
    assert lp(gp, rows=0, logits=None, tokens=None, logp=None, top_ids=None, top_logp=None) == OK


def test_token_logprobs_workspace(gp):
    n = ctypes.c_size_t()
    f = gp.load().gp_token_logprobs_workspace
    for args in ((2, 1, 10, 0), (0, -1, 10, 0), (0, 1, 0, 0), (0, 1, 10, -1), (0, 1, 10, 33)):
        assert f(*args, ctypes.byref(n)) == INVALID
    assert f(0, 1, 10, 0, None) == INVALID
    assert gp.gp_token_logprobs_workspace(gp.GP_BF16, 0, 10, 1) >= 0


def back(gp, **kw):
    a = dict(dtype=gp.GP_F32, logits=A, rows=4, vocab=10, ld=12, tokens=A, scale=1.0, clip=0.0, lse=A, entropy=A,
             dlogp=A, dentropy=A, dlogits=A + 4096, ldd=10, stream=None)
    a.update(kw)
    return gp.load().gp_token_logprobs_backward(*a.values())


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(logits=None), dict(rows=-1), dict(vocab=0), dict(ld=9), dict(ldd=9), dict(scale=0.0),
    dict(clip=-0.5), dict(lse=None), dict(dlogits=None), dict(tokens=None), dict(entropy=None),
    dict(dlogp=None, dentropy=None), dict(lse=A + 2), dict(entropy=A + 1), dict(dlogp=A + 2), dict(dentropy=A + 2),
    dict(tokens=A + 1), dict(dlogits=A + 4098),
    # an output that overlaps the logits without being them: another stride, another start, the last element
    dict(dlogits=A), dict(dlogits=A + 4, ldd=12), dict(dlogits=A + (3 * 12 + 9) * 4), dict(dlogits=A - 3 * 10 * 4)])
def test_token_logprobs_backward_refuses(gp, kw):
    assert back(gp, **kw) == INVALID
    assert "token_logprobs" in gp.gp_last_error()


def test_token_logprobs_backward_of_no_rows(gp):
    assert back(gp, rows=0, logits=None, lse=None, tokens=None, entropy=None, dlogits=None) == OK


def norm(gp, tensors=((A, 10),), **kw):
    arr = (gp.gp_grad_tensor * max(1, len(tensors)))(*[gp.gp_grad_tensor(*t) for t in tensors])
    a = dict(dtype=gp.GP_F32, grads=arr, n=len(tensors), max_norm=1.0, out=A, ws=A, ws_bytes=1 << 20, stream=None)
    a.update(kw)
    return gp.load().gp_grad_norm(*a.values())


@pytest.mark.parametrize("kw", [
    dict(dtype=5), dict(n=-1), dict(grads=None), dict(out=None), dict(out=A + 2), dict(ws=None), dict(ws=A + 4),
    dict(ws_bytes=2048 * 8), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=math.nan),
    dict(tensors=((None, 3),)), dict(tensors=((A + 2, 3),)), dict(tensors=((A, 3), (A, -1))),
    dict(tensors=((A, 1 << 41),))])
def test_grad_norm_refuses(gp, kw):
    assert norm(gp, **kw) == INVALID
    assert "grad_norm" in gp.gp_last_error()


def test_grad_norm_workspace(gp):
    assert gp.gp_grad_norm_workspace(3) >= 2048 * 8
    with pytest.raises(gp.GpError):
        gp.gp_grad_norm_workspace(-1)


def adamw(gp, tensor=None, cfg=None, **kw):
    t = dict(param=A, grad=A, m=A, v=A, m_scale=None, v_scale=None, copy=None, count=10, weight_decay=0.1)
    t.update(tensor or {})
    c = dict(param_dtype=gp.GP_F32, grad_dtype=gp.GP_F32, state_bits=32, seed=0, lr=1e-3, beta1=0.9, beta2=0.999,
             eps=1e-8)
    c.update(cfg or {})
    arr, conf = (gp.gp_adamw_tensor * 1)(gp.gp_adamw_tensor(*t.values())), gp.gp_adamw_config(*c.values())
    a = dict(tensors=arr, n=1, cfg=ctypes.byref(conf), step=1, step_dev=None, factor=None, stream=None)
    a.update(kw)
    return gp.load().gp_adamw_step(*a.values())


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(tensors=None), dict(cfg={"param_dtype": 2}), dict(cfg={"grad_dtype": 2}),
    dict(cfg={"state_bits": 16}), dict(cfg={"lr": -1.0}), dict(cfg={"lr": math.nan}), dict(cfg={"lr": math.inf}),
    dict(cfg={"beta1": 1.0}), dict(cfg={"beta1": -0.1}), dict(cfg={"beta2": 1.0}), dict(cfg={"beta2": math.nan}),
    dict(cfg={"eps": 0.0}), dict(cfg={"eps": 1e-60}), dict(cfg={"eps": math.inf}), dict(step=0), dict(step=-1),
    dict(step=1, step_dev=A), dict(step=0, step_dev=A + 4), dict(factor=A + 1), dict(tensor={"param": None}),
    dict(tensor={"grad": None}), dict(tensor={"m": None}), dict(tensor={"v": None}), dict(tensor={"count": -1}),
    dict(tensor={"count": 1 << 41}), dict(tensor={"weight_decay": -0.1}), dict(tensor={"weight_decay": 1001.0}),
    dict(tensor={"weight_decay": math.nan}), dict(tensor={"m_scale": A}), dict(tensor={"v_scale": A}),
    dict(cfg={"state_bits": 8}), dict(cfg={"state_bits": 8}, tensor={"m_scale": A}),
    dict(cfg={"param_dtype": 1}, tensor={"copy": A}), dict(tensor={"param": A + 2}), dict(tensor={"grad": A + 2}),
    dict(tensor={"m": A + 2}), dict(tensor={"v": A + 1}), dict(tensor={"copy": A + 1}),
    dict(cfg={"state_bits": 8}, tensor={"m_scale": A, "v_scale": A + 2})])
def test_adamw_refuses(gp, kw):
    assert adamw(gp, **kw) == INVALID
    assert "adamw" in gp.gp_last_error()


def test_wrappers_refuse_without_a_device(gp):
    torch = pytest.importorskip("torch")
    from paper_1811_06965_amd import ops
    z, tok = torch.zeros(3, 5), torch.zeros(3, dtype=torch.int32)
    bad = [lambda: ops.token_logprobs(z, tok), lambda: ops.token_logprobs(z.double(), tok),
           lambda: ops.token_logprobs(z.t(), tok), lambda: ops.token_logprobs(z[0], tok),
           lambda: ops.token_logprobs(z, tok.long()), lambda: ops.token_logprobs(z, tok[:2]),
           lambda: ops.token_logprobs(z[:1].expand(3, 5), tok),
           lambda: ops.token_logprobs_backward(z, tok, torch.zeros(3), dlogp=torch.zeros(3)),
           lambda: ops.token_logprobs_backward(z, tok, torch.zeros(2), dlogp=torch.zeros(3)),
           lambda: ops.grad_norm([z]), lambda: ops.grad_norm([]), lambda: ops.AdamW([z], [z]),
           lambda: ops.AdamW([], [])]
    for f in bad:
        with pytest.raises(ValueError):
            f()


def test_struct_fields_match_the_header(gp):
    import re
    h = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gp.h")).read()
    for name in ("gp_grad_tensor", "gp_adamw_tensor", "gp_adamw_config"):
        end = h.index("} %s;" % name)
        body = re.sub(r"/\*.*?\*/", "", h[h.rindex("typedef struct {", 0, end):end], flags=re.S)
        fields = [f.strip(" *") for decl in re.findall(r"(?:void\*|float\*|long long|double|int|unsigned) ([^;]+);", body)
                  for f in decl.split(",")]
        assert fields == [f for f, _ in getattr(gp, name)._fields_], name
    for name in ("GP_TOP_MAX", "GP_STATE_BLOCK"):
        assert int(re.search(r"#define %s (\d+)" % name, h).group(1)) == getattr(gp, name)
