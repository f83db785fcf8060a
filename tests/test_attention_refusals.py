"""Attention on the caller's tensors without a GPU: every bad argument is reported by the host before a device is touched
(the addresses are made up), sizes of zero are fine, and the map of distances to buckets is the formula's."""
import ctypes
import math
import os

import pytest

OK, INVALID, UNSUPPORTED = 0, 1, 6
A = 1 << 20  # an address that nothing reads


@pytest.fixture(scope="module")
def gp():
    from paper_1811_06965_amd import build, gp as g
    if not os.path.exists(g.LIB_PATH):
        build.build()
    g.load()
    return g


def config(gp, **kw):
    c = dict(dtype=gp.GP_BF16, batch=2, heads=4, kv_heads=2, q_len=8, k_len=16, head_dim=64, causal=0, scale=0.125,
             q_lens=None, k_lens=None, q_starts=None, bias=None, bucket_of=None, buckets=0, max_distance=0)
    c.update(kw)
    return gp.gp_attention_config(*c.values())


def tensors(gp, c, backward):
    """Made-up addresses of tensors far apart, with the strides of contiguous ones."""
    names = ["q", "k", "v", "out"] + (["dout", "dq", "dk", "dv"] if backward else [])
    t = {}
    for i, n in enumerate(names):
        key = n in ("k", "v", "dk", "dv")
        heads, length = (c.kv_heads, c.k_len) if key else (c.heads, c.q_len)
        t[n] = dict(data=A * (i + 1), seq=length * heads * c.head_dim, row=heads * c.head_dim, head=c.head_dim)
    return t


def call(gp, cfg=None, backward=False, change=None, **kw):
    c = cfg if cfg is not None else config(gp)
    t = tensors(gp, c, backward)
    for name, d in (change or {}).items():
        t[name].update(d)
    rows = {n: ctypes.byref(gp.gp_head_rows(d["data"], d["seq"], d["row"], d["head"])) for n, d in t.items()}
    rows.update({n: None for n in kw.pop("null", ())})
    a = dict(lse=A, dbias=None, ws=A * 64, ws_bytes=1 << 40)
    a.update(kw)
    lib = gp.load()
    if backward:
        return lib.gp_attention_backward(ctypes.byref(c), rows["q"], rows["k"], rows["v"], rows["out"], a["lse"], rows["dout"],
                                         rows["dq"], rows["dk"], rows["dv"], a["dbias"], a["ws"], a["ws_bytes"], None)
    return lib.gp_attention(ctypes.byref(c), rows["q"], rows["k"], rows["v"], rows["out"], a["lse"], a["ws"], a["ws_bytes"], None)


BIAS = dict(bias=A, bucket_of=A, buckets=32, max_distance=128)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), INVALID), (dict(batch=-1), INVALID), (dict(q_len=-1), INVALID), (dict(k_len=-1), INVALID),
    (dict(k_len=(1 << 28) + 1), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(kv_heads=3), INVALID),
    (dict(heads=65536, kv_heads=65536), INVALID), (dict(batch=1 << 22), INVALID), (dict(batch=1 << 21), INVALID), (dict(q_len=1 << 28), INVALID),
    (dict(head_dim=0), INVALID), (dict(head_dim=60), INVALID), (dict(head_dim=136), UNSUPPORTED), (dict(scale=0.0), INVALID),
    (dict(scale=-1.0), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(q_lens=A + 1), INVALID),
    (dict(k_lens=A + 2), INVALID), (dict(q_starts=A + 2), INVALID), (dict(buckets=4), INVALID), (dict(max_distance=4), INVALID),
    (dict(BIAS, bucket_of=None), INVALID), (dict(BIAS, buckets=0), INVALID), (dict(BIAS, max_distance=0), INVALID),
    (dict(BIAS, bias=A + 2), INVALID), (dict(BIAS, buckets=1025), UNSUPPORTED), (dict(BIAS, max_distance=1025), UNSUPPORTED)])
def test_configurations(gp, backward, kw, status):
    assert call(gp, config(gp, **kw), backward) == status
    assert "attention" in gp.gp_last_error()
    n = ctypes.c_size_t()
    assert gp.load().gp_attention_workspace(ctypes.byref(config(gp, **kw)), backward, ctypes.byref(n)) == status


@pytest.mark.parametrize("name", ["q", "k", "v", "out", "dout", "dq", "dk", "dv"])
@pytest.mark.parametrize("d", [dict(data=None), dict(data=A + 8), dict(seq=-64), dict(row=-64), dict(head=-64), dict(row=63),
                               dict(row=32), dict(row=1 << 24), dict(head=65), dict(seq=1025), dict(seq=1 << 50)])
def test_tensors(gp, name, d):
    backward = name.startswith("d")
    assert call(gp, backward=backward, change={name: d}) == INVALID
    assert "attention" in gp.gp_last_error()


def test_strides_past_any_address(gp):
    assert call(gp, config(gp, heads=512, kv_heads=2), change={"q": dict(head=1 << 40)}) == INVALID
    assert call(gp, config(gp, batch=1 << 20, heads=2), change={"k": dict(seq=1 << 30)}) == INVALID


def test_other_arguments(gp):
    assert call(gp, null=["q"]) == INVALID and call(gp, null=["out"]) == INVALID
    assert call(gp, lse=A + 2) == INVALID and call(gp, ws=A + 8) == INVALID
    assert call(gp, backward=True, lse=None) == INVALID
    assert call(gp, backward=True, dbias=A) == INVALID  # without a bias
    assert call(gp, config(gp, **BIAS), True, dbias=A + 2) == INVALID
    assert call(gp, backward=True, ws=None) == INVALID and call(gp, backward=True, ws_bytes=8) == INVALID
    split = config(gp, q_len=1, k_len=100000)
    assert gp.gp_attention_workspace(split, 0) > 0
    assert call(gp, split, ws=None) == INVALID and call(gp, split, ws_bytes=16) == INVALID
    lib = gp.load()
    assert lib.gp_attention(None, None, None, None, None, None, None, 0, None) == INVALID
    assert lib.gp_attention_workspace(ctypes.byref(config(gp)), 0, None) == INVALID


def test_overlaps(gp):
    q = dict(data=A, seq=8 * 256, row=256, head=64)
    assert call(gp, change=dict(out=q)) == INVALID
    assert call(gp, change=dict(out=dict(data=A + 8 * 256 * 2))) == INVALID  # the second sequence
    # out in the gaps that the rows of q leave is not an overlap; one head's gap too few is
    wide = dict(seq=8 * 512, row=512)
    assert call(gp, change=dict(q=wide, out=dict(data=A + 192 * 2, **wide))) == INVALID
    # an output whose own rows overlap
    assert call(gp, change=dict(out=dict(head=0))) == INVALID
    assert call(gp, change=dict(out=dict(seq=0))) == INVALID
    assert call(gp, change=dict(out=dict(head=32))) == INVALID
    for x, y in (("dq", "q"), ("dk", "v"), ("dv", "k"), ("dq", "dout"), ("dq", "out")):
        assert call(gp, backward=True, change={x: dict(data=tensors(gp, config(gp), True)[y]["data"])}) == INVALID
    assert call(gp, backward=True, change=dict(dv=dict(data=7 * A))) == INVALID  # dk's
    assert call(gp, backward=True, change=dict(dk=dict(head=0))) == INVALID


def test_nothing_to_do(gp):
    """No launch: no device is there."""
    assert call(gp, config(gp, batch=0)) == OK
    assert call(gp, config(gp, q_len=0), null=["q", "out"]) == OK
    assert call(gp, config(gp, batch=0), backward=True, ws=None, ws_bytes=0) == OK
    for kw in (dict(batch=0), dict(q_len=0), dict(k_len=0), dict(q_len=0, k_len=0), dict(q_len=0, k_len=0, **BIAS)):
        for backward in (0, 1):
            assert gp.gp_attention_workspace(config(gp, **kw), backward) >= 0


def test_struct_fields_match_the_header(gp):
    import re
    h = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gp.h")).read()
    for name in ("gp_head_rows", "gp_attention_config"):
        end = h.index("} %s;" % name)
        body = re.sub(r"/\*.*?\*/", "", h[h.rindex("typedef struct {", 0, end):end], flags=re.S)
        fields = [f.strip(" *") for decl in re.findall(r"(?:void\*|const int\*|const float\*|long|float|int) ([^;]+);", body)
                  for f in decl.split(",")]
        assert fields == [f for f, _ in getattr(gp, name)._fields_], name
    for name in ("GP_BUCKETS_MAX", "GP_DISTANCE_MAX"):
        assert int(re.search(r"#define %s (\d+)" % name, h).group(1)) == getattr(gp, name)


@pytest.mark.parametrize("buckets,distance,both", [
    (32, 128, 1), (32, 128, 0), (4, 2, 1), (2, 2, 0), (3, 3, 0), (20, 60, 0), (64, 500, 1), (1024, 1024, 1), (1024, 1000, 0), (6, 1024, 1),
    (128, 33, 1)])
def test_buckets(gp, buckets, distance, both):
    from tests.attention_reference import buckets_of
    if buckets > 500:  # whole numbers of thousands of digits: the borders alone, in 50 digits
        from decimal import Decimal, getcontext
        getcontext().prec = 50
        n = buckets // 2 if both else buckets
        half = n // 2

        def side(d):
            if d < half:
                return d
            x = (Decimal(d) / half).ln() / (Decimal(distance) / half).ln() * (n - half)
            return min(n - 1, half + int(x + Decimal("1e-40")))
        want = [side(abs(d)) + (n if d > 0 and both else 0) if d <= 0 or both else 0 for d in range(-distance, distance + 1)]
    else:
        want = buckets_of(buckets, distance, both)
    assert gp.gp_relative_buckets(buckets, distance, both) == want


@pytest.mark.parametrize("args", [(1, 8, 0), (0, 8, 0), (-4, 8, 0), (3, 8, 1), (2, 8, 1), (33, 128, 1), (32, 8, 1), (32, 16, 0), (32, 1025, 1),
                                  (1025, 1024, 0), (32, -1, 1), (32, 0, 1)])
def test_buckets_refused(gp, args):
    with pytest.raises(gp.GpError):
        gp.gp_relative_buckets(*args)
    assert gp.load().gp_relative_buckets(32, 128, 1, None) == INVALID


def test_wrappers_refuse_without_a_device(gp):
    torch = pytest.importorskip("torch")
    from paper_1811_06965_amd import ops
    q = torch.zeros(1, 2, 4, 64)
    for f in (lambda: ops.attention(q, q, q), lambda: ops.attention(q[0], q, q), lambda: ops.attention(q.double(), q, q),
              lambda: ops.RelativeBias(torch.zeros(4, 32)), lambda: ops.RelativeBias(torch.zeros(4)),
              lambda: ops.attention_backward(q, q, q, q, torch.zeros(1, 4, 2), q)):
        with pytest.raises(ValueError):
            f()
