"""Attention with a bias before infinities and NaN that a mask hides: by position or by the bias's buckets, in keys, values, queries
and their gradients, in both types, with keys that are split over workgroups and not.  The results and all the gradients are the
formulas' and, to the bit, those of finite values in the same places."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_attention_rows import compare, make, ops  # noqa: E402, F401 (ops: the fixture)
from tests.attention_reference import buckets_of  # noqa: E402

BAD = [math.inf, -math.inf, math.nan]
SPLIT, WHOLE = dict(B=2, H=4, K=2), dict(B=16, H=16, K=16)


def unchanged(clean, again):
    for x, y in zip(clean, again):
        for s, t in zip(x, y):
            assert s is None or torch.equal(s, t)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("size,dh", [(SPLIT, 64), (SPLIT, 128), (WHOLE, 64), (WHOLE, 96), (WHOLE, 24)])
def test_behind_the_position(ops, dtype, bad, size, dh):  # noqa: F811
    """Queries from 20 before the keys on: the first see none, the last keys are seen by none."""
    q, k, v, dout, kw, table = make(dtype=dtype, Sq=150, Sk=280, dh=dh, buckets=32, causal=True, **size)
    starts = torch.full((size["B"],), 100, dtype=torch.int32, device="cuda")
    starts[1] = -20
    kw["q_starts"] = starts
    clean = compare(ops, q, k, v, dout, kw, table, 60)
    for b, keys in ((0, 250), (1, 130)):
        k[b, keys:], v[b, keys:] = bad, bad
    q[1, :20], dout[1, :20] = bad, bad
    r = ops.attention(q, k, v, bias=ops.RelativeBias(table, 60, bidirectional=False), **kw)
    assert (r.out[1, :20] == 0).all() and (r.lse[1, :, :20] == -math.inf).all()
    q0, g0 = q.clone(), dout.clone()
    q0[1, :20], g0[1, :20] = 0, 0  # the formulas' rows; what the call is given is `q` and `dout`
    again = compare(ops, q0, k, v, g0, kw, table, 60)
    unchanged(clean[:1], again[:1])
    bias = ops.RelativeBias(table, 60, bidirectional=False)
    for out in (r.out, None):
        one = ops.attention_backward(q, k, v, out, r.lse, dout, bias=bias, **kw)
        two = ops.attention_backward(q0, k, v, out, r.lse, g0, bias=bias, **kw)
        unchanged([two], [one])
        assert (one.dq[1, :20] == 0).all() and (one.dk[1, 130:] == 0).all() and (one.dv[1, 130:] == 0).all()
    unchanged(clean[1:], again[1:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("size,dh", [(SPLIT, 64), (SPLIT, 96), (WHOLE, 64), (WHOLE, 128), (WHOLE, 24)])
@pytest.mark.parametrize("Sq", [3, 70])
def test_outside_the_buckets_window(ops, dtype, bad, size, dh, Sq):  # noqa: F811
    """Buckets that mask keys 26 and more away on either side: keys before and behind all the queries' windows."""
    q, k, v, dout, kw, table = make(dtype=dtype, Sq=Sq, Sk=300, dh=dh, buckets=32, starts=120, **size)
    of = buckets_of(32, 40, True)
    hidden = [b for b in set(of) if all(abs(d - 40) >= 26 for d in range(81) if of[d] == b)]
    table[:, hidden] = -math.inf
    near = max(abs(d - 40) for d in range(81) if of[d] not in hidden)
    assert 8 <= near < 40 and hidden
    clean = compare(ops, q, k, v, dout, kw, table, 40)
    for b, start in enumerate(kw["q_starts"].tolist()):
        first, last = start - near, min(300, start + Sq + near)
        assert 0 < first and last < 300
        for t in (k, v):
            t[b, :first], t[b, last:] = bad, bad
    # the formulas drop keys that no pair of the lengths sees: these are masked by the bias alone, so they are given as 0
    k0, v0 = (torch.where(t.isfinite(), t, torch.zeros_like(t)) for t in (k, v))
    again = compare(ops, q, k0, v0, dout, kw, table, 40)
    unchanged(clean, again)
    bias = ops.RelativeBias(table, 40)
    r = ops.attention(q, k, v, bias=bias, **kw)
    unchanged([clean[0]], [r])
    unchanged([clean[1]], [ops.attention_backward(q, k, v, r.out, r.lse, dout, bias=bias, **kw)])
    unchanged([ops.attention_backward(q, k0, v0, None, r.lse, dout, bias=bias, **kw)],
              [ops.attention_backward(q, k, v, None, r.lse, dout, bias=bias, **kw)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [SPLIT, WHOLE])
@pytest.mark.parametrize("bad", BAD)
def test_a_value_that_some_rows_see(ops, dtype, size, bad):  # noqa: F811
    """One value that is not finite, in a window of keys: what depends on it is not finite, and all else is as it was."""
    q, k, v, dout, kw, table = make(dtype=dtype, Sq=260, Sk=260, buckets=32, causal=True, **size)
    of = buckets_of(32, 40, False)
    hidden = [b for b in set(of) if all(d - 40 <= -20 or d > 40 for d in range(81) if of[d] == b)]
    table[:, hidden] = -math.inf
    bias = ops.RelativeBias(table, 40, bidirectional=False)
    r = ops.attention(q, k, v, bias=bias, **kw)
    clean = ops.attention_backward(q, k, v, r.out, r.lse, dout, bias=bias, **kw)
    i = torch.arange(260, device="cuda")
    dist = (i[None] - i[:, None]).clamp(-40, 40) + 40
    sees = (i[None] <= i[:, None]) & ~torch.isin(torch.tensor(of, device="cuda")[dist], torch.tensor(hidden, device="cuda"))
    v[0, 60, 0] = bad  # of the first key head
    rows = sees[:, 60]
    keys = sees[rows].any(0)
    group = size["H"] // size["K"]
    r2 = ops.attention(q, k, v, bias=bias, **kw)
    assert torch.equal(r.lse, r2.lse)
    b = ops.attention_backward(q, k, v, r2.out, r2.lse, dout, bias=bias, **kw)
    assert rows.sum() > 5 and not keys.all()
    assert not b.dq[0, rows, :group].isfinite().any() and not b.dk[0, 60, 0].isfinite().any()
    assert torch.equal(b.dq[0, ~rows], clean.dq[0, ~rows]) and torch.equal(b.dq[0, :, group:], clean.dq[0, :, group:])
    assert torch.equal(b.dk[0, ~keys], clean.dk[0, ~keys]) and torch.equal(b.dk[0, :, 1:], clean.dk[0, :, 1:])
    assert torch.equal(b.dv, clean.dv)  # the weights and dout alone
    assert torch.equal(b.dq[1:], clean.dq[1:]) and torch.equal(b.dk[1:], clean.dk[1:])
    assert torch.equal(b.dbias[group:], clean.dbias[group:])
    seen = [x for x in set(of) if x not in hidden]
    assert not b.dbias[:group, seen].isfinite().any() and (b.dbias[:group, hidden] == 0).all()
