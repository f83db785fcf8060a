"""Gradients in bf16 whose delta is rid of the rounding of out, by the norms of their errors (attention_delta.py has the bounds, and
test_attention_delta.py what exceeds them): with a bias, where the sums of dS correct it in one pass (no workgroup's keys are
split), or it is summed from the weights (split keys, and calls without out); without a bias and without out."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import attention_delta as ad  # noqa: E402
from tests.attention_reference import buckets_of, visible  # noqa: E402


@pytest.fixture(scope="module")
def ops():
    from paper_1811_06965_amd import ops as o
    return o


def gradients(ops, size, causal, buckets, distance=60, with_out=True):
    q, k, v, dout, table = ad.inputs(**size, buckets=buckets, device="cuda", seed=size["dh"])
    ok, dist = visible(size["B"], size["Sq"], size["Sk"], causal=causal)
    of = buckets_of(buckets, distance, not causal) if buckets else None
    e = ad.exact(q, k, v, dout, size["dh"] ** -0.5, ok, table, of, dist)
    kw = dict(causal=causal, bias=ops.RelativeBias(table, distance, bidirectional=not causal) if buckets else None)
    r = ops.attention(q, k, v, **kw)
    b = ops.attention_backward(q, k, v, r.out if with_out else None, r.lse, dout, **kw)
    return e, {"dq": b.dq, "dk": b.dk, "dbias": b.dbias}


WHOLE = dict(B=16, H=16, K=8, Sq=150, Sk=200)  # 512 blocks of 128 rows: none is split
SPLIT = dict(B=2, H=4, K=2, Sq=300, Sk=520)    # 24 blocks


@pytest.mark.parametrize("dh", [32, 64, 72, 96, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_corrected_by_the_sums_of_ds(ops, dh, causal):
    e, got = gradients(ops, dict(WHOLE, dh=dh), causal, 32)
    r = ad.ratios(got, *ad.bounds(e, refined=True))
    assert all(x <= 1.0 for x in r.values()), r


@pytest.mark.parametrize("dh", [32, 64, 72, 96, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size,with_out,buckets", [(SPLIT, True, 32), (SPLIT, False, 32), (WHOLE, False, 32), (SPLIT, False, 0), (WHOLE, False, 0)])
def test_from_the_weights(ops, dh, causal, size, with_out, buckets):
    e, got = gradients(ops, dict(size, dh=dh), causal, buckets, with_out=with_out)
    r = ad.ratios(got, *ad.bounds(e, refined=False))
    assert set(r) == ({"dq", "dk", "dbias"} if buckets else {"dq", "dk"})
    assert all(x <= 1.0 for x in r.values()), r
