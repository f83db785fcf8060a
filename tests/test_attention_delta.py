"""The bounds of attention_delta.py see what they are for, on the CPU: gradients imitated in bf16 are within them, and leave them
when delta keeps the rounding of out, is corrected the wrong way, by 1% too little, or is left out."""
import pytest

torch = pytest.importorskip("torch")

from tests import attention_delta as ad  # noqa: E402
from tests.attention_reference import buckets_of, visible  # noqa: E402

SIZES = [dict(B=2, H=4, K=2, Sq=150, Sk=200, dh=64), dict(B=3, H=2, K=2, Sq=90, Sk=70, dh=96)]


def case(size, causal, buckets=32, distance=60):
    q, k, v, dout, table = ad.inputs(**size, buckets=buckets, device="cpu", seed=3)
    ok, dist = visible(size["B"], size["Sq"], size["Sk"], causal=causal, device="cpu")
    of = buckets_of(buckets, distance, not causal) if buckets else None
    return ad.exact(q, k, v, dout, size["dh"] ** -0.5, ok, table, of, dist)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("refined", [False, True])
@pytest.mark.parametrize("buckets", [0, 32])
def test_right_gradients(size, causal, refined, buckets):
    e = case(size, causal, buckets)
    ref, lim = ad.bounds(e, refined)
    for delta_of in (lambda d0, s: d0 + s, lambda d0, s: e["delta"]):
        r = ad.ratios(ad.imitation(e, delta_of, refined), ref, lim)
        assert set(r) == ({"dq", "dk", "dbias"} if buckets else {"dq", "dk"})
        assert all(x <= 1.0 for x in r.values()), r


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("name,wrong", [("out's rounding", lambda d0, s: d0), ("the wrong sign", lambda d0, s: d0 - s),
                                        ("1% off", lambda d0, s: 1.01 * (d0 + s)), ("left out", lambda d0, s: 0.0 * s)])
def test_wrong_deltas(size, causal, name, wrong):
    e = case(size, causal)
    for refined in (False, True):
        ref, lim = ad.bounds(e, refined)
        r = ad.ratios(ad.imitation(e, wrong, refined), ref, lim)
        assert r["dbias"] > 10 and r["dk"] > 1.2, (name, r)
        assert refined or r["dq"] > 1.2, (name, r)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("causal", [False, True])
def test_a_mean_key_that_stays(size, causal):
    """dq whose dS' are summed without taking the mean key off, and with it taken off twice."""
    e = case(size, causal)
    ref, lim = ad.bounds(e, True)
    d0 = (e["g"] * e["out"].bfloat16().double()).sum(3, keepdim=True)
    first = (e["p"] * (e["dp"] - d0)).bfloat16().double()
    for times in (0.0, 2.0, -1.0):
        dq = ad.mm(first, e["k"]) - times * first.sum(3, keepdim=True) * ad.mm(e["p"], e["k"])
        r = ad.ratios(ad.gradients(e, e["ds"], dq), ref, lim)
        assert r["dq"] > 1.2, (times, r)
