"""Gradients in bf16 whose delta is rid of the rounding of out, by the norms of their errors (attention_delta.py has the bounds, and
test_attention_delta.py what exceeds them): with out, where the sums of dS correct it in one pass, with a bias and without, with keys that
are split over workgroups and not; without out, where it is summed from the weights."""
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


@pytest.mark.parametrize("dh", [32, 64, 72, 96, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size,buckets", [(WHOLE, 0), (SPLIT, 0), (SPLIT, 32), (dict(B=3, H=2, K=1, Sq=70, Sk=600), 0)])
def test_corrected_without_a_bias_and_over_splits(ops, dh, causal, size, buckets):
    e, got = gradients(ops, dict(size, dh=dh), causal, buckets)
    r = ad.ratios(got, *ad.bounds(e, refined=True))
    assert set(r) == ({"dq", "dk", "dbias"} if buckets else {"dq", "dk"})
    assert all(x <= 1.0 for x in r.values()), r


@pytest.mark.parametrize("Sk", [2, 7, 12])
@pytest.mark.parametrize("size", [dict(B=31, H=2, K=2, Sq=12), dict(B=16, H=16, K=16, Sq=150)])
def test_few_keys(ops, size, Sk):
    """Weights that are large, so that all that delta is off by reaches dK too."""
    e, got = gradients(ops, dict(size, Sk=Sk, dh=64), False, 0)
    r = ad.ratios(got, *ad.bounds(e, refined=True))
    assert all(x <= 1.0 for x in r.values()), r


def test_split_rows_captured_and_ragged(ops):
    """The launch that joins the splits, in a graph, with sequences that end early or hold nothing; replayed with other inputs."""
    g = torch.Generator(device="cuda").manual_seed(9)
    B, H, K, Sq, Sk, dh = 3, 4, 2, 150, 700, 64
    q, dout = (torch.randn(B, Sq, H, dh, generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn(B, Sk, K, dh, generator=g, device="cuda").bfloat16() for _ in range(2))
    q_lens = torch.tensor([150, 33, 100], dtype=torch.int32, device="cuda")
    k_lens = torch.tensor([700, 650, 0], dtype=torch.int32, device="cuda")

    def step():
        r = ops.attention(q, k, v, q_lens=q_lens, k_lens=k_lens)
        return [*r, *ops.attention_backward(q, k, v, r.out, r.lse, dout, q_lens=q_lens, k_lens=k_lens)[:3]]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for _ in range(3):
        for t in (q, k, v, dout):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(step(), outs))
        dq, dk, dv = outs[2:]
        assert (dq[1, 33:] == 0).all() and (dq[2] == 0).all() and (dk[1, 650:] == 0).all() and (dk[2] == 0).all() and (dv[2] == 0).all()
        assert dq[:2].isfinite().all() and (dq[0] != 0).any()
