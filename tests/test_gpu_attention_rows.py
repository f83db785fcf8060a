"""Attention on the caller's tensors and its gradients against the formulas in 64 bits (attention_reference.py says what a
result may be off by): one query to long lengths, keys fewer and more than the queries, ragged batches, empty rows, shared
heads, odd widths, packed and transposed layouts, a learned bias by buckets, masks, what is not finite behind them."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.attention_reference import attention as formulas, buckets_of, check, visible  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ops():
    from paper_1811_06965_amd import ops as o
    return o


def layout(kind, B, S, H, dh, dt, g, n=1):
    """n tensors [B, S, H, dh] of random values: apart, packed beside each other, or with the heads first."""
    shape = {"rows": (n, B, S, H, dh), "packed": (B, S, n, H, dh), "heads": (n, B, H, S, dh)}[kind]
    t = torch.randn(shape, generator=g, device="cuda").to(dt)
    if kind == "rows":
        return list(t)
    if kind == "packed":
        return [t[:, :, i] for i in range(n)]
    return [x.transpose(1, 2) for x in t]


def lens(B, n, g, zero=False):
    t = torch.randint(0, n + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    t[0] = n
    if zero and B > 1:
        t[-1] = 0
    return t


def make(dtype="bf16", B=2, H=4, K=4, Sq=33, Sk=70, dh=64, layout_q="rows", layout_kv="packed", ragged=False, starts=None,
         buckets=0, distance=0, causal=False, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[dtype]
    q, dout = layout(layout_q, B, Sq, H, dh, dt, g, 2)
    k, v = layout(layout_kv, B, Sk, K, dh, dt, g, 2)
    kw = dict(causal=causal)
    if ragged:
        kw.update(q_lens=lens(B, Sq, g), k_lens=lens(B, Sk, g, zero=True))
    if starts is not None:
        kw["q_starts"] = torch.tensor([starts + 3 * b for b in range(B)], dtype=torch.int32, device="cuda")
    table = torch.randn(H, buckets, generator=g, device="cuda") if buckets else None
    return q, k, v, dout, kw, table


def compare(ops, q, k, v, dout, kw, table=None, distance=0, both=True, scale=None):
    B, Sq, H, dh = q.shape
    ok, dist = visible(B, Sq, k.shape[1], **kw)
    bias = of = None
    if table is not None:
        bias = ops.RelativeBias(table, distance, bidirectional=not kw["causal"])
        of = buckets_of(table.shape[1], distance, not kw["causal"])
        assert bias.bucket_of.tolist() == of
    c = dh ** -0.5 if scale is None else scale
    ref = formulas(q, k, v, c, ok, table, of, dist, dout if both else None)
    r = ops.attention(q, k, v, scale=scale, bias=bias, **kw)
    check("out", r.out, ref)
    check("lse", r.lse, ref)
    if not both:
        return r, None
    grads = []
    for out in (r.out, None):
        b = ops.attention_backward(q, k, v, out, r.lse, dout, scale=scale, bias=bias, **kw)
        for name in ("dq", "dk", "dv") + (("dbias",) if table is not None else ()):
            check(name, getattr(b, name), ref)
        grads.append(b)
    return r, grads[0]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [
    dict(Sq=1, Sk=1, B=1, H=1, K=1, dh=8), dict(Sq=1, Sk=7, H=8, K=2), dict(Sq=1, Sk=200, B=4, ragged=True),
    dict(Sq=1, Sk=5000, B=3, H=6, K=2, dh=128, ragged=True), dict(Sq=1, Sk=3001, H=8, K=1, dh=40),
    dict(Sq=3, Sk=129, H=12, K=2, dh=96, ragged=True), dict(Sq=5, Sk=64, H=40, K=1, dh=72),
    dict(Sq=31, Sk=33, H=2, K=1), dict(Sq=32, Sk=4096, B=1, H=2, K=2)])
def test_few_queries(ops, dtype, kw):
    compare(ops, *make(dtype=dtype, **kw))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [8, 24, 40, 64, 72, 96, 128])
def test_widths(ops, dtype, dh):
    compare(ops, *make(dtype=dtype, Sq=77, Sk=140, H=6, K=2, B=3, dh=dh, ragged=True, seed=dh))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Sq,Sk", [(64, 31), (65, 32), (127, 64), (128, 65), (129, 128), (300, 1), (2, 700), (257, 513)])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(ops, dtype, Sq, Sk, causal):
    compare(ops, *make(dtype=dtype, Sq=Sq, Sk=Sk, ragged=True, causal=causal, seed=Sq))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout_q", ["rows", "packed", "heads"])
@pytest.mark.parametrize("layout_kv", ["rows", "heads"])
def test_layouts(ops, dtype, layout_q, layout_kv):
    compare(ops, *make(dtype=dtype, Sq=70, Sk=90, H=4, K=2, layout_q=layout_q, layout_kv=layout_kv))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_broadcast_inputs(ops, dtype):
    """One sequence's keys for all of a batch, one head's for all heads, one query row's gradient for all rows: strides of 0."""
    q, k, v, dout, kw, _ = make(dtype=dtype, B=3, Sq=40, Sk=100, H=4, K=4)
    k, v = k[:1].expand(3, -1, -1, -1), v[:, :, :1].expand(-1, -1, 4, -1)
    one = dout[:, :, :1].expand(-1, -1, 4, -1)
    compare(ops, q, k, v, one, kw)
    r = ops.attention(q, k, v)
    for a, b in zip(ops.attention_backward(q, k, v, r.out, r.lse, one),
                    ops.attention_backward(q, k.contiguous(), v.contiguous(), r.out, r.lse, one.contiguous())):
        assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("starts", [-40, 0, 25, 400, 2 ** 30, -2 ** 31 + 1])
def test_starts(ops, dtype, starts):
    """A chunk of queries at a later position; before all keys (empty rows) and far behind them."""
    if abs(starts) > 10000:
        q, k, v, dout, kw, _ = make(dtype=dtype, Sq=40, Sk=100, causal=True)
        kw["q_starts"] = torch.tensor([starts, 0], dtype=torch.int32, device="cuda")
        compare(ops, q, k, v, dout, kw)
    else:
        compare(ops, *make(dtype=dtype, Sq=40, Sk=100, causal=True, starts=starts))
        compare(ops, *make(dtype=dtype, Sq=9, Sk=50, H=8, K=2, causal=True, starts=starts))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Sq,Sk,buckets,distance,dh,K", [
    (1, 300, 32, 128, 64, 4), (50, 50, 8, 3 + 2, 64, 4), (200, 200, 32, 128, 64, 4), (331, 331, 20, 60, 24, 4), (100, 390, 64, 500, 128, 2),
    (33, 1500, 1024, 1024, 40, 1), (260, 40, 32, 17, 96, 2)])
def test_bias(ops, dtype, causal, Sq, Sk, buckets, distance, dh, K):
    if distance <= buckets // (2 if causal else 4):
        distance = buckets // 2 + 1
    args = make(dtype=dtype, Sq=Sq, Sk=Sk, dh=dh, K=K, buckets=buckets, causal=causal, ragged=Sq > 60,
                starts=5 if Sq == 100 else None, seed=Sq)
    compare(ops, *args, distance=distance)


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("bf16", 96), ("bf16", 32), ("f32", 40)])
@pytest.mark.parametrize("causal", [False, True])
def test_bias_without_splits(ops, dtype, dh, causal):
    """Enough rows that no workgroup's keys are split, over several tiles of them."""
    compare(ops, *make(dtype=dtype, B=16, H=16, K=8, Sq=150, Sk=200, dh=dh, buckets=32, causal=causal, ragged=True, seed=dh), distance=60)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_few_queries_before_keys_that_are_not_finite(ops, dtype, bad):
    q, k, v, dout, kw, _ = make(dtype=dtype, Sq=3, Sk=400, H=6, K=2, causal=True, starts=200)
    clean = compare(ops, q, k, v, dout, kw)
    k[0, 203:], v[0, 203:], k[1, 206:], v[1, 206:] = bad, bad, bad, bad
    again = compare(ops, q, k, v, dout, kw)
    for x, y in zip(clean, again):
        for s, t in zip(x, y):
            assert s is None or torch.equal(s, t)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low", [-1e30, -math.inf, torch.finfo(torch.float32).min])
def test_masking_bias(ops, dtype, low):
    """Buckets that mask: a window of keys, and a head without any key."""
    q, k, v, dout, kw, table = make(dtype=dtype, Sq=90, Sk=150, buckets=32)
    table[:, 12:16] = low
    table[:, 26:] = low
    table[1] = low
    r, b = compare(ops, q, k, v, dout, kw, table, 40)
    assert (r.out[:, :, 1] == 0).all() and (r.lse[:, 1] == -math.inf).all() and (b.dbias[1] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_masked_places_that_are_not_finite(ops, dtype, bad):
    """Rows behind the lengths, and keys and queries that a mask hides, hold what is not finite."""
    q, k, v, dout, kw, _ = make(dtype=dtype, Sq=100, Sk=120, B=2, causal=True)
    kw.update(q_lens=torch.tensor([100, 70], dtype=torch.int32, device="cuda"),
              k_lens=torch.tensor([110, 50], dtype=torch.int32, device="cuda"))
    clean = compare(ops, q, k, v, dout, kw)
    for b, (n, m) in enumerate(((100, 110), (70, 50))):
        q[b, n:], dout[b, n:], k[b, m:], v[b, m:] = bad, bad, bad, bad
    k[0, 100:], v[0, 100:] = bad, bad  # behind every query
    again = compare(ops, q, k, v, dout, kw)
    for x, y in zip(clean, again):
        for s, t in zip(x, y):
            assert s is None or torch.equal(s, t)
    # a window of 0 to 15 keys back alone, then keys that only some rows see are bad: the others stay right
    table = torch.full((4, 32), -math.inf, device="cuda")
    table[:, :8] = 0.5
    v[0, 40] = bad
    bias = ops.RelativeBias(table, 20, bidirectional=False)
    r = ops.attention(q, k, v, bias=bias, **kw)
    back = ops.attention_backward(q, k, v, r.out, r.lse, dout, bias=bias, **kw)
    seen = torch.zeros(100, dtype=torch.bool, device="cuda")
    of = buckets_of(32, 20, False)
    for i in range(100):
        d = max(-20, min(20, 40 - i))
        seen[i] = i >= 40 and of[d + 20] < 8
    assert r.out[0][~seen].isfinite().all() and not r.out[0][seen].isfinite().any()
    assert r.lse[0].isfinite().all()
    assert back.dq[0][~seen].isfinite().all()
    if bad == bad:
        assert (r.out[0][seen] == bad).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(ops, dtype):
    """Scores that differ by hundreds, in rising and falling order: the reference of a row's sums follows."""
    q, k, v, dout, kw, _ = make(dtype=dtype, Sq=40, Sk=300, B=1, H=2, K=2)
    k[:, :, 0] *= torch.linspace(0, 30, 300, device="cuda").to(k.dtype)[:, None]
    k[:, :, 1] *= torch.linspace(30, 0, 300, device="cuda").to(k.dtype)[:, None]
    compare(ops, q, k, v, dout, kw, both=False)
    compare(ops, q, k, v, dout, kw, both=False, scale=3.0)


def test_what_is_not_finite_comes_out(ops):
    q, k, v, dout, kw, _ = make(Sq=40, Sk=50, B=1, H=2, K=2)
    k[0, 7, 0] = math.nan
    r = ops.attention(q, k, v)
    assert r.out[0, :, 0].isnan().all() and r.lse[0, 0].isnan().all() and r.out[0, :, 1].isfinite().all()
    q[0, 3, 1] = math.inf
    r = ops.attention(q, k, v)
    assert r.out[0, 3, 1].isnan().all() and r.out[0, 4, 1].isfinite().all()


@pytest.mark.parametrize("Sq,Sk,B", [(0, 5, 2), (5, 0, 2), (0, 0, 2), (4, 4, 0)])
def test_nothing(ops, Sq, Sk, B):
    table = torch.randn(2, 32, device="cuda")
    bias = ops.RelativeBias(table)
    q, k = torch.randn(B, Sq, 2, 64, device="cuda"), torch.randn(B, Sk, 2, 64, device="cuda")
    r = ops.attention(q, k, k.clone(), bias=bias)
    assert (r.out == 0).all() and (r.lse == -math.inf).all()
    b = ops.attention_backward(q, k, k.clone(), r.out, r.lse, q.clone(), bias=bias)
    assert all((t == 0).all() for t in b) and b.dbias.shape == table.shape and b.dk.shape == k.shape


def test_gradients_are_differences(ops):
    """The gradient of sum dout out against differences of the forward pass in 64 bits' place: fp32, a step of 2^-6, whose
    third-order term is below 2^-12 / 6 of the third derivative (bounded by the size of the inputs here: 1e-2 in all)."""
    q, k, v, dout, kw, table = make(dtype="f32", B=1, H=2, K=1, Sq=6, Sk=9, dh=8, buckets=8, causal=False)
    bias = ops.RelativeBias(table, 6)
    r = ops.attention(q, k, v, bias=bias)
    b = ops.attention_backward(q, k, v, r.out, r.lse, dout, bias=bias)
    h = 2.0 ** -6
    g = torch.Generator(device="cuda").manual_seed(5)
    for t, d in ((q, b.dq), (k, b.dk), (v, b.dv), (table, b.dbias)):
        way = torch.randn(t.shape, generator=g, device="cuda")
        way /= way.norm()
        base = t.clone()
        ends = []
        for s in (1, -1):
            t.copy_(base + s * h * way)
            ends.append(float((ops.attention(q, k, v, bias=bias).out.double() * dout.double()).sum()))
        t.copy_(base)
        assert abs((ends[0] - ends[1]) / (2 * h) - float((d.double() * way.double()).sum())) < 1e-2


def test_gradients_into_packed_tensors(ops):
    """dq, dk and dv beside each other in one tensor, as the projection's gradient takes them."""
    q, k, v, dout, kw, _ = make(Sq=60, Sk=60, H=4, K=2, causal=True)
    r = ops.attention(q, k, v, **kw)
    b = ops.attention_backward(q, k, v, r.out, r.lse, dout, **kw)
    pack = torch.full((2, 60, 9, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    ops.attention_backward(q, k, v, r.out, r.lse, dout, grads=(pack[:, :, :4], pack[:, :, 4:6], pack[:, :, 6:8]), **kw)
    assert torch.equal(pack[:, :, :8], torch.cat((b.dq, b.dk, b.dv), 2)) and (pack[:, :, 8] == 7).all()


def test_the_same_bits_on_any_stream(ops):
    q, k, v, dout, kw, table = make(Sq=200, Sk=300, buckets=32, H=4, K=2, ragged=True)
    bias = ops.RelativeBias(table)

    def run():
        r = ops.attention(q, k, v, bias=bias, **kw)
        return [*r, *ops.attention_backward(q, k, v, r.out, r.lse, dout, bias=bias, **kw)]

    first = run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(run())
    torch.cuda.synchronize()
    for other in got:
        assert all(torch.equal(x, y) for x, y in zip(first, other))


def test_captured(ops):
    """Two graphs, one of a token's step and one of a training step, replayed in turn with other inputs."""
    q1, k1, v1, _, kw1, _ = make(Sq=1, Sk=3000, H=8, K=2, B=2, ragged=True)
    q, k, v, dout, kw, table = make(Sq=100, Sk=130, buckets=32, causal=True)
    bias = ops.RelativeBias(table, bidirectional=False)

    def token():
        return list(ops.attention(q1, k1, v1, **kw1))

    def step():
        r = ops.attention(q, k, v, bias=bias, **kw)
        return [*r, *ops.attention_backward(q, k, v, r.out, r.lse, dout, bias=bias, **kw)]

    graphs, outs = [], []
    for f in (token, step):
        f()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(f())
        graphs.append(g)
    for seed in range(3):
        for t in (q1, k1, v1, q, k, v, dout, table):
            t.copy_(torch.randn(t.shape, device="cuda"))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for f, o in zip((token, step), outs):
            assert all(torch.equal(x, y) for x, y in zip(f(), o))


def test_keys_past_four_gigabytes(ops):
    """The second sequence and the last rows of a long cache lie past 2^32 bytes."""
    H, dh, Sk = 2, 64, 100
    big = torch.empty(2, 3 << 30, dtype=torch.bfloat16, device="cuda")
    at = 2200 << 20
    k, v = (torch.as_strided(big, (2, Sk, H, dh), (3 << 30, 1 << 20, dh, 1), at + off) for off in (0, H * dh))
    g = torch.Generator(device="cuda").manual_seed(1)
    for t in (k, v):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    q = torch.randn(2, 3, H, dh, generator=g, device="cuda").bfloat16()
    r = ops.attention(q, k, v)
    s = ops.attention(q, k.contiguous(), v.contiguous())
    assert torch.equal(r.out, s.out) and torch.equal(r.lse, s.lse)


def test_refusals(ops):
    q, k, v, dout, kw, table = make(Sq=8, Sk=9)
    r = ops.attention(q, k, v)
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    bias = ops.RelativeBias(torch.zeros(4, 32, device="cuda"))
    bad = [lambda: ops.attention(q[0], k, v), lambda: ops.attention(q.half(), k, v), lambda: ops.attention(q, k.float(), v),
           lambda: ops.attention(q, k[:1], v[:1]), lambda: ops.attention(q, k, v[:, :8]), lambda: ops.attention(q, k.cpu(), v),
           lambda: ops.attention(q, k, v, k_lens=n.long()), lambda: ops.attention(q, k, v, k_lens=n[:1]),
           lambda: ops.attention(q, k, v, k_lens=n.cpu()), lambda: ops.attention(q.transpose(2, 3), k, v),
           lambda: ops.attention(q[:, :, :2], k[:, :, :2], v[:, :, :2], bias=bias),
           lambda: ops.attention(q.requires_grad_(), k, v), lambda: ops.RelativeBias(torch.zeros(32, device="cuda")),
           lambda: ops.RelativeBias(torch.zeros(4, 32)),
           lambda: ops.attention_backward(q.detach(), k, v, r.out, r.lse[:, :1], dout),
           lambda: ops.attention_backward(q.detach(), k, v, r.out.float(), r.lse, dout),
           lambda: ops.attention_backward(q.detach(), k, v, r.out, r.lse, dout[:1])]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    q = q.detach()
    from paper_1811_06965_amd import gp
    narrow = torch.zeros(1, 4, 2, 68, device="cuda", dtype=torch.bfloat16)
    for f in (lambda: ops.attention(q[:, :, :3], k, v), lambda: ops.attention(narrow, narrow, narrow),
              lambda: ops.attention(q, k, v, scale=0.0), lambda: ops.RelativeBias(torch.zeros(4, 31, device="cuda")),
              lambda: ops.attention(*[torch.zeros(1, 2, 1, 136, device="cuda", dtype=torch.bfloat16)] * 3),
              lambda: ops.attention(q[..., 4:60], k[..., 4:60], v[..., 4:60]),
              lambda: ops.attention_backward(q, k, v, r.out, r.lse, dout, grads=(q, torch.empty_like(k), torch.empty_like(v))),
              lambda: ops.attention_backward(q, k, v, r.out, r.lse, dout, grads=(torch.empty_like(q), v, torch.empty_like(v)))):
        with pytest.raises(gp.GpError):
            f()
