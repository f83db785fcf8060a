"""The divergence from a teacher's most likely tokens and its gradient against the formulas in 64 bits: widths around the
kernels' steps, row strides, starts off every alignment, split rows, both types, rows that name few tokens or none, tokens
named twice, masks, shares of 0, what is not finite.

Bounds, per value, from the roundings made (u = 2^-24; S the largest finite |s| of a row, n the terms that a thread adds):
* a term of the sums: E = (3 S + 8) u of itself; the sums R = E + 2 (n + 64) u, n = max(V / 256, min(V, 8192) / 64);
  an lse: L = R + 2 u (|lse| + 1); log p: L + 2 u |s|;
* q = exp(t - shift): Q = u (3 |t| + 3 |shift| + 4) of itself; a term q (log q - log p): q (Q |log q - log p| + u 3 |log q| + log p's) and
  the sum of `top` of them top u of their absolute sum; the share that is left is formed in 64 bits and rounded once; its
  term: left (2 u |log left| + both L's) and 4 u of itself;
* gradient: W p: p (2 u (|s| + |lse|) + L + 8 u); q: Q q; of a token that is not named (W R - left) exp(s - rest): the first
  factor R (2 u (|rest| + |lse|) + both L's + 4 u) + 2 u left, the second like p; then half a step of the type.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def ops():
    from paper_1811_06965_amd import ops as o
    return o


def make(rows, vocab, top, dtype, pad=0, offset=0, seed=0, ragged=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((offset + rows * (vocab + pad) + 8,), 7.0, device="cuda").to(DT[dtype])
    z = buf[offset:offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    z.copy_(torch.randn(rows, vocab, generator=g, device="cuda") * 3.0)
    ids = torch.rand(rows, vocab, generator=g, device="cuda").topk(top, 1).indices
    z.scatter_add_(1, ids[:, :top // 2 + 1], torch.full((rows, top // 2 + 1), 6.0, device="cuda").to(z.dtype))
    t = torch.log_softmax(torch.randn(rows, top, generator=g, device="cuda") * 2.5, 1)
    t = t + torch.log(0.6 + 0.39 * torch.rand(rows, 1, generator=g, device="cuda"))
    if ragged and rows > 2:
        left = torch.randint(1, top + 1, (rows, 1), generator=g, device="cuda")
        left[rows // 2] = 0
        left[0] = top
        gone = torch.arange(top, device="cuda") >= left
        ids = torch.where(gone, -1, ids)
        t = torch.where(gone, math.nan, t)
    return buf, z, ids.to(torch.int32), t.float().contiguous()


def formulas(z, ids, t, scale, clip, rest, dloss):
    """Results in float64 and bounds."""
    V, top = z.shape[1], ids.shape[1]
    x = z.double()
    if clip > 0:
        x = x.clamp(-clip, clip)
    x = torch.where(x <= -1e30, -math.inf, x)
    s = x * scale
    named = ids >= 0
    at = ids.clamp(min=0).long()
    some = named.any(1)
    t = torch.where(named, t.double(), -math.inf)
    shift = torch.zeros(len(z), dtype=torch.float64, device=z.device) if rest else torch.logsumexp(t, 1)
    shift = torch.where(shift == -math.inf, 0.0, shift)
    logq = t - shift[:, None]
    q = torch.exp(logq)
    left = (1 - q.sum(1)).clamp(min=0) * some if rest else torch.zeros_like(shift)
    inside = torch.zeros(z.shape, dtype=torch.float64, device=z.device).scatter_add_(1, at, named.double()) > 0
    target = torch.zeros(z.shape, dtype=torch.float64, device=z.device).scatter_add_(1, at, torch.where(named, q, 0.0))
    lse = torch.logsumexp(s, 1)
    far = torch.logsumexp(torch.where(inside, -math.inf, s), 1)
    logp = torch.where(lse[:, None] > -math.inf, s.gather(1, at) - lse[:, None], -math.inf)
    terms = torch.where(named & (q > 0), q * (logq - logp), 0.0)
    active = (left > 0) & (far > -math.inf)
    extra = torch.where(active, left * (torch.log(left.clamp(min=1e-300)) - torch.where(active, far - lse, 0.0)), 0.0)
    loss = terms.sum(1) + extra
    S = torch.where(s.isfinite(), s.abs(), 0.0).amax(1)
    n = max(V / 256, min(V, 8192) / 64)
    R = (3 * S + 8) * U + 2 * (n + 64) * U

    def fin(v):
        return torch.where(v.isfinite(), v.abs(), 0.0)
    L, F = R + 2 * U * (fin(lse) + 1), R + 2 * U * (fin(far) + 1)
    Q = U * (3 * fin(t) + 3 * shift.abs()[:, None] + 4)
    gap = fin(logq - logp)
    loss_off = torch.where(named, q * (Q * gap + 3 * U * fin(logq) + L[:, None] + 2 * U * fin(s.gather(1, at))), 0.0).sum(1)
    loss_off += top * U * fin(terms).sum(1) + torch.where(active, left * (2 * U * torch.log(left.clamp(min=1e-300)).abs() + L + F), 0.0) + 4 * U * fin(extra)
    r = dict(loss=loss, lse=lse, rest_lse=far)
    r.update({"~loss": loss_off, "~lse": L, "~rest_lse": F})
    # gradient
    W = torch.where(some, q.sum(1) + torch.where(active, left, 0.0), 0.0)[:, None]
    ok = lse > -math.inf
    p = torch.where(ok[:, None], torch.exp(s - lse[:, None]), 0.0)
    k = (dloss.double() * scale)[:, None]
    share = torch.where(active, left / torch.exp(torch.where(active, far - lse, 0.0)), 0.0)[:, None]
    d = torch.where(inside, W * p - target, (W - share) * p)
    qoff = torch.zeros_like(target).scatter_add_(1, at, torch.where(named, (Q + U) * q, 0.0))
    poff = 2 * U * (fin(s) + fin(lse)[:, None]) + L[:, None] + 8 * U
    Rr = torch.where(active, torch.exp(torch.where(active, far - lse, 0.0)), 1.0)[:, None]
    fo = 2 * U * (fin(far) + fin(lse))[:, None] + (L + F)[:, None] + 4 * U
    away = torch.where(active[:, None], p / Rr * (Rr * fo + 2 * U * left[:, None]) + ((W - share) * p).abs() * (2 * U * (fin(s) + fin(far)[:, None]) + F[:, None] + 8 * U),
                       W * p * poff)
    lim = torch.where(inside, W * p * poff + qoff, away) + 2 * U * d.abs()
    live = (some & ok)[:, None]
    if clip > 0:
        live = live & (z.double().abs() <= clip)
    d = torch.where(live, d * k, 0.0)
    r["grad"] = d
    r["~grad"] = torch.where(live, lim * k.abs(), 0.0) + HALF[z.dtype] * d.abs() + 2.0 ** -120
    return r


def check(name, got, ref):
    a, b, lim = got.double(), ref[name], ref["~" + name]
    bad = ~((a == b) | (a.isnan() & b.isnan())) & ~((a - b).abs() <= lim)
    assert not bad.any(), (name, int(bad.sum()), float((a - b)[bad].abs().max()), float(((a - b).abs() / lim)[bad].max()))


def compare(ops, z, ids, t, scale=1.0, clip=0.0, rest=True, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dloss = torch.rand(len(z), generator=g, device="cuda") - 0.3
    ref = formulas(z, ids, t, scale, clip, rest, dloss)
    r = ops.distill(z, ids, t, scale=scale, clip=clip, rest=rest)
    for name in ("loss", "lse") + (("rest_lse",) if rest else ()):
        check(name, getattr(r, name), ref)
    assert rest or r.rest_lse is None
    d = ops.distill_backward(z, ids, t, r.lse, dloss, rest_lse=r.rest_lse, scale=scale, clip=clip, rest=rest)
    check("grad", d, ref)
    return r, d, dloss


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (3, 2, 2), (5, 7, 3), (4, 8, 8), (3, 9, 1), (7, 257, 100), (2, 256, 256), (4, 2047, 20),
                                            (6, 2049, 64), (9, 4111, 65), (3, 20001, 128), (200, 32000, 32)])
def test_widths(ops, dtype, rest, rows, vocab, top):
    compare(ops, *make(rows, vocab, top, dtype, seed=vocab)[1:], rest=rest)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab", [(2, 140001), (1, 300000), (100, 140001)])
def test_long_rows(ops, dtype, rest, rows, vocab):
    """Rows split over workgroups, and windows of a row that one workgroup takes."""
    compare(ops, *make(rows, vocab, 40, dtype)[1:], rest=rest)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 3, 8])
@pytest.mark.parametrize("pad", [0, 1, 5])
def test_strides(ops, dtype, offset, pad):
    buf, z, ids, t = make(5, 1003, 9, dtype, pad=pad, offset=offset)
    before = buf.clone()
    r, d, dloss = compare(ops, z, ids, t)
    assert torch.equal(buf, before)
    ops.distill_backward(z, ids, t, r.lse, dloss, rest_lse=r.rest_lse, out=z)  # in place
    assert torch.equal(z, d)
    z.copy_(before[offset:offset + 5 * (1003 + pad)].view(5, -1)[:, :1003])
    assert torch.equal(buf, before)  # nothing beside the rows was written


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("scale,clip", [(0.25, 0.0), (2.0, 0.0), (1.0, 4.0), (0.5, 2.5)])
def test_scale_and_clip(ops, dtype, rest, scale, clip):
    compare(ops, *make(40, 5001, 33, dtype)[1:], scale=scale, clip=clip, rest=rest)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
def test_tokens_named_twice(ops, dtype, rest):
    _, z, ids, t = make(6, 900, 20, dtype, ragged=False)
    ids[:, 10:] = ids[:, :10]
    ids[1, :] = ids[1, 0]
    compare(ops, z, ids, t, rest=rest)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low", [-math.inf, -1e30, None])
def test_masks(ops, dtype, low):
    _, z, ids, t = make(8, 3000, 16, dtype, ragged=False)
    low = torch.finfo(z.dtype).min if low is None else low
    g = torch.Generator(device="cuda").manual_seed(1)
    hide = torch.rand(z.shape, generator=g, device="cuda") < 0.3
    hide.scatter_(1, ids.long(), False)
    hide[3] = True                                   # nothing but the named tokens
    hide[3].scatter_(0, ids[3].long(), False)
    hide[4] = True                                   # nothing at all
    z[hide] = low
    for rest in (False, True):
        r, d, dloss = compare(ops, z, ids, t, rest=rest)
        assert r.lse[4] == -math.inf and r.loss[4] == math.inf and (d[4] == 0).all()
        assert not rest or (r.rest_lse[3] == -math.inf and r.loss[3].isfinite())
        assert (d[hide] == 0).all()
    z[5, ids[5, 2].long()] = low  # a token that the teacher gives weight cannot occur
    t[6, 3] = -math.inf           # a weight of 0 for a token that cannot
    z[6, ids[6, 3].long()] = low
    for rest in (False, True):
        r = ops.distill(z, ids, t, rest=rest)
        assert r.loss[5] == math.inf and r.loss[6].isfinite()


def test_what_is_not_finite(ops):
    _, z, ids, t = make(8, 3000, 16, "f32", ragged=False)
    z[0, 77], z[1, 99] = math.nan, math.inf
    z[2, ids[2, 0].long()] = math.nan
    t[3, 4] = math.nan
    ids[4, 5], ids[5, 6] = 3000, -2
    r = ops.distill(z, ids, t)
    d = ops.distill_backward(z, ids, t, r.lse, torch.ones(8, device="cuda"), rest_lse=r.rest_lse)
    assert r.loss[:6].isnan().all() and r.loss[6:].isfinite().all()
    for row in (0, 2, 4, 5):
        assert d[row].isnan().all(), row
    assert d[6:].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_little_left(ops, dtype):
    """A student that gives the rest almost nothing, and a teacher that does: R far below an ulp of the whole sum."""
    _, z, ids, t = make(5, 2000, 8, dtype, ragged=False)
    z.scatter_add_(1, ids.long(), torch.full((5, 8), 60.0, device="cuda").to(z.dtype))
    compare(ops, z, ids, t)
    t += math.log(1.0000001)
    z.scatter_(1, ids.long(), 200.0)  # and nothing that fp32 can hold
    r = ops.distill(z, ids, t)
    d = ops.distill_backward(z, ids, t, r.lse, torch.ones(5, device="cuda"), rest_lse=r.rest_lse)
    assert r.loss.isfinite().all() and d.isfinite().all()


def test_gradients_are_differences(ops):
    """fp32, a step of 2^-6 along a unit vector: the third-order term is below 2^-12 / 6 of the third derivative, whose size is
    that of a cumulant of values within 1 of each other (at most 1), and sums of losses below 2^5 are off by 2^-17, over 2^-5: 1e-3 in all."""
    _, z, ids, t = make(4, 50, 6, "f32", ragged=False)
    g = torch.Generator(device="cuda").manual_seed(2)
    way = torch.randn(z.shape, generator=g, device="cuda")
    way /= way.norm()
    h = 2.0 ** -6
    for rest in (False, True):
        r = ops.distill(z, ids, t, rest=rest)
        d = ops.distill_backward(z, ids, t, r.lse, torch.ones(4, device="cuda"), rest_lse=r.rest_lse, rest=rest)
        ends = [float(ops.distill((z + sign * h * way).contiguous(), ids, t, rest=rest).loss.double().sum()) for sign in (1, -1)]
        assert abs((ends[0] - ends[1]) / (2 * h) - float((d.double() * way.double()).sum())) < 1e-3


def test_nothing(ops):
    z = torch.zeros(0, 50, device="cuda")
    ids, t = torch.zeros(0, 3, dtype=torch.int32, device="cuda"), torch.zeros(0, 3, device="cuda")
    r = ops.distill(z, ids, t)
    assert r.loss.numel() == 0
    assert ops.distill_backward(z, ids, t, r.lse, r.loss, rest_lse=r.rest_lse).shape == z.shape


def test_from_a_teachers_logits(ops):
    """As it is used: the teacher's alternatives, the student's loss, its gradient into the logits' own memory; captured,
    and replayed with other logits.  A student that is its teacher has a loss of 0 up to the bounds."""
    g = torch.Generator(device="cuda").manual_seed(4)
    teacher = torch.randn(64, 8000, generator=g, device="cuda").bfloat16() * 3
    student = torch.randn(64, 8000, generator=g, device="cuda").bfloat16() * 3
    weight = torch.full((64,), 1 / 64, device="cuda")

    def step(z):
        a = ops.token_logprobs(teacher, top=24)
        r = ops.distill(z, a.top_ids, a.top_logp)
        return [r.loss, r.lse, r.rest_lse, ops.distill_backward(z, a.top_ids, a.top_logp, r.lse, weight, rest_lse=r.rest_lse)]

    a = ops.token_logprobs(teacher, top=24)
    compare(ops, student, a.top_ids, a.top_logp)
    same, _, _ = compare(ops, teacher, a.top_ids, a.top_logp)
    ref = formulas(teacher, a.top_ids, a.top_logp, 1.0, 0.0, True, weight)
    assert (same.loss.double().abs() <= 2 * ref["~loss"] + 1e-5).all()
    step(student)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(student)
    for _ in range(3):
        student.copy_(torch.randn(student.shape, generator=g, device="cuda") * 3)
        teacher.copy_(torch.randn(student.shape, generator=g, device="cuda") * 3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(step(student), out))


def test_more_rows_than_a_launch_holds(ops):
    rows = (1 << 21) + 5
    g = torch.Generator(device="cuda").manual_seed(6)
    z = torch.randn(rows, 3, generator=g, device="cuda")
    ids = torch.randint(0, 3, (rows, 1), generator=g, device="cuda", dtype=torch.int32)
    t = -torch.rand(rows, 1, generator=g, device="cuda")
    compare(ops, z, ids, t)


def test_refusals(ops):
    from paper_1811_06965_amd import gp
    _, z, ids, t = make(4, 50, 6, "f32", ragged=False)
    v = torch.zeros(4, device="cuda")
    bad = [lambda: ops.distill(z, ids.long(), t), lambda: ops.distill(z, ids, t.double()), lambda: ops.distill(z, ids[:3], t[:3]),
           lambda: ops.distill(z, ids, t[:, :5]), lambda: ops.distill(z, ids.cpu(), t), lambda: ops.distill(z, ids, t.cpu()),
           lambda: ops.distill(z.half(), ids, t), lambda: ops.distill(z.t(), ids, t), lambda: ops.distill(z, ids[:, ::2], t[:, ::2]),
           lambda: ops.distill(z.clone().requires_grad_(), ids, t), lambda: ops.distill(z, ids, t.clone().requires_grad_()),
           lambda: ops.distill_backward(z, ids, t, v[:3], v, rest_lse=v), lambda: ops.distill_backward(z, ids, t, v, v.double(), rest_lse=v),
           lambda: ops.distill_backward(z, ids, t, v, v, rest_lse=v, out=z[:3])]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ops.distill_backward(z, ids, t, v, v), lambda: ops.distill(z, ids, t, scale=0.0), lambda: ops.distill(z, ids, t, clip=-1.0),
              lambda: ops.distill(z, ids[:, :0].contiguous(), t[:, :0].contiguous()),
              lambda: ops.distill(z, torch.zeros(4, 257, dtype=torch.int32, device="cuda"), torch.zeros(4, 257, device="cuda"))):
        with pytest.raises(gp.GpError):
            f()
