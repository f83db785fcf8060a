"""Token log probabilities and their gradient against a plain implementation in
64 bits: widths around the kernels' steps, row strides, starts off every
alignment, both types, masks (also of the type's lowest value, and rows without
any allowed token), NaN and infinities, padding, ties among the alternatives.

Tolerances, per value, from the roundings made (u = 2^-24, half a step of fp32):
* s = scale x is rounded once: |s| u; a difference of two such values, its
  multiplication by log2 e and the exponential add |d| u + |s| u + 4 u relative
  to a term of the sums, at most E = (3 max|s| + 8) u, where only finite s count;
* a thread adds at most ceil(V / 256) + 8 of them (its own, at 256 threads a
  row or more, with two roundings a term for the rescaling) and up to 16 joins
  follow: the sums are off by R = E + 2 (V / 256 + 32) u relative;
* lse = m + log(sum): R + |lse| 2 u + |log(sum)| 2 u; logp adds |s| 2 u;
* the entropy log(a) - b / a: the terms of b are e |d|, so b / a is off by
  R (2 H + |d| at the mean) <= R (2 H + 2 log V + 4).
The gradient g = scale (a ([v = t] - p) - b p (d + H)), d = s - lse:
* p is off by p (|s| + |lse|) 2 u + 4 p u; d by (|s| + |lse|) 2 u;
* a handful of products and sums: 8 u of the absolute terms; then one rounding
  to the type, half a step: 2^-8 (bf16) or 2^-24 of the value.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ops():
    from paper_1811_06965_amd import ops as o
    return o


def make(rows, vocab, pad, dtype, seed, offset=0, masked=0.0, low=False):
    """Logits [rows, vocab] at an element offset into a buffer, rows vocab + pad apart, and tokens."""
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((offset + rows * (vocab + pad) + 8,), 7.0).to(DT[dtype])
    z = torch.randn(rows, vocab, generator=g) * 3.0
    z[torch.rand(z.shape, generator=g) < 0.002] += 9.0
    z = z.to(DT[dtype])
    if masked:
        z[torch.rand(z.shape, generator=g) < masked] = torch.finfo(z.dtype).min if low else -math.inf
    buf = buf.cuda()
    view = buf[offset:offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    view.copy_(z)
    tok = torch.randint(0, vocab, (rows,), generator=g).to(torch.int32).cuda()
    return buf, view, tok


def reference(z, scale, clip):
    """x, s, lse, p, log p (0 where p is), entropy in float64; a logit of -1e30 or less cannot occur."""
    x = z.double().cpu().numpy()
    if clip > 0:
        x = np.clip(x, -clip, clip)
    s = np.where(x <= -1e30, -np.inf, x * scale)
    with np.errstate(all="ignore"):
        m = s.max(1, keepdims=True)
        empty = m[:, 0] == -np.inf
        mm = np.where(empty[:, None], 0.0, m)
        e = np.exp(s - mm)
        a = e.sum(1, keepdims=True)
        lse = np.where(empty, -np.inf, (mm + np.log(a))[:, 0])
        p = np.where(empty[:, None], 0.0, e / a)
        d = np.where(s == -np.inf, 0.0, s - np.where(empty, 0.0, lse)[:, None])
        h = -(p * d).sum(1)
    return x, s, lse, p, d, h


def same_special(got, want):
    """NaN and infinities in the same places; returns the finite mask."""
    assert np.array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    assert np.array_equal(np.isinf(got) & ~np.isnan(got), inf) and np.array_equal(got[inf], want[inf])
    return np.isfinite(want)


def largest(s):
    """The largest |s| of a row among the terms that count (the others are below e^-200)."""
    with np.errstate(all="ignore"):
        near = np.isfinite(s) & (s > np.where(np.isfinite(s), s, -np.inf).max(1, keepdims=True) - 200)
    return np.where(near, np.abs(s), 0.0).max(1)


def check_forward(ops, z, tok, scale=1.0, clip=0.0, top=0):
    r = ops.token_logprobs(z, tok, scale=scale, clip=clip, top=top)
    V = z.shape[1]
    x, s, lse, p, d, h = reference(z, scale, clip)
    big, n = largest(s), lambda t: t.double().cpu().numpy()
    R = (3 * big + 8) * U + 2 * (V / 256 + 32) * U
    fine = same_special(n(r.lse), lse)
    L = np.where(fine, np.abs(lse), 0.0)
    tol = R + 2 * L * U + 2 * (math.log(V) + 1) * U + big * U
    assert (np.abs(n(r.lse) - lse)[fine] <= tol[fine]).all()
    fine = same_special(n(r.entropy), h)
    tol_h = R * (2 * np.abs(h) + 2 * math.log(V) + 4) + 4 * (math.log(V) + 1) * U
    assert (np.abs(n(r.entropy) - h)[fine] <= tol_h[fine]).all()
    t = tok.cpu().numpy()
    with np.errstate(all="ignore"):
        want = np.where(lse == -np.inf, -np.inf, s[np.arange(len(t)), np.clip(t, 0, V - 1)] - lse)
        big = np.maximum(big, np.where(np.isfinite(want), np.abs(want) + L, 0.0))  # the token asked for may be far off
    want = np.where(t == -1, 0.0, np.where((t < -1) | (t >= V), np.nan, want))
    fine = same_special(n(r.logp), want)
    assert (np.abs(n(r.logp) - want)[fine] <= (tol + 2 * big * U + np.abs(want) * U)[fine]).all()
    if not top:
        assert r.top_ids is None and r.top_logp is None
        return r
    key = np.where(np.isnan(x), np.inf, x)  # a NaN before everything: first by being NaN, then by value, then index
    for i in range(len(t)):
        order = np.lexsort((np.arange(V), -key[i], ~np.isnan(x[i])))[:top]
        assert r.top_ids[i].cpu().tolist() == order.tolist(), i
        with np.errstate(all="ignore"):
            want = s[i][order] - lse[i] if lse[i] != -np.inf else np.full(top, -np.inf)
        got = n(r.top_logp[i])
        fine = same_special(got, want)
        assert (np.abs(got - want)[fine] <= (tol[i] + 2 * (big[i] + np.abs(want)) * U)[fine]).all()
    return r


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,offset,scale,clip,top", [
    (1, 1, 0, 0, 1.0, 0.0, 1), (3, 2, 0, 0, 1.0, 0.0, 2), (2, 7, 1, 1, 0.5, 0.0, 7), (5, 63, 0, 3, 1.0, 2.0, 5),
    (1, 64, 0, 0, 2.0, 0.0, 32), (33, 65, 5, 0, 1.0, 0.0, 20), (4, 255, 1, 1, 1.0, 0.0, 1), (7, 257, 0, 5, 1.25, 4.0, 8),
    (3, 1000, 24, 0, 1.0, 0.0, 3), (2, 4097, 3, 2, 1.0, 0.0, 32), (9, 8192, 0, 0, 0.7, 0.0, 4),
    (1, 32000, 0, 0, 1.0, 10.0, 5), (17, 32003, 0, 1, 1.0, 0.0, 20), (1, 131072, 0, 0, 1.0, 0.0, 32),
    (3, 131071, 2, 7, 1.0, 0.0, 32), (300, 2048, 0, 0, 1.0, 0.0, 0), (2, 300000, 0, 0, 1.0, 0.0, 32),
    (600, 9001, 0, 0, 1.0, 0.0, 2)])
def test_logprobs(ops, dtype, rows, vocab, pad, offset, scale, clip, top):
    buf, z, tok = make(rows, vocab, pad, dtype, rows * 7 + vocab, offset)
    before = buf.clone()
    a = check_forward(ops, z, tok, scale, clip, top)
    b = ops.token_logprobs(z, tok, scale=scale, clip=clip, top=top)
    for x, y in zip(a, b):  # the same bits each time
        assert (x is None and y is None) or torch.equal(x.view(torch.int32), y.view(torch.int32))
    assert torch.equal(buf, before)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 300, 9001, 70000])
@pytest.mark.parametrize("low", [False, True])
def test_masks(ops, dtype, vocab, low):
    _, z, tok = make(9, vocab, 3, dtype, vocab, 1, masked=0.6, low=low)
    floor = torch.finfo(z.dtype).min if low else -math.inf
    z[2] = floor                 # nothing allowed
    z[3] = floor
    z[3, vocab - 1] = 1.5        # one token, the last
    z[4] = floor
    z[4, 0] = -20.0
    z[5, 1:] = floor
    z[5, 0] = 0.25
    tok[3], tok[4], tok[5] = vocab - 1, 1, 0
    tok[6] = -1
    r = check_forward(ops, z, tok, 1.0, 0.0, 5)
    assert r.logp[6] == 0.0 and r.logp[3] == 0.0 and r.entropy[3] == 0.0
    assert r.lse[2] == -math.inf and r.logp[2] == -math.inf and r.entropy[2] == 0.0
    assert r.top_ids[2].tolist() == [0, 1, 2, 3, 4] and bool((r.top_logp[2] == -math.inf).all())
    if not low:
        check_forward(ops, z, tok, 1.0, 3.0, 5)  # the clip lifts -inf to its bound


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("clip", [0.0, 1e29, 1e31, 3e38])
def test_the_largest_values(ops, dtype, clip):
    """Logits at both ends of their type beside ordinary ones and masks, unclipped and with clips past every mask."""
    big = float(torch.finfo(DT[dtype]).max)
    z = torch.zeros(5, 700)
    z[0, 3], z[0, 5] = big, -big
    z[1, 3:9] = big
    z[2], z[2, 699] = -math.inf, -big
    z[3], z[3, 2], z[3, 4] = -big, -1e28, 5.0
    z[4, ::2], z[4, 1::4] = -math.inf, big
    z = z.to(DT[dtype]).cuda()
    tok = torch.tensor([3, 4, 699, 4, 1], dtype=torch.int32, device="cuda")
    r = ops.token_logprobs(z, tok, clip=clip, top=6)
    x = z.double().cpu()
    x = x.clamp(-clip, clip) if clip else x
    s = torch.where(x <= -1e30, -math.inf, x)
    none = (s == -math.inf).all(1)
    s = s - torch.where(none, 0.0, s.amax(1))[:, None]  # (the largest first: its logarithm is lost beside 1e38)
    ref = torch.where(none[:, None], -math.inf, s - torch.where(none, 0.0, torch.logsumexp(s, 1))[:, None])
    p = ref.exp()
    h = -torch.where(p > 0, p * ref, 0.0).sum(1)
    # sums of up to 700 equal terms: 2 (700 / 64 + 32) u, and the logarithm's rounding
    assert torch.allclose(r.entropy.double().cpu(), h, rtol=0, atol=1e-5)
    want = ref[torch.arange(5), tok.cpu().long()]
    got = r.logp.double().cpu()
    assert torch.equal(torch.isinf(got), torch.isinf(want))
    fine = ~torch.isinf(want)
    assert ((got - want)[fine].abs() <= 1e-5 + want[fine].abs() * U).all()
    for i in range(5):
        order = sorted(range(700), key=lambda v: (-max(float(x[i, v]), -1e30), v))[:6]
        assert r.top_ids[i].tolist() == order, i
    one = torch.ones(5, device="cuda")
    dz = ops.token_logprobs_backward(z, tok, r.lse, r.entropy, one, one, clip=clip)
    assert not dz.isnan().any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [9, 5000, 70001])
def test_special_values_and_tokens(ops, dtype, vocab):
    _, z, tok = make(8, vocab, 0, dtype, 3 + vocab)
    z[0, vocab // 2] = math.nan
    z[1, 3] = math.inf
    z[2, 1] = z[2, vocab - 2] = math.inf
    z[3] = math.nan
    z[4, vocab - 1] = -math.inf
    tok[5], tok[6], tok[7] = vocab, -2, 2 ** 31 - 1
    r = check_forward(ops, z, tok, 1.0, 0.0, 4)
    assert r.logp[4:].isnan().tolist() == [False, True, True, True]
    assert r.top_ids[0, 0] == vocab // 2 and r.top_ids[3].tolist() == [0, 1, 2, 3]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(3, 64), (2, 5003), (70, 40000), (2, 131072)])
def test_alternatives_in_hard_orders(ops, dtype, rows, vocab):
    """Rising, falling and constant rows, rows whose large values lie a power of two apart (all in one thread's
    part), a block of equal values across every step, zeros of both signs."""
    v = torch.arange(vocab, dtype=torch.float64)
    kinds = [v / vocab, -v / vocab, torch.zeros(vocab), torch.where(v % 2 == 0, 0.0, -0.0)]
    for step in (64, 256, 512, 1024, 2048, 4096, 8192):
        kinds.append(torch.where(v % step == step // 2, 10.0 + v / vocab, -1.0))
    kinds.append(torch.where((v > vocab // 3) & (v < vocab // 3 + 2500), 5.0, -v / vocab))
    kinds.append(torch.where(v < 3, 1.0, -math.inf))
    z = torch.stack(kinds).to(DT[dtype]).cuda()
    z = z.repeat((rows + len(kinds) - 1) // len(kinds), 1)
    tok = torch.zeros(len(z), dtype=torch.int32, device="cuda")
    check_forward(ops, z, tok, 1.0, 0.0, 32)
    check_forward(ops, z[:len(kinds)], tok[:len(kinds)], 1.0, 0.0, 1)
    check_forward(ops, z[:2], tok[:2], 1.0, 0.5, 20)  # a clip that makes ties


def test_optional_outputs_and_scratch(ops):
    """Outputs left out, and less scratch than asked for: the same alternatives, sums within the tolerance."""
    from paper_1811_06965_amd import gp
    _, z, tok = make(2, 100003, 0, "f32", 5)
    full = check_forward(ops, z, tok, 1.0, 0.0, 7)
    none = ops.token_logprobs(z, None, top=7)
    assert none.logp is None and torch.equal(none.top_ids, full.top_ids) and torch.equal(none.lse, full.lse)
    need = gp.gp_token_logprobs_workspace(gp.GP_F32, 2, 100003, 7)
    st = torch.cuda.current_stream().cuda_stream
    lse = reference(z, 1.0, 0.0)[2]
    for size in {0, 16, max(0, need - 1), need, need + 1000}:
        ws = torch.full((size + 16,), 0xFF, dtype=torch.uint8, device="cuda")
        ids = torch.empty(2, 7, dtype=torch.int32, device="cuda")
        top, out = torch.empty(2, 7, device="cuda"), torch.empty(2, device="cuda")
        gp.gp_token_logprobs(gp.GP_F32, z.data_ptr(), 2, 100003, 100003, None, 1.0, 0.0, None, out.data_ptr(), None, 7,
                             ids.data_ptr(), top.data_ptr(), ws.data_ptr() if size else None, size, st)
        torch.cuda.synchronize()
        assert torch.equal(ids, full.top_ids)
        R = (3 * 32 + 8) * U + 2 * (100003 / 256 + 32) * U  # logits here stay below 32
        assert (np.abs(out.double().cpu().numpy() - lse) <= R + 32 * 6 * U).all()
        assert bool((ws[size:] == 0xFF).all())
    gp.gp_token_logprobs(gp.GP_F32, z.data_ptr(), 2, 100003, 100003, None, 1.0, 0.0, None, None, None, 0, None, None,
                         None, 0, st)  # nothing asked for
    torch.cuda.synchronize()


def test_rows_past_32_bits(ops):
    """Logits whose offsets pass 2^32 elements and 2^33 bytes: the last rows are right, forward and backward."""
    rows, vocab = 33600, 128000
    z = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda")
    z.fill_(-3.0)
    tail = z[-3:]
    tail.copy_(torch.randn(3, vocab).bfloat16())
    tok = torch.arange(rows, dtype=torch.int32, device="cuda") % vocab
    r = ops.token_logprobs(z, tok, top=3)
    check_forward(ops, tail, tok[-3:], 1.0, 0.0, 3)
    part = ops.token_logprobs(tail, tok[-3:], top=3)
    assert torch.equal(r.top_ids[-3:], part.top_ids)
    assert torch.allclose(r.lse[-3:], part.lse, rtol=0, atol=1e-4)
    assert abs(float(r.lse[rows // 2]) - (math.log(vocab) - 3.0)) < 1e-3
    one = torch.ones(rows, device="cuda")
    dz = ops.token_logprobs_backward(z, tok, r.lse, dlogp=one, out=z)
    sums = dz[-3:].double().sum(1)
    assert (sums.abs() < 1e-2).all() and float(dz[-1, int(tok[-1])]) > 0.9


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_rows_than_a_launch_holds(ops, dtype):
    """More workgroups than one launch can have, 64 threads of the forward's and 256 of the
    gradient's each: every row, the last ones and those at a launch's seam too."""
    rows, vocab = 2 ** 26 + 5, 3
    z = torch.empty(rows, vocab, dtype=DT[dtype], device="cuda")
    z.copy_(torch.arange(rows * vocab, device="cuda", dtype=torch.int32).view(rows, vocab).remainder_(61).sub_(30))
    tok = torch.arange(rows, dtype=torch.int32, device="cuda").remainder_(3)
    r = ops.token_logprobs(z, tok, scale=0.1, top=2)
    one = torch.ones(rows, device="cuda")
    dz = ops.token_logprobs_backward(z, tok, r.lse, r.entropy, one, one, scale=0.1)
    # every row is one of 61 * 3 (the first value's remainder by 61, the token's by 3), to the bit
    for got in (r.logp, r.entropy, r.top_ids, r.top_logp, dz):
        whole = got[:rows // 183 * 183].view(-1, 183, *got.shape[1:])
        assert bool((whole == whole[:1]).all()) and torch.equal(got[rows // 183 * 183:], got[:rows % 183])
    check_forward(ops, z[:183], tok[:183], 0.1, 0.0, 2)
    part = ops.token_logprobs(z[:183], tok[:183], scale=0.1, top=2)
    for got, want in zip(r, part):
        assert torch.equal(got[:183], want)
    want = ops.token_logprobs_backward(z[:183], tok[:183], part.lse, part.entropy, one[:183], one[:183], scale=0.1)
    assert torch.equal(dz[:183], want)  # test_gradient holds such rows to the formula


# ------------------------------------------------------------------- gradient
def check_backward(ops, buf, z, tok, scale, clip, seed, use=(True, True), inplace=False, pad_out=0):
    rows, V = z.shape
    g = torch.Generator().manual_seed(seed)
    f = ops.token_logprobs(z, tok, scale=scale, clip=clip)
    a = torch.randn(rows, generator=g).cuda() if use[0] else None
    b = (torch.randn(rows, generator=g) * 0.3).cuda() if use[1] else None
    zc = z.clone()
    if inplace:
        out = z
    else:
        obuf = torch.full((rows * (V + pad_out) + 3,), 5.0, device="cuda", dtype=z.dtype)
        out = obuf[1:1 + rows * (V + pad_out)].view(rows, V + pad_out)[:, :V]
    got = ops.token_logprobs_backward(z, tok if use[0] else None, f.lse, f.entropy if use[1] else None, a, b,
                                      scale=scale, clip=clip, out=out)
    got = got.double().cpu().numpy()
    x, s, lse, p, d, h = reference(zc, scale, clip)
    raw = zc.double().cpu().numpy()
    n = lambda t: np.zeros((rows, 1)) if t is None else t.double().cpu().numpy()[:, None]  # noqa: E731
    t = tok.cpu().numpy()
    av, bv, hv = n(a).copy(), n(b), n(f.entropy)
    av[t == -1] = 0.0
    lv = n(f.lse)
    with np.errstate(all="ignore"):
        empty = lv == -np.inf
        p = np.where(empty | (s == -np.inf), 0.0, np.exp(s - lv))
        d = np.where(s == -np.inf, 0.0, s - np.where(empty, 0.0, lv))
        one = np.zeros_like(s)
        ok = (t >= 0) & (t < V) & ~empty[:, 0]
        one[np.arange(rows)[ok], t[ok]] = 1.0
        want = scale * (av * (one - p) - bv * p * (d + hv))
        if clip > 0:
            want = np.where(np.abs(raw) <= clip, want, 0.0)
        mag = np.where(s == -np.inf, 0.0, np.abs(s)) + np.where(np.isfinite(lv), np.abs(lv), 0.0)
        terms = p * (np.abs(av) + np.abs(bv) * (np.abs(d) + np.abs(hv) + 1))
        # a probability below the smallest normal float, 2^-126, counts as 0
        flush = 2.0 ** -126 * (np.abs(av) + np.abs(bv) * (np.abs(d) + np.abs(hv)))
        tol = scale * (terms * (4 * mag + 16) * U + np.abs(av) * one * 8 * U + flush)
    half = 2.0 ** -8 if z.dtype == torch.bfloat16 else U
    # below the normal range a step is 2^-133 (bf16) or 2^-149
    tol = tol * (1 + half) + np.abs(want) * half + 2.0 ** (-133 if z.dtype == torch.bfloat16 else -126)
    bad = (t < -1) | (t >= V)
    if use[0] and bad.any():
        assert np.isnan(got[bad]).all()
    keep = ~bad if use[0] else np.ones(rows, bool)
    assert not np.isnan(got[keep]).any()
    assert (np.abs(got - want)[keep] <= tol[keep]).all()
    if not inplace:
        assert torch.equal(z, zc)
        o = obuf.clone()
        o[1:1 + rows * (V + pad_out)].view(rows, V + pad_out)[:, :V] = 5.0
        assert bool((o == 5.0).all())  # nothing behind a row was written


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,offset,scale,clip,pad_out", [
    (1, 1, 0, 0, 1.0, 0.0, 0), (2, 2, 0, 1, 1.0, 0.0, 0), (5, 63, 2, 3, 0.5, 0.0, 1), (3, 64, 0, 0, 1.0, 2.0, 0),
    (33, 255, 1, 0, 1.25, 0.0, 9), (4, 1000, 24, 0, 1.0, 3.0, 24), (9, 4099, 0, 1, 1.0, 0.0, 5),
    (300, 2048, 0, 0, 1.0, 0.0, 0), (3, 32000, 0, 0, 1.0, 5.0, 0), (2, 131071, 1, 7, 1.0, 0.0, 0)])
@pytest.mark.parametrize("use", [(True, True), (True, False), (False, True)])
def test_gradient(ops, dtype, rows, vocab, pad, offset, scale, clip, pad_out, use):
    buf, z, tok = make(rows, vocab, pad, dtype, rows + vocab, offset)
    check_backward(ops, buf, z, tok, scale, clip, 1, use, pad_out=pad_out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("clip", [0.0, 4.0])
@pytest.mark.parametrize("vocab", [5, 300, 9001])
@pytest.mark.parametrize("low", [False, True])
def test_gradient_of_masks_padding_and_bad_tokens(ops, dtype, clip, vocab, low):
    buf, z, tok = make(9, vocab, 3, dtype, vocab, 1, masked=0.6, low=low)
    z[2] = z[3] = torch.finfo(z.dtype).min if low else -math.inf
    z[3, vocab - 1] = 1.5
    tok[3] = vocab - 1
    tok[4], tok[5], tok[6] = -1, vocab, -7
    check_backward(ops, buf, z, tok, 1.0, clip, 2)
    check_backward(ops, buf, z, tok, 1.0, clip, 2, use=(False, True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_in_place(ops, dtype):
    buf, z, tok = make(6, 5003, 5, dtype, 8, 1)
    before = buf.clone()
    check_backward(ops, buf, z, tok, 1.0, 0.0, 3, inplace=True)
    view = lambda t: t[1:1 + 6 * 5008].view(6, 5008)[:, 5003:]  # noqa: E731
    assert torch.equal(view(buf), view(before)) and torch.equal(buf[:1], before[:1])


def test_gradient_against_differences(ops):
    """Central differences of the forward pass in 64 bits at 40 logits: h = 1e-4, so the formula is met to 1e-7
    relative to the terms (error h^2 / 6 times third derivatives of order one)."""
    torch.manual_seed(0)
    z = torch.randn(3, 40, device="cuda") * 2
    tok = torch.tensor([3, 39, 0], dtype=torch.int32, device="cuda")
    a, b = torch.tensor([0.7, -1.1, 0.4], device="cuda"), torch.tensor([0.2, -0.5, 1.3], device="cuda")
    f = ops.token_logprobs(z, tok, scale=1.3)
    dz = ops.token_logprobs_backward(z, tok, f.lse, f.entropy, a, b, scale=1.3).double().cpu().numpy()

    def value(x):
        s = x * 1.3
        lse = np.log(np.exp(s).sum(1))
        p = np.exp(s - lse[:, None])
        h = lse - (p * s).sum(1)
        return a.double().cpu().numpy() * (s[np.arange(3), tok.cpu().numpy()] - lse) + b.double().cpu().numpy() * h

    x = z.double().cpu().numpy()
    for v in range(40):
        e = np.zeros_like(x)
        e[:, v] = 1e-4
        diff = (value(x + e) - value(x - e)) / 2e-4
        assert (np.abs(diff - dz[:, v]) < 1e-6).all()


def test_no_rows(ops):
    z = torch.empty(0, 100, device="cuda")
    tok = torch.empty(0, dtype=torch.int32, device="cuda")
    r = ops.token_logprobs(z, tok, top=3)
    assert r.logp.shape == (0,) and r.top_ids.shape == (0, 3)
    assert ops.token_logprobs_backward(z, tok, r.lse, r.entropy, r.lse, r.entropy).shape == (0, 100)


def test_two_streams_and_a_graph(ops):
    """Two calls side by side on two streams, and both directions captured and replayed on new inputs, with eager
    work between the replays: every result is the eager one, bit for bit."""
    cases = [make(3, 70001, 0, "bf16", s)[1:] for s in (1, 2)]
    want = [ops.token_logprobs(z, t, top=9) for z, t in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i] = ops.token_logprobs(*cases[i], top=9)
        torch.cuda.synchronize()
        for w, r in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(w, r))
    z, tok = cases[0][0].clone(), cases[0][1].clone()
    one = torch.ones(3, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = ops.token_logprobs(z, tok, top=9)
        dz = ops.token_logprobs_backward(z, tok, r.lse, r.entropy, one, one)
    for k in range(4):
        z.copy_(cases[k % 2][0])
        tok.copy_(cases[k % 2][1])
        graph.replay()
        torch.cuda.synchronize()
        e = want[k % 2]
        assert all(torch.equal(x, y) for x, y in zip(e, r))
        assert torch.equal(dz, ops.token_logprobs_backward(z, tok, e.lse, e.entropy, one, one))
