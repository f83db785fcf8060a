"""Attention and its gradients from their formulas in 64 bits, with bounds of what a computation in fp32 (and bf16 products)
may be off by (test infrastructure).

u = 2^-24 is half a step of fp32, e that of the type (bf16 2^-8, fp32 u).  Inputs are exact.  Per pair:
* s = scale q.k + bias: dh products and as many sums of |q_d k_d|, a scaling (its factor rounded once more, to log 2
  units), a sum: S = u (dh + 8) scale |q|.|k| + 4 u (|s| + |bias|); the exponential 4 u; the largest S of a row enters its lse too;
* p is off by P = p (S + Smax + (Sk + 16) u) of itself, Sk sums among them (in any order), and is rounded by e before a product;
* out: sum (P + e p + Sk u p) |v| + e |out|;
* dP = dout.v: dh u |dout|.|v|; delta: what out is off by, times |dout|, and dh u |dout|.|out|; from the weights alone,
  sum P |dP| + p (dh + Sk) u |dout|.|v|; the larger of the two is taken;
* dS = p (dP - delta): D = P |dP - delta| + p (dP's + delta's) + 3 u |dS|;
* dq: scale (sum (D + e |dS| + Sk u |dS|) |k|) + e |dq|; dk with the rows of all heads that share the key; dv with P + e p and |dout|;
* dbias: sum over a bucket of D + n u |dS|, n the sums that any value passes through: at most those of a row of blocks (Sk), 32 in
  each block, and the joins (Sq + batch).
"""
import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def buckets_of(buckets, max_distance, bidirectional):
    """Bucket by distance from -max_distance to max_distance, borders in whole numbers."""
    n = buckets // 2 if bidirectional else buckets
    half = n // 2

    def side(d):
        if d < half:
            return d
        t = 0
        while t + 1 < n - half and d ** (n - half) * half ** (t + 1) >= max_distance ** (t + 1) * half ** (n - half):
            t += 1
        return half + t

    before = [side(d) for d in range(max_distance + 1)]
    behind = [n + side(d) if bidirectional else 0 for d in range(1, max_distance + 1)]
    return before[::-1] + behind


def visible(B, Sq, Sk, q_lens=None, k_lens=None, q_starts=None, causal=False, device="cuda"):
    """(pairs that count [B, Sq, Sk], distance key - position [B, Sq, Sk])."""
    def col(t, default):
        t = torch.full((B,), default, device=device) if t is None else t.long()
        return t[:, None, None]
    i, j = torch.arange(Sq, device=device)[:, None], torch.arange(Sk, device=device)[None]
    dist = j - (i + col(q_starts, 0))
    ok = (j < col(k_lens, Sk)) & (i < col(q_lens, Sq))
    return (ok & (dist <= 0) if causal else ok), dist


def attention(q, k, v, scale, ok, table=None, of=None, dist=None, dout=None):
    """A dict of float64 results and of their bounds ("~name"): out, lse and, with dout, dq, dk, dv, dbias."""
    e, dt = HALF[q.dtype], torch.float64
    B, Sq, H, dh = q.shape
    Sk, K = k.shape[1], k.shape[2]
    g = H // K

    def heads(t):  # [B, H, S, dh]
        t = t.to(dt).permute(0, 2, 1, 3)
        return t.repeat_interleave(H // t.shape[1], 1).contiguous()

    def rows(t):
        return t.permute(0, 2, 1, 3)

    def mm(a, b):
        return torch.matmul(a.contiguous(), b.contiguous())

    ok = ok[:, None]
    qh, kh, vh = heads(q), heads(k), heads(v)
    live_q, live_k = ok.any(3)[..., None], ok.any(2)[..., None]
    qh, kh, vh = (torch.where(l, t, 0.0) for l, t in ((live_q, qh), (live_k, kh), (live_k, vh)))
    s = mm(qh, kh.transpose(2, 3)) * scale
    off = U * (dh + 8) * scale * mm(qh.abs(), kh.abs().transpose(2, 3)) + 4 * U * s.abs()
    if table is not None:
        D = (len(of) - 1) // 2
        bucket = torch.tensor(of, device=q.device)[dist.clamp(-D, D) + D]
        bias = table.to(dt)[:, bucket].transpose(0, 1)
        masked = bias <= -1e30
        ok = ok & ~masked
        bias = torch.where(masked, 0.0, bias)
        s, off = s + bias, off + 4 * U * bias.abs()
    ok = ok.expand(B, H, Sq, Sk)
    x = torch.where(ok, s, -math.inf)
    lse = torch.logsumexp(x, 3)
    some = lse > -math.inf
    p = torch.where(some[..., None], torch.exp(x - torch.where(some, lse, 0.0)[..., None]), 0.0)
    off = torch.where(ok, off, 0.0)
    most = off.amax(3, keepdim=True) if Sk else torch.zeros(B, H, Sq, 1, dtype=dt, device=q.device)
    P = p * (off + most + (Sk + 16) * U)
    out = mm(p, vh)
    lim = mm(P + (e + Sk * U) * p, vh.abs()) + e * out.abs()
    r = {"out": rows(out), "~out": rows(lim), "lse": lse, "~lse": most[..., 0] + (Sk + 16) * U + 4 * U * lse.abs()}
    r["~lse"] = torch.where(some, r["~lse"], 0.0)
    if dout is None:
        return r
    gh = torch.where(live_q, heads(dout), 0.0)
    dp, mag = mm(gh, vh.transpose(2, 3)), mm(gh.abs(), vh.abs().transpose(2, 3))
    delta = (gh * out).sum(3, keepdim=True)
    d_off = torch.maximum((gh.abs() * lim).sum(3, keepdim=True) + dh * U * (gh * out).abs().sum(3, keepdim=True),
                          (P * dp.abs() + p * (dh + Sk) * U * mag).sum(3, keepdim=True)) + 4 * U * delta.abs()
    ds = p * (dp - delta)
    D_off = P * (dp - delta).abs() + p * (dh * U * mag + d_off) + 3 * U * ds.abs()
    r["dq"] = rows(mm(ds, kh)) * scale
    r["~dq"] = rows(mm(D_off + (e + Sk * U) * ds.abs(), kh.abs())) * scale + (e + U) * r["dq"].abs()

    def shared(t):  # [B, H, Sk, dh] -> sums over the heads of a group, rows first
        return rows(t.view(B, K, g, Sk, dh).sum(2))

    n = Sq * g + 16
    r["dk"] = shared(mm(ds.transpose(2, 3), qh)) * scale
    r["~dk"] = shared(mm((D_off + (e + n * U) * ds.abs()).transpose(2, 3), qh.abs())) * scale + (e + U) * r["dk"].abs()
    r["dv"] = shared(mm(p.transpose(2, 3), gh))
    r["~dv"] = shared(mm((P + (e + n * U) * p).transpose(2, 3), gh.abs())) + e * r["dv"].abs()
    if table is not None:
        m = Sk + 64 + Sq + B

        def by_bucket(t):
            z = torch.zeros(H, table.shape[1], dtype=dt, device=q.device)
            for b in range(B):
                z.index_add_(1, bucket[b if bucket.shape[0] > 1 else 0].reshape(-1), t[b].reshape(H, -1))
            return z
        r["dbias"], r["~dbias"] = by_bucket(ds), by_bucket(D_off + m * U * ds.abs())
    return r


def check(name, got, ref, floor=1e-37):
    """Every value within its bound; infinities and NaN in the same places."""
    a, b, lim = got.double(), ref[name], ref["~" + name]
    same = (a == b) | (a.isnan() & b.isnan())
    bad = ~same & ~((a - b).abs() <= lim + floor)
    assert not bad.any(), (name, int(bad.sum()), float((a - b)[bad].abs().max()), float(((a - b).abs() / (lim + floor))[bad].max()))
