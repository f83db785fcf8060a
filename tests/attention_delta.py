"""How far the gradients that depend on delta = sum_j p_j dP_j may be off as a whole (the 2-norm of a tensor's error), when delta is
rid of the rounding of out (test infrastructure).  attention_reference.py's bounds are of single values and add every error up at
its largest, so that they have room for out's rounding in every row; here errors that have nothing to do with each other
are added in squares, which leaves no room for it.

u = 2^-24; a rounding to bf16 is off by at most r = 2^-8 / sqrt(3) of a value on the root mean square.  Per pair:
* a weight p is off by w of itself, w = u ((sqrt(dh) + 8) scale |q|.|k| + 4 (|scale q.k| + |bias|) + (dh / 16 + 8) (|lse| + 1)): dh sums
  whose roundings differ, a scaling and a sum, and the lse, from which the dh / 16 products may start;
* dP by g = u ((sqrt(dh) + 8) |dout|.|v| + (dh / 16 + 4) |delta|);
* delta by d = sum p (w (|dP| + |delta|) + g + sqrt(Sk) u (|dP| + |delta|)) + 4 u |delta|, whichever of its two forms is taken;
* dS by D = w |dS| + p (g + d).
Sums of D within a row are absolute (its errors may be common to the row), over rows in squares.
* dbias: a row's D over the bucket; Sq + 64 roundings of sums at most as large as the rows' absolute sum.
* dq, delta known beforehand: r |dS| |k| in squares, D |k|, r |dq|.
* dq, with the row's mean key R taken off as often as the rounded dS' add up to: r |dS'| |k - R| in squares, D |k - R|, r |dq|, and that
  sum, sqrt((delta - d0)^2 + sum (r dS')^2), times what sum p k is off by, sqrt(sum (r p k)^2) + sum w p |k|; d0 = dout . (out rounded).
* dk: r |dS| |q| and D |q| in squares over the rows, r |dk|.
"""
import math

import torch

U = 2.0 ** -24
R = 2.0 ** -8 / math.sqrt(3.0)


def heads_first(t, H):
    t = t.double().permute(0, 2, 1, 3)
    return t.repeat_interleave(H // t.shape[1], 1).contiguous()


def mm(a, b):
    return torch.matmul(a.contiguous(), b.contiguous())


def inputs(B, H, K, Sq, Sk, dh, buckets, device, seed=0, dtype=torch.bfloat16):
    """Keys and values around a vector that they share, which makes delta and out large beside what dS is made of."""
    g = torch.Generator(device=device).manual_seed(seed)

    def rn(*shape):
        return torch.randn(*shape, generator=g, device=device)
    q, dout = rn(B, Sq, H, dh), rn(B, Sq, H, dh)
    k, v = rn(B, Sk, K, dh) + 3.0 * rn(K, dh), rn(B, Sk, K, dh) + 6.0 * rn(K, dh)
    table = rn(H, buckets) if buckets else None
    return q.to(dtype), k.to(dtype), v.to(dtype), dout.to(dtype), table


def exact(q, k, v, dout, scale, ok, table=None, of=None, dist=None):
    """64-bit results and the pieces that the bounds and the imitation below are made of."""
    H, K = q.shape[2], k.shape[2]
    qh, kh, vh, gh = (heads_first(t, H) for t in (q, k, v, dout))
    x = mm(qh, kh.transpose(2, 3)) * scale
    bias = torch.zeros_like(x)
    bucket = None
    if table is not None:
        far = (len(of) - 1) // 2
        bucket = torch.tensor(of, device=q.device)[dist.clamp(-far, far) + far]
        bias = table.double()[:, bucket].transpose(0, 1).expand_as(x)
    s = torch.where(ok[:, None], x + bias, -math.inf)
    lse = torch.logsumexp(s, 3, keepdim=True)
    p = torch.exp(s - lse)
    o = mm(p, vh)
    dp = mm(gh, vh.transpose(2, 3))
    delta = (p * dp).sum(3, keepdim=True)
    ds = p * (dp - delta)
    return dict(q=qh, k=kh, v=vh, g=gh, x=x, bias=bias, bucket=bucket, lse=lse, p=p, out=o, dp=dp, delta=delta, ds=ds, scale=scale,
                groups=K, buckets=0 if table is None else table.shape[1])


def gradients(e, ds, dq=None):
    """dq (unless given), dk and dbias, rows first, of these dS [B, H, Sq, Sk]."""
    B, H, Sq, Sk = ds.shape
    r = {"dq": (mm(ds, e["k"]) if dq is None else dq).permute(0, 2, 1, 3) * e["scale"]}
    dk = mm(ds.transpose(2, 3), e["q"]) * e["scale"]
    r["dk"] = dk.view(B, e["groups"], -1, Sk, dk.shape[-1]).sum(2).permute(0, 2, 1, 3)
    if e["bucket"] is not None:
        r["dbias"] = by_bucket(e, ds).sum((0, 2))
    return r


def by_bucket(e, t):
    """Sums of t [B, H, Sq, Sk] over a row's pairs of each bucket: [B, H, Sq, buckets]."""
    z = torch.zeros(*t.shape[:3], e["buckets"], dtype=t.dtype, device=t.device)
    return z.scatter_add_(3, e["bucket"][:, None].expand_as(t), t)


def bounds(e, refined):
    """Of the norm of the error of dq, dk and dbias.  refined: the row's mean key is taken off dq."""
    B, H, Sq, Sk = e["p"].shape
    dh = e["q"].shape[-1]
    p, ds, dp, delta, scale = e["p"], e["ds"], e["dp"], e["delta"], e["scale"]
    many = math.sqrt(dh) + 8
    w = U * (many * scale * mm(e["q"].abs(), e["k"].abs().transpose(2, 3)) + 4 * (e["x"].abs() + e["bias"].abs()) +
             (dh / 16 + 8) * (e["lse"].abs() + 1))
    g = U * (many * mm(e["g"].abs(), e["v"].abs().transpose(2, 3)) + (dh / 16 + 4) * delta.abs())
    size = dp.abs() + delta.abs()
    d = (p * (w * size + g + math.sqrt(Sk) * U * size)).sum(3, keepdim=True) + 4 * U * delta.abs()
    D = w * ds.abs() + p * (g + d)
    exact_grads = gradients(e, ds)

    def norm2(t):
        return float((t * t).sum())
    r = {}
    if e["bucket"] is not None:
        rows = by_bucket(e, ds).abs().sum((0, 2))
        r["dbias"] = math.sqrt(norm2(by_bucket(e, D)) + (Sq + 64) * norm2(U * rows))
    if refined:
        mean = mm(p, e["k"])
        d0 = (e["g"] * e["out"].bfloat16().double()).sum(3, keepdim=True)
        first = p * (dp - d0)
        # by feature: the sum over keys of dS'^2 (k - R)^2, and
        sq = mm(first ** 2, e["k"] ** 2) - 2 * mean * mm(first ** 2, e["k"]) + mean ** 2 * (first ** 2).sum(3, keepdim=True)
        # sum D |k - R| <= sqrt(sum D) sqrt(sum D (k - R)^2), by Cauchy and Schwarz
        spread = (mm(D, e["k"] ** 2) - 2 * mean * mm(D, e["k"]) + mean ** 2 * D.sum(3, keepdim=True)).clamp(min=0)
        total = torch.sqrt((delta - d0) ** 2 + R * R * (first ** 2).sum(3, keepdim=True))
        of_mean = R * torch.sqrt(mm(p ** 2, e["k"] ** 2)) + mm(w * p, e["k"].abs())
        per_row = torch.sqrt(D.sum(3, keepdim=True) * spread) + total * of_mean
        e2 = R * R * norm2(torch.sqrt(sq.clamp(min=0))) + norm2(per_row)
    else:
        e2 = R * R * float(mm(ds ** 2, e["k"] ** 2).sum()) + norm2(mm(D, e["k"].abs()))
    r["dq"] = scale * math.sqrt(e2) + R * math.sqrt(norm2(exact_grads["dq"]))
    e2 = float(mm(((R * ds) ** 2 + D ** 2).transpose(2, 3), e["q"] ** 2).sum())
    r["dk"] = scale * math.sqrt(e2) + R * math.sqrt(norm2(exact_grads["dk"]))
    return exact_grads, r


def ratios(got, ref, lim):
    """The error of each gradient over its bound."""
    return {n: float((got[n].double() - ref[n]).norm()) / lim[n] for n in lim}


def imitation(e, delta_of, refined):
    """The gradients as a bf16 computation makes them, from delta_of(d0, sum of dS'): P and dS rounded to bf16 before their products,
    and the results once."""
    p, dp = e["p"], e["dp"]

    def b(t):
        return t.bfloat16().double()
    d0 = (e["g"] * b(e["out"])).sum(3, keepdim=True)
    first = p * (dp - d0)
    delta = delta_of(d0, first.sum(3, keepdim=True))
    ds = p * (dp - delta)
    dq = None
    if refined:
        dq = mm(b(first), e["k"]) - b(first).sum(3, keepdim=True) * mm(b(p), e["k"])
    r = gradients(e, b(ds), mm(b(ds), e["k"]) if dq is None else dq)
    if "dbias" in r:
        r["dbias"] = by_bucket(e, ds).sum((0, 2))  # from dS as it is
    for n in ("dq", "dk"):
        r[n] = b(r[n])
    return r
