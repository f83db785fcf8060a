"""Operators of an encoder-decoder that is trained from a teacher, measured one call at a time.

Three operators: attention to an encoder's states of another length, over a
ragged batch, with shared heads and for single tokens ("cross"); self-attention
with a learned relative position bias by buckets ("bias"); the distillation loss
against a teacher's top log probabilities ("distill").  Each has its backward pass.

With ``own`` false a pass computes them from their formulas in elementary
torch operations, in 32 bits and rounded once; with ``own`` true through the
package's entry points (``paper_1811_06965_amd.ops``).  Inputs come from the
seed alone and are the same on both sides.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ESZ = {"f32": 4, "bf16": 2}


# -------------------------------------------------------------------- cases
def _attn(name, **kw):
    base = dict(name=name, op="cross", grad=False, dtype="bf16", batch=1, heads=16, kv_heads=16, d_head=64, q_len=1,
                k_len=256, fill=1.0, empty=False, causal=False, buckets=0, max_distance=0)
    return {**base, **kw}


def _bias(name, **kw):
    return _attn(name, **{"op": "bias", "buckets": 32, "max_distance": 128, **kw})


def _distill(name, **kw):
    base = dict(name=name, op="distill", grad=False, dtype="bf16", rows=1, vocab=32000, pad=0, top=32, scale=1.0,
                clip=0.0, rest=True)
    return {**base, **kw}


def listed():
    return [
        # four sequences being translated, one token each, to encoder states of up to 200 tokens: latency
        _attn("cross-token", batch=4, k_len=200, fill=0.4),
        # sixteen long documents answered token by token, four query heads to a key head
        _attn("cross-token-long", batch=16, heads=32, kv_heads=8, d_head=128, k_len=32768, fill=0.3),
        # a mini-batch of the d_model 1024 decoder, its sources longer than its targets, and its backward pass
        _attn("cross-1024", batch=64, q_len=256, k_len=320, fill=0.5),
        _attn("cross-1024-grad", grad=True, batch=64, q_len=256, k_len=320, fill=0.5),
        # fp32 at odd lengths and an odd width, shared heads, one sequence without any key
        _attn("cross-odd-grad", grad=True, dtype="f32", batch=3, heads=6, kv_heads=2, d_head=40, q_len=77, k_len=501,
              fill=0.3, empty=True),
        # a long document summarised: one sequence, 50000 states
        _attn("cross-long", heads=16, kv_heads=4, d_head=128, q_len=1000, k_len=50000),
        # the encoder's self-attention at the benchmark's length
        _bias("bias-256", batch=8, q_len=256, k_len=256),
        # longer sequences in training
        _bias("bias-2048-grad", grad=True, batch=4, q_len=2048, k_len=2048),
        # a decoder's own bias: causal, fp32, odd
        _bias("bias-odd-grad", grad=True, dtype="f32", batch=2, heads=5, kv_heads=5, d_head=24, q_len=331, k_len=331,
              causal=True, buckets=20, max_distance=60),
        # fp32 logits at an odd width and row stride, 100 of the teacher's tokens
        _distill("distill-odd", dtype="f32", rows=93, vocab=50021, pad=27, top=100, scale=0.5),
        # one micro-batch of the translation decoder with its vocabulary and clip
        _distill("distill-1024-grad", grad=True, rows=1024, clip=10.0, rest=False),
        # a long batch under a large vocabulary
        _distill("distill-4096", rows=4096, vocab=128000, top=64),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["cross", "cross", "bias", "bias", "distill"])
        if op == "distill":
            c = _distill("", grad=rng.random() < 0.5, rows=log_int(1, 4096), vocab=log_int(130, 131072),
                         pad=rng.choice([0, 0, 1, 8, 21]), dtype=rng.choice(["bf16", "f32"]),
                         top=rng.choice([1, 8, 20, 32, 64, 100, 128]), scale=rng.choice([1.0, 1.0, 0.5, 0.25]),
                         clip=rng.choice([0.0, 0.0, 10.0]), rest=rng.random() < 0.5)
            fits = c["rows"] * c["vocab"] * ESZ[c["dtype"]] <= 1.0e9
        else:
            dtype = rng.choice(["bf16", "bf16", "f32"])
            kv = rng.choice([1, 2, 4, 5, 8, 16])
            c = dict(dtype=dtype, batch=log_int(1, 64), kv_heads=kv, d_head=rng.choice([24, 32, 40, 64, 64, 96, 128, 128]),
                     grad=rng.random() < 0.5, fill=rng.choice([1.0, 0.7, 0.3]))
            if op == "bias":
                n = log_int(2, 8192)
                c = _bias("", **c, heads=kv, q_len=n, k_len=n, causal=rng.random() < 0.5,
                          buckets=rng.choice([8, 32, 32, 64]), max_distance=rng.choice([40, 128, 128, 500]))
            else:
                c = _attn("", **c, heads=kv * rng.choice([1, 1, 2, 4]), q_len=rng.choice([1, log_int(2, 4096)]),
                          k_len=log_int(2, 65536))
                c["grad"] = c["grad"] and c["q_len"] > 1
            scores = c["batch"] * c["heads"] * c["q_len"] * c["k_len"]
            w = work(c)
            fits = scores <= 8.0e8 and w["bytes"] <= 1.4e9 and w["flops"] <= 4.0e11
        if fits:
            del c["name"]
            return c


# -------------------------------------------------------------------- sizes
def _key_lens(c):
    """Keys of each sequence: from all of them down to a share `fill`, evenly."""
    B, n = c["batch"], c["k_len"]
    if B == 1:
        return [n]
    lens = [max(1, round(n * (1.0 - (1.0 - c["fill"]) * b / (B - 1)))) for b in range(B)]
    if c["empty"]:
        lens[-1] = 0
    return lens


def _pairs(c):
    """Pairs of a query and a key that it may see, over the batch."""
    if not c["causal"]:
        return c["q_len"] * sum(_key_lens(c))
    return sum(min(i + 1, n) for n in _key_lens(c) for i in range(c["q_len"]))


def work(case):
    c = case
    if c["op"] == "distill":
        n = c["rows"] * c["vocab"]
        side = c["rows"] * (8 * c["top"] + 12)
        if c["grad"]:
            return {"bytes": 2 * n * ESZ[c["dtype"]] + side, "flops": 5.0 * n}
        return {"bytes": n * ESZ[c["dtype"]] + side, "flops": 4.0 * n}
    q = c["batch"] * c["q_len"] * c["heads"] * c["d_head"]
    kv = sum(_key_lens(c)) * c["kv_heads"] * c["d_head"]
    rows = c["batch"] * c["q_len"] * c["heads"]
    bias = 4 * c["heads"] * c["buckets"]
    if c["grad"]:
        # q, out, dout, dq; k, v read; dk, dv written whole
        whole = c["batch"] * c["k_len"] * c["kv_heads"] * c["d_head"]
        return {"bytes": (4 * q + 2 * kv + 2 * whole) * ESZ[c["dtype"]] + 4 * rows + 2 * bias,
                "flops": 10.0 * c["heads"] * c["d_head"] * _pairs(c)}
    return {"bytes": (2 * q + 2 * kv) * ESZ[c["dtype"]] + 4 * rows + bias,
            "flops": 4.0 * c["heads"] * c["d_head"] * _pairs(c)}


# ------------------------------------------------------------------- inputs
def _edges(c):
    """Distances at which the buckets of one side begin: the first half one by one, the rest spaced evenly in the
    logarithm up to max_distance.  Whole numbers, so that no border is rounded."""
    n = c["buckets"] // (1 if c["causal"] else 2)
    half, far = n // 2, c["max_distance"]
    edges = list(range(1, half + 1))
    for t in range(1, n - half):
        d = half
        while d ** (n - half) * half ** t < far ** t * half ** (n - half):
            d += 1
        edges.append(d)
    return edges


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    if c["op"] == "distill":
        return _distill_inputs(c, g)
    dt = DTYPES[c["dtype"]]
    B, H, K, dh = c["batch"], c["heads"], c["kv_heads"], c["d_head"]

    def rn(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    # queries and keys with the spread that trained layers give scores, a direction that all keys of a head share,
    # keys and values side by side as one projection makes them
    s = {"case": c, "q": (rn(B, c["q_len"], H, dh) * 1.5).to(dt)}
    kv = torch.empty(B, c["k_len"], 2, K, dh, device="cuda", dtype=dt)
    shared = rn(K, dh) * 0.5
    for b in range(B):
        kv[b] = rn(c["k_len"], 2, K, dh)
        kv[b, :, 0] += shared.to(dt)
    s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
    order = torch.randperm(B, device="cuda", generator=g)
    s["k_lens"] = torch.tensor(_key_lens(c), dtype=torch.int32, device="cuda")[order]
    s["scale"] = dh ** -0.5
    if c["buckets"]:
        s["table"] = rn(H, c["buckets"])
        s["edges"] = torch.tensor(_edges(c), device="cuda")
    if c["grad"]:
        # what the forward pass left, and the gradient that comes from behind
        out, s["lse"] = _plain_forward(s)[:2]
        s["out"] = out.to(dt)
        s["dout"] = rn(B, c["q_len"], H, dh).to(dt)
    return s


def _distill_inputs(c, g):
    """Logits as a trained student's head gives them, a teacher whose likely tokens the student partly knows.  The
    teacher's log probabilities come largest first; some rows name fewer tokens (-1 behind them), some none."""
    R, V, n = c["rows"], c["vocab"], c["top"]
    z = torch.empty(R, V + c["pad"], device="cuda", dtype=DTYPES[c["dtype"]])
    for r in range(0, R, 512):  # 512 rows at a time, so that the 32-bit draws stay small
        z[r:r + 512] = torch.randn(z[r:r + 512].shape, device="cuda", generator=g) * 2.0 - 4.0
    z = z[:, :V]
    # n different tokens a row: one from each of n equal parts of the vocabulary, in any order
    part = V // n
    ids = torch.argsort(torch.rand(R, n, device="cuda", generator=g), 1) * part
    ids = ids + torch.randint(0, part, (R, n), device="cuda", generator=g)
    known = min(n, 12)
    z.scatter_(1, ids[:, :known], (torch.randn(R, known, device="cuda", generator=g) * 2.5 + 5.0).to(z.dtype))
    t = torch.log_softmax(torch.randn(R, n, device="cuda", generator=g).sort(1, descending=True).values * 2.5, 1)
    t = t + torch.log(0.8 + 0.199 * torch.rand(R, 1, device="cuda", generator=g))
    if R > 3:
        left = torch.randint(1, n + 1, (R, 1), device="cuda", generator=g)
        left = torch.where(torch.rand(R, 1, device="cuda", generator=g) < 0.8, n, left)
        left[R // 2] = 0
        ids = torch.where(torch.arange(n, device="cuda") < left, ids, -1)
    s = {"case": c, "z": z, "ids": ids.to(torch.int32), "teacher": t}
    if c["grad"]:
        loss = _plain_distill(s)
        s["lse"], s["rest_lse"] = loss["lse"], loss.get("rest_lse")
        s["dloss"] = torch.rand(R, device="cuda", generator=g) / R
    return s


# -------------------------------------------------------------- plain forms
def _heads_first(x, groups):
    """[B, S, H, dh] -> fp32 [B, groups, (H / groups) S, dh]: the rows of the heads that share keys together."""
    B, S, H, dh = x.shape
    return x.float().permute(0, 2, 1, 3).reshape(B, groups, H // groups * S, dh)


def _rows_first(x, H):
    """The way back."""
    B, dh = x.shape[0], x.shape[-1]
    return x.reshape(B, H, -1, dh).permute(0, 2, 1, 3)


def _buckets(s):
    """Bucket of every pair of a query and a key: [Sq, Sk]."""
    c = s["case"]
    rel = torch.arange(c["k_len"], device="cuda") - torch.arange(c["q_len"], device="cuda")[:, None]
    dist = (-rel).clamp(min=0) if c["causal"] else rel.abs()
    side = (torch.arange(c["max_distance"] + 1, device="cuda")[:, None] >= s["edges"]).sum(1)
    bucket = side[dist.clamp(max=c["max_distance"])]
    return bucket if c["causal"] else bucket + (rel > 0) * (c["buckets"] // 2)


def _plain_forward(s):
    """(out, lse, weights [B, H, Sq, Sk]) in 32 bits."""
    c = s["case"]
    B, H, K, Sq, Sk = c["batch"], c["heads"], c["kv_heads"], c["q_len"], c["k_len"]
    k, v = _heads_first(s["k"], K), _heads_first(s["v"], K)
    x = (_heads_first(s["q"], K) @ k.transpose(2, 3)).view(B, H, Sq, Sk) * s["scale"]
    if c["buckets"]:
        x = x + s["table"][:, _buckets(s)]
    seen = (torch.arange(Sk, device="cuda") < s["k_lens"][:, None])[:, None, None, :]
    if c["causal"]:
        seen = seen & (torch.arange(Sk, device="cuda") <= torch.arange(Sq, device="cuda")[:, None])
    x = torch.where(seen, x, -math.inf)
    m = x.amax(3, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    total = e.sum(3, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    out = _rows_first(p.view(B, K, -1, Sk) @ v, H)
    return out, (m + torch.log(total))[..., 0], p


def _plain_attention_grad(s):
    c = s["case"]
    B, H, K, Sq, Sk = c["batch"], c["heads"], c["kv_heads"], c["q_len"], c["k_len"]
    out, _, p = _plain_forward(s)
    q, k, v, g = (_heads_first(s[n], K) for n in ("q", "k", "v", "dout"))
    dp = (g @ v.transpose(2, 3)).view(B, H, Sq, Sk)
    delta = (out * s["dout"].float()).sum(3).permute(0, 2, 1)
    ds = p * (dp - delta[..., None])
    shared = ds.view(B, K, -1, Sk)
    dt = s["q"].dtype
    grads = {"dq": _rows_first(shared @ k, H) * s["scale"], "dk": _rows_first(shared.transpose(2, 3) @ q, K) * s["scale"],
             "dv": _rows_first(p.view(B, K, -1, Sk).transpose(2, 3) @ g, K)}
    grads = {n: x.to(dt) for n, x in grads.items()}
    if c["buckets"]:
        grads["dbias"] = _bucket_sums(ds.sum(0), _buckets(s), c["buckets"])
    return grads


def _bucket_sums(x, bucket, n):
    """Sums of x [H, Sq, Sk] over the pairs of each bucket, in 64 bits: [H, n]."""
    H, Sq, Sk = x.shape
    # with the rows upside down and each one place longer than the next one's start, diagonals are columns
    x = torch.nn.functional.pad(x.flip(1), (0, Sq)).view(H, -1)[:, :Sq * (Sq + Sk - 1)]
    diagonals = x.view(H, Sq, Sq + Sk - 1).sum(1, dtype=torch.float64)
    of = torch.cat((bucket[:, 0].flip(0), bucket[0, 1:]))
    return torch.zeros(H, n, dtype=torch.float64, device="cuda").index_add_(1, of, diagonals).float()


def _plain_student(s):
    """(scaled logits, lse) of every row, in 32 bits."""
    c, x = s["case"], s["z"].float()
    if c["clip"] > 0:
        x = x.clamp(-c["clip"], c["clip"])
    x = x * c["scale"]
    m = x.amax(1, keepdim=True)
    return x, (m + torch.log(torch.exp(x - m).sum(1, keepdim=True)))[:, 0]


def _plain_teacher(s):
    """(probabilities [R, n], 0 where no token is named; what they leave of 1)."""
    c = s["case"]
    t = torch.where(s["ids"] >= 0, s["teacher"], -math.inf)
    m = t.amax(1, keepdim=True)
    e = torch.exp(t - torch.where(m == -math.inf, 0.0, m))
    if c["rest"]:
        q = torch.exp(t)
        return q, (1.0 - q.sum(1, dtype=torch.float64)).clamp(min=0).float()
    total = e.sum(1, keepdim=True)
    return e / torch.where(total == 0, 1.0, total), None


def _plain_distill(s):
    c, ids = s["case"], s["ids"]
    x, lse = _plain_student(s)
    q, left = _plain_teacher(s)
    named, at = ids >= 0, ids.clamp(min=0).long()
    logp = x.gather(1, at) - lse[:, None]
    loss = torch.where(named, q * (torch.log(torch.where(named, q, 1.0)) - logp), 0.0).sum(1)
    if not c["rest"]:
        return {"loss": loss, "lse": lse}
    away = torch.zeros_like(x).scatter_add_(1, at, named.float())
    x = torch.where(away > 0, -math.inf, x)
    m = x.amax(1, keepdim=True)
    rest = torch.where(m == -math.inf, -math.inf, m + torch.log(torch.exp(x - torch.where(m == -math.inf, 0.0, m)).sum(1, keepdim=True)))[:, 0]
    term = left * (torch.log(left) - (rest - lse))
    loss = loss + torch.where((left > 0) & (rest > -math.inf) & named.any(1), term, 0.0)
    return {"loss": loss, "lse": lse, "rest_lse": rest}


def _plain_distill_grad(s):
    c, ids = s["case"], s["ids"]
    x, _ = _plain_student(s)
    q, left = _plain_teacher(s)
    named, at = ids >= 0, ids.clamp(min=0).long()
    p = torch.exp(x - s["lse"][:, None])
    target = torch.zeros_like(x).scatter_add_(1, at, torch.where(named, q, 0.0))
    if c["rest"]:
        away = torch.zeros_like(x).scatter_add_(1, at, named.float())
        target = torch.where(away > 0, target, torch.exp(x - s["rest_lse"][:, None]) * left[:, None])
    d = (p - target) * (s["dloss"] * c["scale"])[:, None]
    d = torch.where(named.any(1)[:, None], d, 0.0)
    if c["clip"] > 0:
        d = torch.where(s["z"].float().abs() <= c["clip"], d, 0.0)
    return d.to(s["z"].dtype)


# ---------------------------------------------------------------------- run
def run(state):
    s = state
    c = s["case"]
    if not own:
        if c["op"] == "distill":
            return _plain_distill_grad(s) if c["grad"] else _plain_distill(s)
        if c["grad"]:
            return _plain_attention_grad(s)
        out, lse, _ = _plain_forward(s)
        return {"out": out.to(s["q"].dtype), "lse": lse}
    from paper_1811_06965_amd import ops
    if c["op"] == "distill":
        kw = dict(scale=c["scale"], clip=c["clip"], rest=c["rest"])
        if c["grad"]:
            return ops.distill_backward(s["z"], s["ids"], s["teacher"], s["lse"], s["dloss"], rest_lse=s["rest_lse"], **kw)
        r = ops.distill(s["z"], s["ids"], s["teacher"], **kw)
        return {"loss": r.loss, "lse": r.lse, **({"rest_lse": r.rest_lse} if c["rest"] else {})}
    kw = dict(k_lens=s["k_lens"], causal=c["causal"], scale=s["scale"])
    if c["buckets"]:
        if "bias" not in s:  # a layer's bias, made once
            s["bias"] = ops.RelativeBias(s["table"], c["max_distance"], bidirectional=not c["causal"])
        kw["bias"] = s["bias"]
    if c["grad"]:
        r = ops.attention_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], **kw)
        return {"dq": r.dq, "dk": r.dk, "dv": r.dv, **({"dbias": r.dbias} if c["buckets"] else {})}
    r = ops.attention(s["q"], s["k"], s["v"], **kw)
    return {"out": r.out, "lse": r.lse}


# -------------------------------------------------------------------- exact
def exact(case, seed):
    """The outputs from the definitions, in 64 bits."""
    c, s = case, prepare(case, seed)
    if c["op"] == "distill":
        return _exact_distill(c, s)
    B, H, K = c["batch"], c["heads"], c["kv_heads"]
    bias = None
    if c["buckets"]:
        bias = torch.nn.Parameter(s["table"].double())
        i, j = torch.arange(c["q_len"], device="cuda")[:, None], torch.arange(c["k_len"], device="cuda")[None, :]
        one = c["buckets"] if c["causal"] else c["buckets"] // 2
        where = torch.bucketize((j - i).abs(), s["edges"], right=True)
        where = torch.where(j > i, 0 if c["causal"] else one + where, where)
    lens = s["k_lens"].tolist()
    parts = {n: [] for n in (("dq", "dk", "dv") if c["grad"] else ("out", "lse"))}
    for b in range(B):
        n = lens[b]
        rows = {name: [] for name in parts}
        for h in range(K):  # one key head and the query heads that share it
            hs = slice(h * H // K, (h + 1) * H // K)
            q = s["q"][b, :, hs].double().transpose(0, 1).contiguous().requires_grad_(c["grad"])
            k = s["k"][b, :, h].double().contiguous().requires_grad_(c["grad"])
            v = s["v"][b, :, h].double().contiguous().requires_grad_(c["grad"])
            with torch.set_grad_enabled(c["grad"]):
                if n:
                    a = torch.matmul(q, k[:n].t()) * s["scale"]
                    if bias is not None:
                        a = a + bias[hs][:, where[:, :n]]
                    if c["causal"]:
                        a = a.masked_fill((j > i)[:, :n], -math.inf)
                    lse = torch.logsumexp(a, 2)
                    o = torch.matmul(torch.softmax(a, 2), v[:n])
                else:
                    o, lse = q * 0.0, q.sum(2) * 0.0 - math.inf
            if c["grad"]:
                if n:
                    o.backward(s["dout"][b, :, hs].double().transpose(0, 1))
                for name, x in (("dq", q), ("dk", k), ("dv", v)):
                    d = torch.zeros_like(x) if x.grad is None else x.grad
                    rows[name].append(d.transpose(0, 1) if name == "dq" else d[:, None])
            else:
                rows["out"].append(o.transpose(0, 1))
                rows["lse"].append(lse)
        for name in parts:
            parts[name].append(torch.cat(rows[name], 0 if name == "lse" else 1))
    res = {name: torch.stack(x) for name, x in parts.items()}
    if c["grad"] and bias is not None:
        res["dbias"] = bias.grad
    return res


def _exact_distill(c, s):
    parts = []
    step = max(1, (1 << 26) // c["vocab"])
    for r in range(0, c["rows"], step):
        z = s["z"][r:r + step].double().contiguous().requires_grad_(c["grad"])
        ids, t = s["ids"][r:r + step].long(), s["teacher"][r:r + step].double()
        named = ids >= 0
        some = named.any(1)
        t = t.masked_fill(~named, -math.inf)
        q = torch.exp(t) if c["rest"] else torch.softmax(t, 1).nan_to_num(0.0)
        inside = torch.zeros(z.shape, dtype=torch.bool, device="cuda")
        row, col = named.nonzero(as_tuple=True)
        inside[row, ids[row, col]] = True
        with torch.set_grad_enabled(c["grad"]):
            x = (z.clamp(-c["clip"], c["clip"]) if c["clip"] > 0 else z) * c["scale"]
            lse = torch.logsumexp(x, 1)
            logp = torch.gather(x - lse[:, None], 1, ids.clamp(min=0))
            loss = (torch.special.xlogy(q, q) - torch.where(named, q * logp, 0.0)).sum(1)
            if c["rest"]:
                rest = torch.logsumexp(x.masked_fill(inside, -math.inf), 1)
                left = (1.0 - q.sum(1)).clamp(min=0)
                extra = torch.special.xlogy(left, left) - left * (rest - lse)
                loss = loss + torch.where(some & (rest > -math.inf), extra, 0.0)
        if c["grad"]:
            (loss * some * s["dloss"][r:r + step].double()).sum().backward()
            parts.append(z.grad)
        else:
            parts.append({"loss": loss * some, "lse": lse, **({"rest_lse": rest} if c["rest"] else {})})
    if c["grad"]:
        return torch.cat(parts)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
