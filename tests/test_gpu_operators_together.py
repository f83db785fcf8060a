"""The operators as they are used together: a decoder layer with its own relative bias and attention to encoder states,
trained on a teacher's tokens, and the same attention one token at a time."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.attention_reference import attention as formulas, buckets_of, check, visible  # noqa: E402


@pytest.fixture(scope="module")
def ops():
    from paper_1811_06965_amd import ops as o
    return o


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_one_by_one(ops, dtype):
    """Each token's step over the keys so far gives the row that the whole sequence gives, within both bounds."""
    g = torch.Generator(device="cuda").manual_seed(1)
    B, S, H, K, dh = 3, 45, 4, 2, 64
    q = torch.randn(B, S, H, dh, generator=g, device="cuda").to(dtype)
    kv = torch.randn(B, S, 2, K, dh, generator=g, device="cuda").to(dtype)
    k, v = kv[:, :, 0], kv[:, :, 1]
    table = torch.randn(H, 16, generator=g, device="cuda")
    bias = ops.RelativeBias(table, 30, bidirectional=False)
    lens = torch.tensor([45, 20, 1], dtype=torch.int32, device="cuda")
    ok, dist = visible(B, S, S, q_lens=lens, k_lens=lens, causal=True)
    ref = formulas(q, k, v, dh ** -0.5, ok, table, buckets_of(16, 30, False), dist)
    whole = ops.attention(q, k, v, q_lens=lens, k_lens=lens, causal=True, bias=bias)
    check("out", whole.out, ref)
    outs, lses = [], []
    for i in range(S):
        at = torch.full((B,), i, dtype=torch.int32, device="cuda")
        r = ops.attention(q[:, i:i + 1], k, v, q_lens=(lens > i).int(), k_lens=torch.minimum(lens, at + 1), q_starts=at, bias=bias)
        outs.append(r.out)
        lses.append(r.lse)
    check("out", torch.cat(outs, 1), ref)
    check("lse", torch.cat(lses, 2), ref)


def functions(ops):
    class Attend(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, table, bias, kw):
            r = ops.attention(q, k, v, bias=bias, **kw)
            ctx.save_for_backward(q, k, v, r.out, r.lse)
            ctx.bias, ctx.kw = bias, kw
            return r.out

        @staticmethod
        def backward(ctx, dout):
            q, k, v, out, lse = ctx.saved_tensors
            g = ops.attention_backward(q, k, v, out, lse, dout.contiguous(), bias=ctx.bias, **ctx.kw)
            return g.dq, g.dk, g.dv, g.dbias, None, None

    class Distill(torch.autograd.Function):
        @staticmethod
        def forward(ctx, z, ids, teacher):
            r = ops.distill(z, ids, teacher)
            ctx.save_for_backward(z, ids, teacher, r.lse, r.rest_lse)
            return r.loss

        @staticmethod
        def backward(ctx, dloss):
            z, ids, teacher, lse, rest_lse = ctx.saved_tensors
            return ops.distill_backward(z, ids, teacher, lse, dloss.contiguous(), rest_lse=rest_lse), None, None

    return Attend.apply, Distill.apply


def test_a_decoder_layer_with_a_teacher(ops):
    """Gradients of every weight, fp32, against autograd of the formulas in 64 bits.  A sum of n <= 192 products is off by
    193 u = 1.2e-5 of its absolute sum, which is about sqrt(192) = 14 times its value; ten such products lie on the way to a
    weight's gradient and back: 10 x 14 x 1.2e-5 = 1.7e-3 of its largest value."""
    B, S, M, D, H, K, V, top = 3, 33, 50, 64, 4, 2, 192, 8
    dh = D // H
    g = torch.Generator(device="cuda").manual_seed(2)

    def rn(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * scale

    x, mem, teacher_logits = rn(B, S, D), rn(B, M, D), rn(B * S, V, scale=2.0)
    lens = torch.tensor([50, 31, 0], dtype=torch.int32, device="cuda")
    weight = torch.rand(B * S, generator=g, device="cuda") / S
    weight[-5:] = 0
    sizes = dict(qkv=(D, 3 * D), o=(D, D), q2=(D, D), kv=(D, 2 * K * dh), o2=(D, D), head=(D, V))
    start = {n: rn(*s, scale=s[0] ** -0.5) for n, s in sizes.items()}
    start["table"] = rn(H, 8)
    a = ops.token_logprobs(teacher_logits, top=top)
    attend, distill = functions(ops)

    def layer(p, x, mem, attention, loss):
        qkv = (x @ p["qkv"]).view(B, S, 3, H, dh)
        y = x + attention(qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2], True).reshape(B, S, D) @ p["o"]
        kv = (mem @ p["kv"]).view(B, M, 2, K, dh)
        y = y + attention((y @ p["q2"]).view(B, S, H, dh), kv[:, :, 0], kv[:, :, 1], False).reshape(B, S, D) @ p["o2"]
        return (loss((y @ p["head"]).view(B * S, V)) * weight.to(x.dtype)).sum()

    p = {n: t.clone().requires_grad_() for n, t in start.items()}
    bias = ops.RelativeBias(p["table"], 20, bidirectional=False)
    none = torch.zeros(0, device="cuda")

    def mine(q, k, v, own):
        if own:
            return attend(q, k, v, p["table"], bias, dict(causal=True))
        return attend(q, k, v, none, None, dict(k_lens=lens))

    total = layer(p, x, mem, mine, lambda z: distill(z, a.top_ids, a.top_logp))
    total.backward()

    e = {n: t.double().requires_grad_() for n, t in start.items()}
    of = torch.tensor(buckets_of(8, 20, False), device="cuda")

    def exact(q, k, v, own):
        k, v = (t.repeat_interleave(H // t.shape[2], 2) for t in (k, v))
        s = torch.matmul(q.transpose(1, 2), k.permute(0, 2, 3, 1)) * dh ** -0.5
        ok, dist = visible(B, S, k.shape[1], k_lens=None if own else lens, causal=own)
        if own:
            s = s + e["table"][:, of[dist[0].clamp(-20, 20) + 20]]
        # a sequence without keys: its scores are masked to one value, and what comes out is thrown away
        empty = ~ok.any(2)[:, None, :, None]
        w = torch.softmax(s.masked_fill(~ok[:, None], -1e300), 3)
        return torch.matmul(w.masked_fill(empty, 0.0), v.transpose(1, 2)).transpose(1, 2)

    def exact_loss(z):
        logp = torch.log_softmax(z, 1)
        q = torch.exp(a.top_logp.double())
        inside = torch.zeros_like(z, dtype=torch.bool).scatter_(1, a.top_ids.long(), True)
        rest = 1 - q.sum(1)
        away = torch.logsumexp(logp.masked_fill(inside, -math.inf), 1)
        return (q * (torch.log(q) - logp.gather(1, a.top_ids.long()))).sum(1) + rest * (torch.log(rest) - away)

    want = layer(e, x.double(), mem.double(), exact, exact_loss)
    want.backward()
    total, want = float(total.detach()), float(want.detach())
    assert abs(total - want) <= 1.7e-3 * abs(want)
    for n in start:
        d, r = p[n].grad.double(), e[n].grad
        assert (d - r).abs().max() <= 1.7e-3 * r.abs().max(), (n, float((d - r).abs().max() / r.abs().max()))

    # and the update with them
    params = [t.detach() for t in p.values()]
    grads = [t.grad for t in p.values()]
    factor = ops.grad_norm(grads, 1.0)
    ops.AdamW(params, grads, lr=1e-3).step(factor=factor[1:])
    for t, n in zip(params, start):
        assert t.isfinite().all() and not torch.equal(t, start[n])
    again = ops.attention(x.view(B, S, H, dh), x.view(B, S, H, dh), x.view(B, S, H, dh).clone(), causal=True,
                          bias=ops.RelativeBias(p["table"].detach(), 20, bidirectional=False))
    with torch.no_grad():  # the table is read at every call: the updated one
        other = ops.attention(x.view(B, S, H, dh), x.view(B, S, H, dh), x.view(B, S, H, dh).clone(), causal=True, bias=bias)
    assert torch.equal(again.out, other.out)
