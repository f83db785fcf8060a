"""A partition that updates with AdamW (and clips its gradient's norm), and one
that scores sequences under its vocabulary head, through the C ABI.

Tolerances as in test_gpu_parity (fp32 1e-4 of the largest value; bf16 2e-2), the
update against the same fp32 operations on the host, and bit for bit where two
schedules do the same work.
"""
import math

import numpy as np
import pytest

import synth
from parity import rel_err

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TINY = synth.CONFIGS["tiny"]
ADAMW = dict(optimizer="adamw", weight_decay=0.1)
ENC = synth.CONFIGS["enc512"].with_(name="enc512_small", layers=2, batch=8, micro=4)
DEC_F32 = synth.PartitionConfig("dec_f32", layers=2, d_model=32, d_ff=64, heads=2, seq=8, batch=4, micro=2,
                                dtype="f32", kind="decoder", loss="xent_ls", vocab=40, label_smoothing=0.1, mem_seq=6)
DEC_BF16 = synth.PartitionConfig("dec_bf16", layers=2, d_model=128, d_ff=256, heads=2, seq=64, batch=4, micro=2,
                                 dtype="bf16", kind="decoder", loss="xent_ls", vocab=1000, label_smoothing=0.1,
                                 mem_seq=32)


def tensors(pair):
    return [(k, v) for d in list(pair[0]) + [pair[1]] for k, v in d.items()]


@pytest.mark.parametrize("clip", [0.0, 0.05, 1e6])
@pytest.mark.parametrize("cfg", [TINY, DEC_F32], ids=lambda c: c.name)
def test_steps_match_oracle(cfg, clip):
    """Three fp32 steps against the oracle: the loss before each, and the parameters after.  Where a gradient element is
    near zero the ratio m / sqrt(v) has its sign and size from round-off, so elements are compared whose gradient stays
    over 1e-3 of their tensor's largest in every step: 2e-2 of the step taken."""
    from oracle import gpipe
    from paper_1811_06965_amd.runtime import Partition
    cfg = cfg.with_(**ADAMW, max_grad_norm=clip)
    case = synth.make_case(cfg, 31, perturb=True)
    lr = 1e-3
    with Partition(cfg) as part:
        part.load_params(case["layers"], case["head"])
        inp = part.device_inputs(case)
        ref, state, solid = dict(case), None, None
        for _ in range(3):
            r = gpipe.gpipe_step(cfg, ref, cfg.micro, lr=lr, opt_state=state)
            out = part.step(inp["x"], inp["mem"], inp["dy"], lr=lr)
            assert abs(out["loss"] - r["loss"]) <= 1e-4 * abs(r["loss"])
            g = tensors((r["grads"], {k: r["head_grads"][k] for k in ref["head"]}))
            if clip:
                norm = math.sqrt(sum(float((v ** 2).sum()) for _, v in g))
                assert abs(part.grad_norm() / norm - 1) <= 1e-4
            big = [np.abs(v) > 1e-3 * np.abs(v).max() for _, v in g]
            solid = big if solid is None else [a & b for a, b in zip(solid, big)]
            ref = dict(ref, layers=r["layers"], head=r["head"])
            state = r["opt_state"]
        got = tensors(part.params())
    begin = tensors((case["layers"], case["head"]))
    for (k, a), (_, b), (_, w), ok in zip(got, tensors((ref["layers"], ref["head"])), begin, solid):
        if k in ("bk", "xbk"):  # their gradients are zero, round-off altogether
            continue
        assert np.abs(b - w).max() > 1e-4, k
        err = np.abs(a - b)[ok] - 4e-7 * np.abs(b)[ok]
        assert (err <= 2e-2 * np.maximum(np.abs(b - w)[ok], 1e-3 * 0.1)).all(), (k, err.max())


@pytest.mark.parametrize("clip", [0.0, 0.02])
@pytest.mark.parametrize("cfg", [ENC, DEC_BF16, TINY], ids=lambda c: c.name)
def test_update_applies_the_accumulated_gradient(cfg, clip):
    """Every parameter moves by the AdamW step of its accumulated gradient, two steps in a row: fp32 on the host in the
    same order, the bias corrections in 64 bits (the device's are within 4 u): the step within 2^-20 of it, and
    three roundings of the parameter."""
    from paper_1811_06965_amd.runtime import Partition
    cfg = cfg.with_(**ADAMW, max_grad_norm=clip)
    case = synth.make_case(cfg, 26, perturb=True)
    f, lr = np.float32, 1e-3
    with Partition(cfg) as part:
        part.load_params(case["layers"], case["head"])
        inp = part.device_inputs(case)
        m = v = None
        for t in (1, 2):
            w0 = tensors(part.params())
            part.step(inp["x"], inp["mem"], inp["dy"], lr=lr, want_y=False)
            torch.cuda.synchronize()
            g, w1 = tensors(part.grads()), tensors(part.params())
            if m is None:
                m, v = [np.zeros_like(x) for _, x in g], [np.zeros_like(x) for _, x in g]
            factor = f(1)
            if clip:
                norm = math.sqrt(sum(float((x.astype(np.float64) ** 2).sum()) for _, x in g))
                assert abs(part.grad_norm() / norm - 1) < 1e-6
                factor = f(min(1.0, clip / norm))
            for i, ((k, a), (_, gg), (_, b)) in enumerate(zip(w0, g, w1)):
                gg = gg * factor
                m[i] = m[i] * f(0.9) + gg * f(1 - float(f(0.9)))
                v[i] = v[i] * f(0.999) + gg * gg * f(1 - float(f(0.999)))
                decay = lr * 0.1 if k.lstrip("x").startswith("w") else 0.0
                b1, b2 = float(f(0.9)), float(f(0.999))
                den = np.sqrt(v[i]) * f(1 / math.sqrt(1 - b2 ** t)) + f(1e-8)
                step = f(lr / (1 - b1 ** t)) * m[i] / den
                want = a * f(1 - decay) - step
                tol = np.spacing(np.maximum(np.abs(want), np.abs(a))) * 3 + np.abs(step) * 2.0 ** -19
                assert (np.abs(b - want) <= tol).all(), (k, np.abs(b - want).max())


@pytest.mark.parametrize("cfg", [ENC, DEC_BF16], ids=lambda c: c.name)
def test_schedules_and_replays_change_no_bit(cfg, monkeypatch):
    """Three steps: each layer's update as soon as the last backward is past it, the whole update at the end, one
    stream, and a captured step replayed (the counter is on the device), with the program's own work between."""
    from paper_1811_06965_amd.runtime import Partition
    cfg = cfg.with_(**ADAMW)
    case = synth.make_case(cfg, 33, perturb=True)
    res = {}
    for name in ("layer", "whole", "one stream", "graph"):
        monkeypatch.setenv("GP_LAYER_UPDATE", "1" if name == "layer" else "0")
        with Partition(cfg) as part:
            part.load_params(case["layers"], case["head"])
            inp = part.device_inputs(case)
            if name == "graph":
                stream = torch.cuda.Stream()
                stream.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(stream):
                    g = part.capture_step(inp["x"], inp["mem"], inp["dy"], lr=1e-3)
                for _ in range(3):
                    g.replay()
                    torch.zeros(100, device="cuda").sum()
                    torch.cuda.synchronize()
            else:
                k = 1 if name == "one stream" else 2
                for _ in range(3):
                    part.step(inp["x"], inp["mem"], inp["dy"], lr=1e-3, want_loss=False, fwd_streams=k, bwd_streams=k)
                torch.cuda.synchronize()
            res[name] = tensors(part.params())
            del inp
    for name in ("whole", "one stream", "graph"):
        for (k, a), (_, b) in zip(res["layer"], res[name]):
            assert np.array_equal(a, b), (name, k)


def test_clipped_step_replays():
    from paper_1811_06965_amd.runtime import Partition
    cfg = ENC.with_(**ADAMW, max_grad_norm=0.01)
    case = synth.make_case(cfg, 34, perturb=True)
    res = []
    for graph in (False, True):
        with Partition(cfg) as part:
            part.load_params(case["layers"], case["head"])
            inp = part.device_inputs(case)
            if graph:
                g = part.capture_step(inp["x"], inp["mem"], inp["dy"], lr=1e-3)
                for _ in range(3):
                    g.replay()
                    torch.cuda.synchronize()
            else:
                for _ in range(3):
                    part.step(inp["x"], inp["mem"], inp["dy"], lr=1e-3)
            res.append((part.grad_norm(), tensors(part.params())))
    assert res[0][0] == res[1][0] > 0.01
    for (k, a), (_, b) in zip(res[0][1], res[1][1]):
        assert np.array_equal(a, b), k


def test_poison_changes_no_bit(monkeypatch):
    """NaN in every workspace region before the phase that rewrites it (padding between parameter blocks included):
    the clipped update and the scores stay the same."""
    from paper_1811_06965_amd.runtime import Partition
    cfg = DEC_BF16.with_(**ADAMW, max_grad_norm=0.01)
    case = synth.make_case(cfg, 35, perturb=True)
    res = []
    for poison in ("0", "1"):
        monkeypatch.setenv("GP_POISON", poison)
        with Partition(cfg) as part:
            part.load_params(case["layers"], case["head"])
            inp = part.device_inputs(case)
            half = cfg.batch // cfg.micro
            for _ in range(2):
                part.step(inp["x"], inp["mem"], inp["dy"], lr=1e-3)
            r = part.score(inp["x"][:half], inp["dy"][:half], inp["mem"][:half], top=5)
            res.append((part.grad_norm(), tensors(part.params()), [t.cpu() for t in r]))
    assert res[0][0] == res[1][0]
    assert all(np.array_equal(a, b) for (_, a), (_, b) in zip(res[0][1], res[1][1]))
    assert all(torch.equal(a, b) for a, b in zip(res[0][2], res[1][2]))


def test_a_norm_that_is_not_finite_skips_the_update():
    from paper_1811_06965_amd import gp
    from paper_1811_06965_amd.runtime import Partition
    cfg = TINY.with_(**ADAMW, max_grad_norm=1.0)
    case = synth.make_case(cfg, 36, perturb=True)
    with Partition(cfg) as part:
        part.load_params(case["layers"], case["head"])
        inp = part.device_inputs(case)
        bad = inp["x"].clone()
        bad[0, 0, 0] = math.nan
        before = tensors(part.params())
        with pytest.raises(gp.GpError) as err:
            part.step(bad, None, inp["dy"], lr=1e-3)
        assert err.value.status == gp.GP_ERR_NONFINITE and not math.isfinite(part.grad_norm())
        part.step(bad, None, inp["dy"], lr=1e-3, want_loss=False)  # skipped on the device alone
        assert all(np.array_equal(a, b) for (_, a), (_, b) in zip(before, tensors(part.params())))
        part.step(inp["x"], None, inp["dy"], lr=1e-3)
        first = tensors(part.params())
    with Partition(cfg) as part:  # the skipped ones were not counted
        part.load_params(case["layers"], case["head"])
        inp = part.device_inputs(case)
        part.step(inp["x"], None, inp["dy"], lr=1e-3)
        assert all(np.array_equal(a, b) for (_, a), (_, b) in zip(first, tensors(part.params())))


def test_memory_and_refusals():
    from paper_1811_06965_amd import gp
    from paper_1811_06965_amd.runtime import Partition
    with Partition(TINY.with_(**ADAMW)) as a, Partition(TINY) as s:
        # masters, gradients and two moments: 16 bytes per parameter
        assert a.memory()["params"] - s.memory()["params"] == 2 * a.memory()["grads"]
        with pytest.raises(gp.GpError) as err:
            a.grad_norm()
        assert err.value.status == gp.GP_ERR_STATE
        with pytest.raises(gp.GpError) as err:
            a.score(torch.zeros(2, 32, 64, device="cuda"))
        assert err.value.status == gp.GP_ERR_UNSUPPORTED
        case = synth.make_case(TINY, 1)
        a.load_params(case["layers"], case["head"])
        inp = a.device_inputs(case)
        for lr in (-1.0, math.nan, 11.0):
            with pytest.raises(gp.GpError) as err:
                a.step(inp["x"], None, inp["dy"], lr=lr)
            assert err.value.status == gp.GP_ERR_INVALID_ARG
            gp.gp_accumulate_and_step(a.h, 0.0, False, torch.cuda.current_stream().cuda_stream)  # the step is still owed


@pytest.mark.parametrize("cfg", [TINY.with_(**ADAMW), ENC.with_(**ADAMW, max_grad_norm=0.05),
                                 DEC_BF16.with_(optimizer="rmsprop", rms_eps=1e-8)], ids=["tiny", "enc", "rmsprop"])
def test_resume_with_the_optimizer_state(cfg):
    """Two steps, everything read, a new partition that takes it, two more: the bits of four steps in one."""
    from paper_1811_06965_amd import gp
    from paper_1811_06965_amd.runtime import Partition
    case = synth.make_case(cfg, 38, perturb=True)
    with Partition(cfg) as part:
        part.load_params(case["layers"], case["head"])
        inp = part.device_inputs(case)
        for k in range(4):
            if k == 2:
                mid, state = part.params(), part.optimizer_state()
            part.step(inp["x"], inp["mem"], inp["dy"], lr=1e-3)
        want, end = tensors(part.params()), part.optimizer_state()
    with Partition(cfg) as part:
        part.load_params(*mid)
        part.load_optimizer_state(state)
        inp = part.device_inputs(case)
        for _ in range(2):
            part.step(inp["x"], inp["mem"], inp["dy"], lr=1e-3)
        assert all(np.array_equal(a, b) for (_, a), (_, b) in zip(want, tensors(part.params())))
        got = part.optimizer_state()
        assert got[0] == end[0] == (4 if cfg.optimizer == "adamw" else 0)
        for a, b in zip(end[1:], got[1:]):
            assert (a is None and b is None) or all(np.array_equal(x, y) for (_, x), (_, y) in zip(tensors(a), tensors(b)))
        assert max(np.abs(x).max() for _, x in tensors(got[2])) > 0
        host = np.zeros(3, dtype=np.float32)
        bad = [lambda: gp.gp_get_moment(part.h, 0, gp.PARAM_ID["bq"], 2, host), lambda: gp.gp_set_updates(part.h, -1),
               lambda: gp.gp_get_moment(part.h, 0, gp.PARAM_ID["bq"], 3, host),
               lambda: gp.gp_set_moment(part.h, 99, 0, 2, host)]
        if cfg.optimizer == "rmsprop":
            bad += [lambda: gp.gp_get_updates(part.h), lambda: gp.gp_get_moment(part.h, 0, 0, 1, host)]
        for f in bad:
            with pytest.raises(gp.GpError) as err:
                f()
            assert err.value.status == gp.GP_ERR_INVALID_ARG


# -------------------------------------------------------------------- scoring
def oracle_scores(cfg, case, sl):
    from oracle import gpipe, transformer as tf
    y, _ = gpipe.partition_forward(cfg, case["layers"], case["x"][sl], None if case["mem"] is None else case["mem"][sl])
    h, _ = tf.layer_norm(y, case["head"]["lnf_g"], case["head"]["lnf_b"], cfg.ln_eps)
    z = tf.linear(h, case["head"]["wout"], case["head"]["bout"]).reshape(-1, cfg.vocab)
    if cfg.logit_clip > 0:
        z = np.clip(z, -cfg.logit_clip, cfg.logit_clip)
    m = z.max(1, keepdims=True)
    lse = (m + np.log(np.exp(z - m).sum(1, keepdims=True)))[:, 0]
    logp = z - lse[:, None]
    return z, lse, logp, -(np.exp(logp) * logp).sum(1)


@pytest.mark.parametrize("clip", [0.0, 0.5])
@pytest.mark.parametrize("cfg", [DEC_F32, DEC_BF16, DEC_BF16.with_(name="one", batch=2, micro=1)], ids=lambda c: c.name)
def test_scores_match_oracle(cfg, clip):
    from paper_1811_06965_amd.runtime import Partition
    cfg = cfg.with_(logit_clip=clip)
    case = synth.make_case(cfg, 41, perturb=True)
    case["head"] = dict(case["head"], wout=synth.round_storage(4.0 * case["head"]["wout"], cfg.dtype))
    n = cfg.batch // cfg.micro
    tol = 1e-4 if cfg.dtype == "f32" else 2e-2
    with Partition(cfg) as part:
        part.load_params(case["layers"], case["head"])
        inp = part.device_inputs(case)
        for a in range(0, cfg.batch, n):
            sl = slice(a, a + n)
            z, lse, logp, h = oracle_scores(cfg, case, sl)
            tok = inp["dy"][sl].clone()
            tok[0, 1] = -1
            r = part.score(inp["x"][sl].contiguous(), tok, inp["mem"][sl].contiguous(), top=4)
            big = np.abs(logp).max()
            d = lambda t: t.double().cpu().numpy()  # noqa: E731
            t = tok.cpu().numpy().ravel()
            want = np.where(t < 0, 0.0, logp[np.arange(len(t)), np.maximum(t, 0)])
            assert np.abs(d(r.logp) - want).max() <= tol * big
            assert np.abs(d(r.lse) - lse).max() <= tol * big and np.abs(d(r.entropy) - h).max() <= tol * big
            ids = r.top_ids.cpu().numpy()
            assert np.abs(d(r.top_logp) - np.take_along_axis(logp, ids, 1)).max() <= tol * big
            best = -np.sort(-logp, 1)[:, :4]
            assert np.abs(np.take_along_axis(logp, ids, 1) - best).max() <= 2 * tol * big
        none = part.score(inp["x"][sl].contiguous(), None, inp["mem"][sl].contiguous(), scale=2.0)
        assert none.logp is None and none.top_ids is None


def test_scoring_between_steps_changes_nothing():
    """Scores on another stream between mini-batches, and of the first one again after training steps on two
    streams: the training's bits are those without scoring, and a score follows the last update."""
    from paper_1811_06965_amd.runtime import Partition
    cfg = DEC_BF16.with_(**ADAMW)
    case = synth.make_case(cfg, 43, perturb=True)
    n = cfg.batch // cfg.micro
    res = []
    for scoring in (False, True):
        with Partition(cfg) as part:
            part.load_params(case["layers"], case["head"])
            inp = part.device_inputs(case)
            x, tok, mem = (inp[k][:n].contiguous() for k in ("x", "dy", "mem"))
            side, scores = torch.cuda.Stream(), []
            side.wait_stream(torch.cuda.current_stream())
            for _ in range(3):
                if scoring:
                    with torch.cuda.stream(side):
                        scores.append(part.score(x, tok, mem, top=3))
                part.step(inp["x"], inp["mem"], inp["dy"], lr=1e-2, want_loss=False)
            torch.cuda.synchronize()
            res.append(tensors(part.params()))
            if scoring:
                means = [float(s.logp.mean()) for s in scores] + [float(part.score(x, tok, mem).logp.mean())]
                assert len(set(means)) == 4  # each after another update
                with Partition(cfg) as fresh:
                    fresh.load_params(case["layers"], case["head"])
                    again = fresh.score(x, tok, mem, top=3)
                    assert all(torch.equal(a, b) for a, b in zip(again, scores[0]))
    assert all(np.array_equal(a, b) for (_, a), (_, b) in zip(*res))


def test_scoring_is_refused_inside_a_mini_batch():
    from paper_1811_06965_amd import gp
    from paper_1811_06965_amd.runtime import Partition
    case = synth.make_case(DEC_F32, 44)
    with Partition(DEC_F32) as part:
        part.load_params(case["layers"], case["head"])
        inp = part.device_inputs(case)
        x, tok, mem = (inp[k][:2].contiguous() for k in ("x", "dy", "mem"))
        st = torch.cuda.current_stream().cuda_stream
        gp.gp_forward_microbatch(part.h, 0, x.data_ptr(), mem.data_ptr(), None, st)
        with pytest.raises(gp.GpError) as err:
            part.score(x, tok, mem)
        assert err.value.status == gp.GP_ERR_STATE
        for bad in (dict(top=41), dict(top=-1), dict(scale=0.0)):
            with pytest.raises((gp.GpError, ValueError, RuntimeError)):
                part.score(x, tok, mem, **bad)
        torch.cuda.synchronize()


# ------------------------------------------------------------- token weights
def oracle_weighted_step(cfg, case, tok, a, b):
    """Loss, dx and gradients of sum a logp + b H over a mini-batch in one pass (float64), the head's gradient through
    the oracle's own layers."""
    from oracle import gpipe, transformer as tf
    y, caches = gpipe.partition_forward(cfg, case["layers"], case["x"], case["mem"])
    hd = case["head"]
    h, ln = tf.layer_norm(y, hd["lnf_g"], hd["lnf_b"], cfg.ln_eps)
    raw = tf.linear(h, hd["wout"], hd["bout"])
    z = np.clip(raw, -cfg.logit_clip, cfg.logit_clip) if cfg.logit_clip > 0 else raw
    m = z.max(-1, keepdims=True)
    logp = z - m - np.log(np.exp(z - m).sum(-1, keepdims=True))
    p = np.exp(logp)
    H = -(p * logp).sum(-1, keepdims=True)
    one = (np.arange(cfg.vocab) == tok[..., None]).astype(float)
    aa = np.where(tok < 0, 0.0, a)[..., None]
    dz = aa * (one - p) - b[..., None] * p * (logp + H)
    if cfg.logit_clip > 0:
        dz = dz * (np.abs(raw) <= cfg.logit_clip)
    loss = float((aa * (one * logp).sum(-1, keepdims=True)).sum() + (b[..., None] * H).sum())
    g = {"wout": np.einsum("nsd,nsv->dv", h, dz), "bout": dz.sum((0, 1))}
    dh = dz @ hd["wout"].T
    dy, dg, db = tf.layer_norm_backward(dh, ln, hd["lnf_g"])
    g["lnf_g"], g["lnf_b"] = dg, db
    dx, dmem, gl = gpipe.partition_backward(cfg, case["layers"], caches, dy)
    return loss, dx, gl, g


@pytest.mark.parametrize("clip", [0.0, 0.7])
@pytest.mark.parametrize("cfg", [DEC_F32, DEC_BF16, DEC_BF16.with_(name="m4", batch=8, micro=4)], ids=lambda c: c.name)
def test_weighted_tokens_match_oracle(cfg, clip):
    """A policy-like objective (weights of both signs, padding, an entropy bonus): loss, input gradient and every
    parameter gradient against the oracle, and the same bits on one stream and on two."""
    from parity import compare_grads, cosine, to_np
    from paper_1811_06965_amd.runtime import Partition
    cfg = cfg.with_(logit_clip=clip)
    case = synth.make_case(cfg, 51, perturb=True)
    case["head"] = dict(case["head"], wout=synth.round_storage(4.0 * case["head"]["wout"], cfg.dtype))
    rng = np.random.default_rng(3)
    tok = np.array(case["labels"])
    tok[rng.random(tok.shape) < 0.2] = -1
    a = (rng.standard_normal(tok.shape) / tok.size).astype(np.float32)
    b = (-0.1 * rng.random(tok.shape) / tok.size).astype(np.float32)
    loss, dx, gl, gh = oracle_weighted_step(cfg, case, tok, a.astype(float), b.astype(float))
    t = lambda v, k: torch.tensor(v, dtype=k, device="cuda")  # noqa: E731
    res = []
    for streams in (1, 2):
        with Partition(cfg) as part:
            part.load_params(case["layers"], case["head"])
            inp = part.device_inputs(case)
            out = part.step(inp["x"], inp["mem"], t(tok, torch.int32), lr=0.0, dlogp=t(a, torch.float32),
                            dentropy=t(b, torch.float32), fwd_streams=streams, bwd_streams=streams)
            torch.cuda.synchronize()
            res.append((out["loss"], out["dx"], part.grads()))
    (l1, d1, g1), (l2, d2, g2) = res
    assert l1 == l2 and torch.equal(d1, d2)
    assert all(np.array_equal(u, v) for (_, u), (_, v) in zip(tensors(g1), tensors(g2)))
    mode, tol = ("rel", 1e-4) if cfg.dtype == "f32" else ("cos", 0.999)
    # the loss adds and cancels terms of both signs: against the sum of their magnitudes
    size = np.abs(a).sum() * np.log(cfg.vocab) + np.abs(b).sum() * np.log(cfg.vocab)
    assert abs(l1 - loss) <= (1e-4 if mode == "rel" else 2e-2) * size
    assert (rel_err(to_np(d1), dx) <= tol) if mode == "rel" else (cosine(to_np(d1), dx) >= tol)
    compare_grads(*g1, gl, gh, mode, tol)


def test_weights_of_the_likelihood_are_the_cross_entropy():
    """dlogp = -1 / (N S) is the head's own loss without label smoothing: the same loss and gradients within fp32."""
    from parity import compare_grads
    from paper_1811_06965_amd import gp
    from paper_1811_06965_amd.runtime import Partition
    cfg = DEC_F32.with_(label_smoothing=0.0)
    case = synth.make_case(cfg, 52, perturb=True)
    res = []
    for weighted in (False, True):
        with Partition(cfg) as part:
            part.load_params(case["layers"], case["head"])
            inp = part.device_inputs(case)
            kw = dict(dlogp=torch.full(inp["dy"].shape, -1.0 / inp["dy"].numel(), device="cuda")) if weighted else {}
            out = part.step(inp["x"], inp["mem"], inp["dy"], **kw)
            res.append((out["loss"], part.grads()))
            if weighted:
                with pytest.raises(ValueError):
                    part.step(inp["x"], inp["mem"], inp["dy"], dlogp=torch.zeros(3, device="cuda"))
    with Partition(TINY) as part:
        with pytest.raises(gp.GpError) as err:
            gp.gp_backward_microbatch_weighted(part.h, 0, 64, 64, None, None, None, None)
        assert err.value.status == gp.GP_ERR_UNSUPPORTED
    assert abs(res[0][0] - res[1][0]) <= 1e-5 * abs(res[0][0])
    compare_grads(*res[1][1], *res[0][1], "rel", 1e-4)


def test_a_weighted_step_replays():
    from paper_1811_06965_amd.runtime import Partition
    cfg = DEC_BF16.with_(**ADAMW, max_grad_norm=0.5)
    case = synth.make_case(cfg, 53, perturb=True)
    res = []
    for graph in (False, True):
        with Partition(cfg) as part:
            part.load_params(case["layers"], case["head"])
            inp = part.device_inputs(case)
            w = torch.linspace(-1, 1, inp["dy"].numel(), device="cuda").view(inp["dy"].shape) / 100
            kw = dict(dlogp=w, dentropy=w * 0.1)
            if graph:
                g = part.capture_step(inp["x"], inp["mem"], inp["dy"], lr=1e-3, **kw)
                for _ in range(3):
                    g.replay()
                    torch.cuda.synchronize()
            else:
                for _ in range(3):
                    part.step(inp["x"], inp["mem"], inp["dy"], lr=1e-3, want_loss=False, **kw)
            res.append(tensors(part.params()))
    assert all(np.array_equal(u, v) for (_, u), (_, v) in zip(*res))
