"""The AdamW fields of a partition's configuration, its memory plan and the
null-partition refusals, on the host; the oracle's AdamW against closed forms."""
import ctypes
import math
import os

import numpy as np
import pytest

import synth


@pytest.fixture(scope="module")
def gp():
    from paper_1811_06965_amd import build, gp as g
    if not os.path.exists(g.LIB_PATH):
        build.build()
    g.load()
    return g


CFG = synth.CONFIGS["tiny"].with_(optimizer="adamw", weight_decay=0.1, max_grad_norm=1.0)


def plan(gp, cfg, **fields):
    from paper_1811_06965_amd.runtime import make_config
    c = make_config(cfg)
    for k, v in fields.items():
        setattr(c, k, v)
    return gp.gp_memory_plan(cfg.layers, cfg.d_model, cfg.d_ff, cfg.heads, c)


@pytest.mark.parametrize("fields", [
    dict(adam_beta1=1.0), dict(adam_beta1=-0.1), dict(adam_beta1=math.nan), dict(adam_beta2=1.0),
    dict(adam_beta2=math.nan), dict(adam_eps=0.0), dict(adam_eps=math.inf), dict(weight_decay=-1.0),
    dict(weight_decay=math.inf), dict(max_grad_norm=-1.0), dict(max_grad_norm=math.nan), dict(rms_decay=0.9),
    dict(rms_eps=1e-8), dict(optimizer=3)])
def test_refused_fields(gp, fields):
    with pytest.raises(gp.GpError) as err:
        plan(gp, CFG, **fields)
    assert err.value.status == gp.GP_ERR_INVALID_ARG


@pytest.mark.parametrize("opt", ["sgd", "rmsprop"])
@pytest.mark.parametrize("field", ["adam_beta1", "adam_beta2", "adam_eps", "weight_decay", "max_grad_norm"])
def test_fields_of_adamw_alone(gp, opt, field):
    with pytest.raises(gp.GpError):
        plan(gp, synth.CONFIGS["tiny"].with_(optimizer=opt), **{field: 0.5})


def test_memory_plan(gp):
    sgd, adamw = plan(gp, synth.CONFIGS["tiny"]), plan(gp, CFG)
    assert adamw["params"] - sgd["params"] == 2 * sgd["grads"] and adamw["stash"] == sgd["stash"]
    assert 0 < plan(gp, CFG.with_(max_grad_norm=0.0))["workspace"] - sgd["workspace"] <= 512
    assert 0 < adamw["workspace"] - sgd["workspace"] <= 32768


def test_null_partitions(gp):
    f = ctypes.c_float()
    lib = gp.load()
    assert lib.gp_get_grad_norm(None, ctypes.byref(f)) == gp.GP_ERR_INVALID_ARG
    assert lib.gp_score_sequences(None, None, None, None, 1.0, None, None, None, 0, None, None, None) == 1
    h = gp.gp_partition_create(2, 64, 256, 4)
    assert lib.gp_get_grad_norm(h, None) == gp.GP_ERR_INVALID_ARG
    assert lib.gp_get_grad_norm(h, ctypes.byref(f)) == gp.GP_ERR_STATE
    assert lib.gp_score_sequences(h, None, None, None, 1.0, None, None, None, 0, None, None, None) == gp.GP_ERR_STATE
    back = lib.gp_backward_microbatch_weighted
    assert back(None, 0, None, None, None, None, None, None) == 1
    assert back(h, 0, 64, None, None, None, None, None) == 1  # neither weight
    assert back(h, 0, 64, 66, None, None, None, None) == 1    # misaligned
    assert back(h, 0, 64, 64, None, None, None, None) == gp.GP_ERR_STATE
    n = ctypes.c_longlong()
    host = (ctypes.c_float * 4)()
    for call in (lambda q: lib.gp_get_moment(q, 0, 0, 1, host, 4), lambda q: lib.gp_set_moment(q, 0, 0, 1, host, 4),
                 lambda q: lib.gp_get_updates(q, ctypes.byref(n)), lambda q: lib.gp_set_updates(q, 1)):
        assert call(None) == 1 and call(h) == gp.GP_ERR_STATE
    assert lib.gp_get_updates(h, None) == 1 and lib.gp_get_moment(h, 0, 0, 1, None, 4) == 1
    gp.gp_partition_destroy(h)


def test_oracle_adamw():
    """From zero moments the first step is lr against the gradient's sign (eps aside), a constant gradient goes on so;
    decay shrinks matrices alone; a clip changes nothing but through eps, as the ratio is scale-free."""
    from oracle import gpipe
    rng = np.random.default_rng(0)
    p = [{"wq": rng.standard_normal((4, 5)), "bq": rng.standard_normal(5), "xwk": rng.standard_normal((2, 2))}]
    g = [{k: rng.standard_normal(v.shape) for k, v in p[0].items()}]
    head = {"lnf_g": np.ones(3)}
    gh = {"lnf_g": np.array([1.0, -2.0, 0.0])}
    cfg = CFG.with_(adam_eps=1e-300, weight_decay=0.5, max_grad_norm=0.0)
    state, q, h = None, p, head
    for t in range(1, 4):
        q, h, state = gpipe.apply_update(cfg, q, h, g, gh, 0.01, state)
        assert state[0] == t
        assert np.allclose(q[0]["bq"], p[0]["bq"] - 0.01 * t * np.sign(g[0]["bq"]), rtol=0, atol=1e-12)
        assert np.allclose(h["lnf_g"], 1 - 0.01 * t * np.array([1, -1, 0]), rtol=0, atol=1e-12)
    one, _, _ = gpipe.apply_update(cfg, p, head, g, gh, 0.01)
    for k in ("wq", "xwk"):
        assert np.allclose(one[0][k], p[0][k] * (1 - 0.01 * 0.5) - 0.01 * np.sign(g[0][k]), rtol=0, atol=1e-12)
    norm = math.sqrt(sum(float((v ** 2).sum()) for v in list(g[0].values()) + [gh["lnf_g"]]))
    cut, _, st = gpipe.apply_update(cfg.with_(max_grad_norm=norm / 4), p, head, g, gh, 0.01)
    assert np.allclose(cut[0]["wq"], one[0]["wq"], rtol=0, atol=1e-12)
    assert np.allclose(st[1][0]["wq"], 0.1 * g[0]["wq"] / 4, rtol=1e-12)
