"""AdamW's 8-bit update and the gradient norm at the ends of the fp32 range, against
the same fp32 operations in numpy (tolerances as in test_gpu_adamw.py)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_adamw import F, U, numpy_step, quantise, random_bits  # noqa: E402


@pytest.fixture(scope="module")
def ops():
    from paper_1811_06965_amd import ops as o
    return o


@pytest.mark.parametrize("top", [1e-21, 1e-20, 1e-19, 3e-18, 1e-15, 1e-14, 1.0, 1e4, 1e18, 1.8e19, 2e19, 3e38])
def test_second_moments_of_every_magnitude(ops, top):
    """v below the normal range (|g| up to 3e-18 and beta2 = 0.999) keeps its root, and a v that passes the largest float
    has an infinite root and a step of 0, as in 32 bits: codes, scales and the parameter's step as numpy's.  The
    parameters start at 0 and eps is far below every root, so that the step is all there is to see."""
    n = 1024
    r = np.random.default_rng(5)
    g = (np.linspace(-1, 1, n) * top).astype(F)
    g[r.random(n) < 0.05] = 0
    h = dict(lr=1e-3, b1=0.9, b2=0.999, eps=1e-30, seed=7)
    p, m, v = np.zeros(n, F), np.zeros(n, np.uint8), np.zeros(n, np.uint8)
    ms, vs = np.zeros(n // 256, F), np.zeros(n // 256, F)
    dp, dg = torch.zeros(n, device="cuda"), torch.from_numpy(g).cuda()
    opt = ops.AdamW([dp], [dg], state_bits=8, lr=h["lr"], eps=h["eps"], betas=(h["b1"], h["b2"]), seed=h["seed"])
    for t in (1, 2, 3):
        old = p
        opt.step()
        with np.errstate(all="ignore"):
            p, m, v, ms, vs = numpy_step(p, g, m, v, ms, vs, h, t, 0.0, 1.0, 8, "f32")
        got = dp.cpu().numpy()
        assert np.array_equal(np.isfinite(got), np.isfinite(p)), t
        assert (np.abs(got - p) <= 16 * U * np.abs(p - old) + 4 * U * np.abs(old)).all(), t
        assert np.array_equal(opt.m_scale[0].cpu().numpy(), ms) and np.array_equal(opt.v_scale[0].cpu().numpy(), vs), t
        kept = np.repeat(np.isfinite(vs), 256)  # the codes of a block with an infinite scale mean nothing
        assert np.array_equal(opt.m[0].view(torch.uint8).cpu().numpy()[kept], m[kept]), t
        assert np.array_equal(opt.v[0].view(torch.uint8).cpu().numpy()[kept], v[kept]), t
        if not kept.all():
            assert top > 1e19
            break
        p = got  # numpy goes on from the device's


def test_the_smallest_eps(ops):
    """No gradient yet and the smallest eps that 8-bit states take: nothing moves."""
    p, g = torch.ones(300, device="cuda"), torch.zeros(300, device="cuda")
    opt = ops.AdamW([p], [g], state_bits=8, lr=1.0, eps=2.0 ** -126)
    opt.step()
    assert bool((p == 1.0).all()) and bool((opt.v_scale[0] == 0).all())


@pytest.mark.parametrize("spread", [[1e4, 1e-2, 1e-9, 1e-14], [1e18, 1e-18], [1.0, 1e-11, 1e-12, 1e-13], [1e-2, 1e-14]])
def test_a_second_moment_beside_a_far_larger_one(ops, spread):
    """What is not zero in v does not become zero, however much larger its block's largest is."""
    n = 1024
    r = np.random.default_rng(6)
    g = (np.array(spread)[r.integers(0, len(spread), n)] * r.uniform(1, 2, n)).astype(F)
    g[::17] = 0
    opt = ops.AdamW([torch.zeros(n, device="cuda")], [torch.from_numpy(g).cuda()], state_bits=8, lr=0.0, betas=(0.0, 0.0),
                    seed=3)
    opt.step()
    codes, scales = quantise(np.sqrt(g * g), random_bits(n, 3, 1)[1], True)
    got = opt.v[0].view(torch.uint8).cpu().numpy()
    assert np.array_equal(opt.v_scale[0].cpu().numpy(), scales)
    assert np.array_equal(got == 0, g * g == 0)
    assert np.array_equal(got, codes)


@pytest.mark.parametrize("count", [4, 4000, 400000])
def test_a_norm_past_the_largest_float(ops, count):
    """The norm is stored in fp32: where that is infinite the factor is a NaN, though fp64 holds the sum of the squares.
    (One launch for the short lists, two for the long one.)"""
    big = torch.full((count,), 3e38, device="cuda")
    r = ops.grad_norm([big], max_norm=1.0)
    assert float(r[0]) == math.inf and math.isnan(float(r[1]))
    r = ops.grad_norm([big[:1]], max_norm=1.0)
    assert abs(float(r[0]) / 3e38 - 1) < 1e-6 and abs(float(r[1]) * 3e38 - 1) < 1e-6


@pytest.mark.parametrize("bits", [32, 8])
def test_after_a_gradient_whose_square_is_infinite(ops, bits):
    """A v that passed the largest float stays infinite: its parameter's steps are 0 from there on, in 8 bits its
    block's too, whether they had a gradient before or not; the other blocks go on, and nothing becomes a NaN."""
    n = 1024
    p, g = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    g[1::2] = 0
    p[:] = 1
    opt = ops.AdamW([p], [g], state_bits=bits, lr=1e-3, seed=2)
    opt.step()
    g[300] = 2e19
    opt.step()
    held = p.clone()
    g[300] = 1
    for _ in range(3):
        opt.step()
    moved = p != held
    want = g != 0
    if bits == 8:
        want[256:512] = False
    want[300] = False
    assert bool(p.isfinite().all()) and torch.equal(moved, want)
