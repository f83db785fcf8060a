"""AdamW over many tensors and the gradient norm against plain implementations.

The update is held to two references: the same fp32 operations in numpy, one
rounding each (32-bit states with their parameters, 8-bit codes and scales, bit for
bit), and the formulas in 64 bits.  With 8-bit states the parameter's step takes a
reciprocal off by 2 u and fused sums: within 16 u of the step and 3 u of the parameter of
numpy's, and where either is rounded to bf16, a step (2^-7) of it.  Tolerances of the latter (u = 2^-24): m and v are two
products and a sum, 3 u of the absolute terms; the parameter's step
x = lr / bc1 m / (sqrt(v) / sqrt(bc2) + eps) has seven roundings beside those of
m and v: 16 u |x|, then the sum with the decayed parameter, 3 u of it, and half a
step of its type.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = [1, 2, 3, 5, 255, 256, 257, 1000, 4095, 4096, 4097, 0, 12289, 64]
F = np.float32


@pytest.fixture(scope="module")
def ops():
    from paper_1811_06965_amd import ops as o
    return o


def bf16_round(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).float().numpy()


def decode(codes):
    return torch.from_numpy(codes.copy()).view(torch.float8_e4m3fn).float().numpy()


def random_bits(n, seed, t):
    M = np.uint64(0xFFFFFFFF)
    i = np.arange(n, dtype=np.uint64)
    h = ((i >> np.uint64(2)) + np.uint64((seed * 0x3C6EF372 + t * 0x1E3779B1) & 0xFFFFFFFF)) & M
    h ^= h >> np.uint64(16)
    h = h * np.uint64(0x6A3F9B15) & M
    h ^= h >> np.uint64(15)
    h = h * np.uint64(0x5D47C1E3) & M
    h ^= h >> np.uint64(16)
    k = np.array([0x4F1BBCDD, 0x7A6D2C8B, 0x35E9A1F7, 0x1D872B41], dtype=np.uint64)[(i & np.uint64(3)).astype(int)]
    h = h * k & M
    return (h & np.uint64(0xFFFF)).astype(np.uint32), (h >> np.uint64(16)).astype(np.uint32)


def quantise(x, rnd, keep):
    """(codes, scales) of blocks of 256: e4m3 of |x| 448 / max|x|, rounded up where the random bits say."""
    n, codes, scales = len(x), np.zeros(len(x), np.uint8), []
    for a in range(0, n, 256):
        b = x[a:a + 256]
        top = np.abs(b).max()
        tiny = top < F(2.0 ** -100)
        scales.append(F(0) if tiny else top * (F(1) / F(448)))
        inv = F(0) if tiny else F(1) / top * F(448)
        y = b * inv
        c = ((np.abs(y) * F(2.0 ** -120)).view(np.uint32) + (rnd[a:a + 256] << np.uint32(4)) + np.uint32(8)) >> np.uint32(20)
        c = np.minimum(c, 126)
        if keep:
            c = np.where((y > 0) & (c == 0), 1, c)
        codes[a:a + 256] = c | np.where(np.signbit(y), 128, 0)  # a zero keeps its sign
    return codes, np.array(scales, F)


def numpy_step(p, g, m, v, ms, vs, h, t, decay, factor, bits, param):
    """One update of one tensor in fp32, one rounding an operation; arrays in, arrays out."""
    b1, c1, b2, c2 = F(h["b1"]), F(1 - h["b1"]), F(h["b2"]), F(1 - h["b2"])
    step_size, inv_root = F(h["lr"] / (1 - h["b1"] ** t)), F(1 / math.sqrt(1 - h["b2"] ** t))
    if bits == 8:
        rep = lambda s: np.repeat(s, 256)[:len(p)]  # noqa: E731
        m, r = decode(m) * rep(ms), decode(v) * rep(vs)
        v = r * r
    g = g * F(factor)
    m = m * b1 + g * c1
    v = v * b2 + g * g * c2
    root = np.sqrt(v)
    p = p * F(1 - h["lr"] * decay) - step_size * m / (root * inv_root + F(h["eps"]))
    if param == "bf16":
        p = bf16_round(p)
    if bits == 8:
        lo, hi = random_bits(len(p), h["seed"], t)
        m, ms = quantise(m, lo, False)
        v, vs = quantise(root, hi, True)
    return p, m, v, ms, vs


class Case:
    """Tensors of SIZES laid end to end (from an odd element on) or on their own, with guards around."""

    def __init__(self, bits, param, grad, copies, seed, sizes=SIZES, offset=1):
        r = np.random.default_rng(seed)
        self.bits, self.param, self.sizes = bits, param, sizes
        self.flat = {}

        def lay(name, values, dtype):
            n = sum(len(x) for x in values)
            host = torch.full((offset + n + 9,), 3.0).to(dtype) if dtype != torch.uint8 else torch.full(
                (offset + n + 9,), 0xAB, dtype=torch.uint8)
            at, views = offset, []
            buf = host.cuda()
            for x in values:
                view = buf[at:at + len(x)]
                view.copy_(torch.from_numpy(np.ascontiguousarray(x)))
                views.append(view)
                at += len(x)
            self.flat[name] = (buf, host, offset, at)
            return views

        mags = [10.0 ** r.uniform(-6, 1) for _ in sizes]
        g = [(r.standard_normal(n) * k * (r.random(n) > 0.1)).astype(F) for n, k in zip(sizes, mags)]
        p = [(r.standard_normal(n) * 0.05).astype(F) for n in sizes]
        m = [(r.standard_normal(n) * k * 0.3).astype(F) for n, k in zip(sizes, mags)]
        root = [(np.abs(r.standard_normal(n)) * k).astype(F) for n, k in zip(sizes, mags)]
        self.p = [bf16_round(x) if param == "bf16" else x for x in p]
        self.g = [bf16_round(x) if grad == "bf16" else x for x in g]
        self.params, self.grads = lay("p", self.p, DT[param]), lay("g", self.g, DT[grad])
        self.copies = lay("c", [np.zeros(n, F) for n in sizes], torch.bfloat16) if copies else None
        self.ms = self.vs = None
        if bits == 32:
            self.m, self.v = m, [x * x for x in root]
            self.dm, self.dv = lay("m", self.m, torch.float32), lay("v", self.v, torch.float32)
            self.dms = self.dvs = None
        else:
            half = lambda x: np.full(len(x), 32768, np.uint32)  # noqa: E731
            qm, qv = [quantise(x, half(x), False) for x in m], [quantise(x, half(x), True) for x in root]
            self.m, self.ms = [q[0] for q in qm], [q[1] for q in qm]
            self.v, self.vs = [q[0] for q in qv], [q[1] for q in qv]
            self.dm = [x.view(torch.float8_e4m3fn) for x in lay("m", self.m, torch.uint8)]
            self.dv = [x.view(torch.float8_e4m3fn) for x in lay("v", self.v, torch.uint8)]
            self.dms, self.dvs = lay("ms", self.ms, torch.float32), lay("vs", self.vs, torch.float32)
        self.decay = [0.0 if i % 3 == 0 else 0.1 for i in range(len(sizes))]
        self.h = dict(lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, seed=seed)

    def optimizer(self, ops, **kw):
        h = self.h
        return ops.AdamW(self.params, self.grads, m=self.dm, v=self.dv, m_scale=self.dms, v_scale=self.dvs,
                         copies=self.copies, weight_decay=self.decay, betas=(h["b1"], h["b2"]), eps=h["eps"],
                         lr=h["lr"], seed=h["seed"], **kw)

    def host_step(self, t, factor=1.0):
        self.old = [x.copy() for x in self.p]
        for i in range(len(self.sizes)):
            if self.sizes[i] == 0:
                continue
            with np.errstate(all="ignore"):
                self.p[i], self.m[i], self.v[i], ms, vs = numpy_step(
                    self.p[i], self.g[i], self.m[i], self.v[i], self.ms and self.ms[i], self.vs and self.vs[i], self.h, t,
                    self.decay[i], factor, self.bits, self.param)
            if self.bits == 8:
                self.ms[i], self.vs[i] = ms, vs

    def check_params(self, i, got):
        """With 8-bit states: near numpy's, which then goes on from the device's."""
        if self.bits == 32:
            assert np.array_equal(got, self.p[i]), i
            return
        fine = np.isfinite(self.p[i])
        step = np.abs(self.old[i] * (1 - self.h["lr"] * self.decay[i]) - self.p[i])
        tol = 16 * U * step + 4 * U * np.abs(self.old[i]) + (2.0 ** -7 * np.abs(self.p[i]) if self.param == "bf16" else 0)
        assert (np.abs(got - self.p[i])[fine] <= tol[fine]).all(), i
        self.p[i] = got

    def check(self):
        bits = lambda x: np.ascontiguousarray(x).view(np.uint8)  # noqa: E731
        for i, n in enumerate(self.sizes):
            self.check_params(i, self.params[i].float().cpu().numpy())
            pairs = [(self.dm[i], self.m[i]), (self.dv[i], self.v[i])]
            if self.bits == 8:
                pairs += [(self.dms[i], self.ms[i]), (self.dvs[i], self.vs[i])]
            for d, x in pairs:
                d = d.view(torch.uint8) if d.dtype == torch.float8_e4m3fn else d
                assert np.array_equal(bits(d.cpu().numpy()), bits(x)), (i, n)
            if self.copies:  # the fp32 parameter as it was stored, rounded
                assert np.array_equal(self.copies[i].float().cpu().numpy(), bf16_round(self.p[i])), (i, n)
        for name, (buf, host, a, b) in self.flat.items():
            x, y = buf.cpu(), host
            assert torch.equal(x[:a].view(torch.uint8), y[:a].view(torch.uint8)), name
            assert torch.equal(x[b:].view(torch.uint8), y[b:].view(torch.uint8)), name


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,copies", [("f32", "f32", True), ("f32", "bf16", False), ("bf16", "f32", False),
                                               ("bf16", "bf16", False)])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_update_bit_for_bit(ops, bits, param, grad, copies, offset):
    c = Case(bits, param, grad, copies, 11 + offset, offset=offset)
    opt = c.optimizer(ops, steps=4)
    for t in (5, 6, 7):
        opt.step()
        c.host_step(t)
        torch.cuda.synchronize()
        c.check()
    assert opt.steps == 7


@pytest.mark.parametrize("bits", [32, 8])
def test_update_of_large_and_many_tensors(ops, bits):
    """More tensors than a launch takes, some empty, and one of many workgroups."""
    c = Case(bits, "f32", "f32", False, 5, sizes=[0] + [7 * i % 301 for i in range(120)] + [300001, 0, 33], offset=3)
    opt = c.optimizer(ops)
    opt.step()
    c.host_step(1)
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("param", ["f32", "bf16"])
@pytest.mark.parametrize("t", [1, 2, 1000, 10 ** 7])
def test_update_against_64_bits(ops, param, t):
    c = Case(32, param, "f32", False, 3)
    p0, m0, v0 = ([x.astype(np.float64) for x in y] for y in (c.p, c.m, c.v))
    c.optimizer(ops, steps=t - 1).step()
    torch.cuda.synchronize()
    for i, n in enumerate(c.sizes):
        g = c.g[i].astype(np.float64)
        m, v = 0.9 * m0[i] + 0.1 * g, 0.999 * v0[i] + 0.001 * g * g
        x = 1e-3 / (1 - 0.9 ** t) * m / (np.sqrt(v / (1 - 0.999 ** t)) + 1e-8)
        p = p0[i] * (1 - 1e-3 * c.decay[i]) - x
        am = 0.9 * np.abs(m0[i]) + 0.1 * np.abs(g)
        assert (np.abs(c.dm[i].double().cpu().numpy() - m) <= 3 * U * am + 1e-44).all()
        assert (np.abs(c.dv[i].double().cpu().numpy() - v) <= 4 * U * v + 1e-44).all()
        with np.errstate(all="ignore"):
            ax = np.where(am > 0, np.abs(x) * (16 * U) + 1e-3 / (1 - 0.9 ** t) * 3 * U * am / (np.sqrt(v / (1 - 0.999 ** t)) + 1e-8), 0)
        half = 2.0 ** -8 if param == "bf16" else U
        tol = ax + 3 * U * np.abs(p0[i]) + (half + U) * np.abs(p)
        assert (np.abs(c.params[i].double().cpu().numpy() - p) <= tol + 1e-44).all(), n


@pytest.mark.parametrize("bits", [32, 8])
def test_factor(ops, bits):
    """A factor on the device scales the gradients; a NaN leaves every byte as it was, the counter on the device
    included."""
    c = Case(bits, "f32", "f32", True, 21)
    opt = c.optimizer(ops, capturable=True)
    torch.cuda.synchronize()
    before = {k: v[0].clone() for k, v in c.flat.items()}
    opt.step(factor=torch.full((1,), math.nan, device="cuda"))
    torch.cuda.synchronize()
    for k, v in c.flat.items():
        assert torch.equal(v[0].view(torch.uint8), before[k].view(torch.uint8)), k
    assert int(opt.step_dev) == 0
    c = Case(bits, "f32", "f32", True, 21)
    opt = c.optimizer(ops)
    opt.step(factor=torch.full((1,), 0.125, device="cuda"))
    c.host_step(1, 0.125)
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_update(ops, bits):
    """The counter on the device: replays take steps 1, 2, 3, ..., with the program's own work between, and equal
    eager steps with the same counter.  Its bias corrections are fp32 functions of t (4 u), so it is
    compared with the host's step within 16 u of the step plus the parameter's rounding."""
    c, e, h = (Case(bits, "f32", "f32", False, 9) for _ in range(3))
    opt, eager, host = c.optimizer(ops, capturable=True), e.optimizer(ops, capturable=True), h.optimizer(ops)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    for k in range(4):
        graph.replay()
        torch.zeros(1000, device="cuda").sum()
        eager.step()
        torch.cuda.synchronize()
        assert int(opt.step_dev) == k + 1 == int(eager.step_dev)
        for name in c.flat:
            assert torch.equal(c.flat[name][0].view(torch.uint8), e.flat[name][0].view(torch.uint8)), name
        if k == 0:
            host.step()
            for a, b in zip(c.params, h.params):
                assert bool(((a - b).abs() <= 16 * U * 1e-2 + 2 * U * b.abs()).all())


def test_host_step_is_refused_in_a_capture(ops):
    from paper_1811_06965_amd import gp
    c = Case(32, "f32", "f32", False, 2, sizes=[64])
    opt = c.optimizer(ops)
    before = c.params[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(gp.GpError) as err:
            opt.step()
    assert err.value.status == gp.GP_ERR_STATE and opt.steps == 0
    assert torch.equal(c.params[0], before)


def test_special_gradients(ops):
    """NaN and infinities reach their element (32 bits) or their block (8 bits) and no other; a zero gradient with
    zero states moves nothing; tiny blocks are stored as zeros."""
    n = 1024
    for bits in (32, 8):
        p = torch.ones(n, device="cuda")
        g = torch.full((n,), 1e-3, device="cuda")
        g[5], g[300], g[512:768] = math.nan, math.inf, 0.0
        g[768:] = 1e-35
        opt = ops.AdamW([p], [g], state_bits=bits, lr=0.5)
        opt.step()
        torch.cuda.synchronize()
        bad = torch.zeros(n, dtype=torch.bool)
        bad[5] = bad[300] = True
        assert torch.equal(p.isnan().cpu(), bad)
        assert bool((p[512:768] == 1.0).all())
        good = ~bad
        good[512:] = False
        assert bool(((p.cpu()[good] - 0.5).abs() < 1e-4).all())  # the first step is lr against the gradient's sign
        if bits == 8:
            assert opt.v_scale[0].isfinite().tolist() == [False, False, True, True]
            assert opt.m_scale[0].isfinite().tolist() == [False, False, True, True]
            assert opt.m_scale[0][3] == 0.0 and bool((opt.m[0].view(torch.uint8)[768:] == 0).all())


@pytest.mark.parametrize("top", [1e-29, 1e-20, 1.0, 8191.0, 8193.0, 1e18, 3e38])
def test_blocks_of_every_magnitude(ops, top):
    """8-bit first moments from the smallest block that is kept to the largest floats: each value within a step of
    e4m3 (an eighth of it, or 2^-9 of the block's 448th), the block's largest exact."""
    g = torch.linspace(-1, 1, 1024, device="cuda") * top
    p = torch.zeros(1024, device="cuda")
    opt = ops.AdamW([p], [g], state_bits=8, betas=(0.0, 0.5), lr=0.0)
    opt.step()
    m = (opt.m[0].double().view(-1, 256) * opt.m_scale[0].double()[:, None]).view(-1)
    step = (g.double().abs() / 8).clamp(min=0) + opt.m_scale[0].double().repeat_interleave(256) * 2.0 ** -9
    assert bool(((m - g.double()).abs() <= step).all())
    most = g.view(-1, 256).abs().amax(1).double()
    assert bool(((m.view(-1, 256).abs().amax(1) / most - 1).abs() < 1e-6).all())


def test_random_rounding_keeps_small_changes(ops):
    """A constant gradient g of 1: v grows by a thousandth of what is left each step, a tenth of what rounding to
    nearest in e4m3 would need to see.  After 400 steps from v = 0.01 the mean root over many elements is that of the
    32-bit states: the roots' random rounding walks with less than 0.35 of relative deviation, and over
    2^16 elements the mean is off by under 0.35 / 256 plus the inflation of the mean square, below 6 percent."""
    n = 1 << 16
    out = []
    for bits in (32, 8):
        p, g = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
        if bits == 32:
            st = dict(m=[torch.zeros(n, device="cuda")], v=[torch.full((n,), 0.01, device="cuda")])
        else:
            one = torch.full((n,), 448.0, device="cuda").to(torch.float8_e4m3fn)
            st = dict(m=[torch.zeros(n, device="cuda").to(torch.float8_e4m3fn)], v=[one],
                      m_scale=[torch.zeros(n // 256, device="cuda")],
                      v_scale=[torch.full((n // 256,), 0.1 / 448, device="cuda")])
        opt = ops.AdamW([p], [g], lr=0.0, seed=3, **st)
        for _ in range(400):
            opt.step()
        if bits == 32:
            out.append((opt.m[0].mean(), opt.v[0].sqrt().mean()))
        else:
            val = lambda q, s: (q.float().view(-1, 256) * s[:, None]).mean()  # noqa: E731
            out.append((val(opt.m[0], opt.m_scale[0]), val(opt.v[0], opt.v_scale[0])))
    (m32, r32), (m8, r8) = out
    assert abs(float(m32) - 1) < 1e-3 and abs(float(r32) - math.sqrt(0.01 + 0.99 * (1 - 0.999 ** 400))) < 1e-3
    assert abs(float(m8 / m32) - 1) < 0.02
    assert abs(float(r8 / r32) - 1) < 0.06


# -------------------------------------------------------------- gradient norm
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[1], [3, 0, 5], SIZES, [7 * i % 97 for i in range(300)], [9000001, 17, 4096],
                                   [120 * 1024], [120 * 1024 + 1], [1023, 1024, 1025] * 29, [3] * 120, [3] * 121,
                                   [0, 5] * 64, [0, 5] * 65])
@pytest.mark.parametrize("offset", [0, 1])
def test_grad_norm(ops, dtype, sizes, offset):
    """Squares are summed in fp64, so the norm is rounded once to fp32: u of it, and the factor twice."""
    g = torch.Generator().manual_seed(sum(sizes))
    buf = (torch.randn(offset + sum(sizes), generator=g) * 0.01).to(DT[dtype]).cuda()
    at, views = offset, []
    for n in sizes:
        views.append(buf[at:at + n])
        at += n
    want = math.sqrt(float((buf[offset:].double() ** 2).sum()))
    r = ops.grad_norm(views, max_norm=0.5 * want)
    again = ops.grad_norm(ops.TensorList(views), max_norm=0.5 * want)
    assert torch.equal(r, again)
    assert abs(float(r[0]) - want) <= 1.01 * U * want
    assert abs(float(r[1]) - 0.5) <= 4 * U
    assert float(ops.grad_norm(views, max_norm=2 * want)[1]) == 1.0
    assert float(ops.grad_norm(views)[1]) == 1.0


def test_grad_norm_special(ops):
    z = torch.zeros(1000, device="cuda")
    assert ops.grad_norm([z], max_norm=1.0).tolist() == [0.0, 1.0]
    assert ops.grad_norm([z[:0]], max_norm=1.0).tolist() == [0.0, 1.0]
    big = torch.full((4, 1000), 3e38, device="cuda")  # squares past fp32, and the norm too: 1.9e40
    r = ops.grad_norm([big[0, :1]], max_norm=1.0)
    assert abs(float(r[0]) / 3e38 - 1) < 1e-6 and abs(float(r[1]) * 3e38 - 1) < 1e-6
    for bad in (math.nan, math.inf, -math.inf):
        z[777] = bad
        r = ops.grad_norm([big[0, :5], z], max_norm=1.0)
        assert not math.isfinite(float(r[0])) and math.isnan(float(r[1]))
    from paper_1811_06965_amd import gp
    out, ws = torch.empty(2, device="cuda"), torch.empty(gp.gp_grad_norm_workspace(0), dtype=torch.uint8, device="cuda")
    gp.gp_grad_norm(gp.GP_F32, None, 0, 1.0, out.data_ptr(), ws.data_ptr(), ws.numel(),
                    torch.cuda.current_stream().cuda_stream)
    assert out.tolist() == [0.0, 1.0]


def test_a_training_step_of_them_together(ops):
    """Logits of a linear map, log probabilities with an entropy bonus, their gradient, the norm, a clipped
    AdamW step with 32- and with 8-bit states, captured and replayed: the parameters follow the plain
    computation in 64 bits.  Ten steps of at most lr = 1e-2 each; a step's sign-like ratio m / sqrt(v) amplifies the
    fp32 gradients' error (1e-5 of the largest) least where they are large: elements whose gradient stays over a
    hundredth of the largest are compared, within 1 percent (32 bits)."""
    torch.manual_seed(4)
    R, D, V = 64, 48, 1003
    x, tok = torch.randn(R, D), torch.randint(0, V, (R,)).to(torch.int32)
    tok[5] = -1
    w0 = torch.randn(D, V) * 0.2
    a, b = -torch.ones(R) / R, -0.01 * torch.ones(R) / R

    w = w0.double().requires_grad_()
    m, v = torch.zeros(D, V, dtype=torch.double), torch.zeros(D, V, dtype=torch.double)
    norms, losses, solid = [], [], torch.ones(D, V, dtype=torch.bool)
    for t in range(1, 11):
        s = torch.log_softmax(x.double() @ w, 1)
        h = -(s.exp() * s).sum(1)
        lp = torch.where(tok < 0, 0.0, s[torch.arange(R), tok.clamp(min=0).long()])
        loss = (a * lp).sum() + (b * h).sum()
        g, = torch.autograd.grad(loss, w)
        norms.append(float(g.norm()))
        losses.append(float(loss))
        solid &= g.abs() > 0.01 * g.abs().max()
        g = g * min(1.0, 0.05 / norms[-1])
        m, v = 0.9 * m + 0.1 * g, 0.999 * v + 0.001 * g * g
        with torch.no_grad():
            w = w * (1 - 1e-2 * 0.1) - 1e-2 / (1 - 0.9 ** t) * m / ((v / (1 - 0.999 ** t)).sqrt() + 1e-8)
        w.requires_grad_()

    xd, td, ad, bd = x.cuda(), tok.cuda(), a.cuda(), b.cuda()
    for bits in (32, 8):
        wd = w0.cuda()
        z, gw = torch.empty(R, V, device="cuda"), torch.empty(D, V, device="cuda")
        opt = ops.AdamW([wd], [gw], state_bits=bits, weight_decay=0.1, lr=1e-2, capturable=True)
        grads = ops.TensorList([gw])

        def step():
            torch.mm(xd, wd, out=z)
            r = ops.token_logprobs(z, td)
            dz = ops.token_logprobs_backward(z, td, r.lse, r.entropy, ad, bd, out=z)
            torch.mm(xd.t(), dz, out=gw)
            f = ops.grad_norm(grads, max_norm=0.05)
            opt.step(factor=f[1:])
            return r, f

        r, f = step()  # the first step outside the graph
        assert abs(float(f[0]) / norms[0] - 1) < 1e-4
        loss = float((ad * r.logp).sum() + (bd * r.entropy).sum())
        assert abs(loss - losses[0]) < 1e-4
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            r, f = step()
        for t in range(1, 10):
            graph.replay()
            torch.cuda.synchronize()
            assert abs(float(f[0]) / norms[t] - 1) < (1e-2 if bits == 32 else 0.1)
        assert int(opt.step_dev) == 10
        moved = (w.detach() - w0.double())[solid]
        got = (wd.double().cpu() - w0.double())[solid]
        assert int(solid.sum()) > 50
        err = ((got - moved).abs() / moved.abs().clamp(min=1e-3)).max()
        if bits == 32:
            assert float(err) < 0.01
        else:
            # e4m3 roundings of up to an eighth in both moments, averaged over ten steps
            assert float((got - moved).norm() / moved.norm()) < 0.125
