"""Calls of the token log probabilities that their description allows: layouts of the
gradient's output, against the gradient into a tensor of its own."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ops():
    from paper_1811_06965_amd import ops as o
    return o


def inputs(ops, z):
    g = torch.Generator(device="cuda").manual_seed(2)
    z.copy_(torch.randn(z.shape, generator=g, device="cuda") * 3)
    tok = torch.arange(z.shape[0], dtype=torch.int32, device="cuda") * 3
    r = ops.token_logprobs(z, tok)
    w = torch.linspace(-1, 1, z.shape[0], device="cuda")
    return dict(tokens=tok, lse=r.lse, entropy=r.entropy, dlogp=w, dentropy=0.1 * w)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,gap", [(50, 0), (50, 3), (4099, 1)])
@pytest.mark.parametrize("first", [True, False])
def test_gradient_beside_its_logits(ops, dtype, vocab, gap, first):
    """Logits and their gradient in columns of one buffer; the other columns are left as they were."""
    buf = torch.full((7, 2 * vocab + 2 * gap), 5.0, device="cuda").to(dtype)
    left, right = buf[:, :vocab], buf[:, vocab + gap:2 * vocab + gap]
    z, out = (left, right) if first else (right, left)
    kw = inputs(ops, z)
    want = ops.token_logprobs_backward(z, **kw)
    before = z.clone()
    assert ops.token_logprobs_backward(z, **kw, out=out) is out
    assert torch.equal(out, want) and torch.equal(z, before)
    assert bool((buf[:, vocab:vocab + gap] == 5).all()) and bool((buf[:, 2 * vocab + gap:] == 5).all())


def test_gradient_of_one_row_in_place_by_another_view(ops):
    buf = torch.zeros(3, 100, device="cuda")
    z, out = buf[:1, :60], buf.view(-1)[:60].view(1, 60)  # row strides of 100 and 60
    kw = inputs(ops, z)
    want = ops.token_logprobs_backward(z, **kw)
    ops.token_logprobs_backward(z, **kw, out=out)
    assert torch.equal(z, want)
