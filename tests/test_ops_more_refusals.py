"""Further refusals of the operators on the caller's own tensors, by the host alone
(the addresses are made up, as in test_ops_refusals.py)."""
import pytest

from test_ops_refusals import A, INVALID, adamw, back, gp  # noqa: F401 (gp: the fixture)


@pytest.mark.parametrize("eps", [1e-39, 1e-45, 2.0 ** -127])
def test_a_subnormal_eps_with_8_bit_states(gp, eps):  # noqa: F811
    assert adamw(gp, cfg={"state_bits": 8, "eps": eps}, tensor={"m_scale": A, "v_scale": A}) == INVALID
    assert "eps" in gp.gp_last_error()


@pytest.mark.parametrize("off", [4, 39, 40 * 4 - 10 * 4 + 4, 40 * 4, 3 * 40 * 4 + 4])
def test_columns_that_overlap(gp, off):  # noqa: F811
    """Four rows of 10 floats, 40 apart, and the same that many bytes on: an element, or a row, in common."""
    assert back(gp, ld=40, ldd=40, dlogits=A + off // 4 * 4) == INVALID
    assert back(gp, ld=40, ldd=40, logits=A + off // 4 * 4, dlogits=A) == INVALID


def test_logits_whose_gradient_would_be_lost():
    """Refused with autograd on, before the device is looked at; taken without."""
    torch = pytest.importorskip("torch")
    from paper_1811_06965_amd import ops
    z, one, tok = torch.zeros(3, 5, requires_grad=True), torch.zeros(3, requires_grad=True), torch.zeros(3).int()
    f = torch.zeros(3)
    calls = [lambda: ops.token_logprobs(z, tok), lambda: ops.token_logprobs(z * 2, tok),
             lambda: ops.token_logprobs_backward(z, tok, f, dlogp=f),
             lambda: ops.token_logprobs_backward(z.detach(), tok, f, dlogp=one),
             lambda: ops.token_logprobs_backward(z.detach(), tok, f, dlogp=f, out=z)]
    for call in calls:
        with pytest.raises(ValueError, match="autograd"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="GPU"):
        ops.token_logprobs(z.detach(), tok)
