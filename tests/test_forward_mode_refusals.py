"""Dual tensors of forward-mode differentiation: the operators give no tangents, so an input that has one is refused, before
the device is looked at (autograd is off for some calls: that keeps no tangent back).  Without a GPU."""
import contextlib
import types

import pytest

torch = pytest.importorskip("torch")
from torch.autograd import forward_ad  # noqa: E402

F = torch.zeros(3)
I = torch.zeros(3, 2, dtype=torch.int32)
T = torch.zeros(3, 2)
Z = torch.zeros(3, 5)
Q = torch.zeros(1, 4, 2, 8)
L = torch.zeros(1, 2, 4)
TABLE = torch.zeros(2, 8)

CALLS = {
    "token_logprobs": (lambda o, a: o.token_logprobs(a[0], I[:, 0]), [Z]),
    "token_logprobs_backward": (lambda o, a: o.token_logprobs_backward(a[0], I[:, 0], a[1], entropy=a[2], dlogp=a[3], dentropy=a[4], out=a[5]),
                                [Z, F, F, F, F, Z]),
    "distill": (lambda o, a: o.distill(a[0], I, a[1]), [Z, T]),
    "distill_backward": (lambda o, a: o.distill_backward(a[0], I, a[1], a[2], a[3], rest_lse=a[4], out=a[5]), [Z, T, F, F, F, Z]),
    "attention": (lambda o, a: o.attention(a[0], a[1], a[2], bias=types.SimpleNamespace(table=a[3])), [Q, Q, Q, TABLE]),
    "attention_backward": (lambda o, a: o.attention_backward(a[0], a[1], a[2], a[3], a[4], a[5], bias=types.SimpleNamespace(table=a[6]),
                                                             grads=(a[7], a[8], a[9])), [Q, Q, Q, Q, L, Q, TABLE, Q, Q, Q]),
}


@pytest.mark.parametrize("name,i", [(n, i) for n, (_, inputs) in CALLS.items() for i in range(len(inputs))])
@pytest.mark.parametrize("mode", [contextlib.nullcontext, torch.no_grad])
def test_a_tangent_that_would_be_lost(name, i, mode):
    from paper_1811_06965_amd import ops
    call, inputs = CALLS[name]
    with forward_ad.dual_level(), mode():
        dual = [forward_ad.make_dual(t.clone(), torch.ones_like(t)) if j == i else t for j, t in enumerate(inputs)]
        with pytest.raises(ValueError, match="tangent"):
            call(ops, dual)
        with pytest.raises(ValueError, match="GPU"):  # within a level, but without one
            call(ops, inputs)


def test_functions_of_a_transform():
    from paper_1811_06965_amd import ops
    with pytest.raises(ValueError, match="tangent"):
        torch.func.jvp(lambda z: ops.token_logprobs(z, I[:, 0]).lse, (Z,), (torch.ones_like(Z),))
