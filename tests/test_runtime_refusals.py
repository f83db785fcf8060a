"""Tensors that a partition's driver refuses before the library is called: on another
device, or of another type or size.  No partition is made (there is no GPU here); the
library would report the missing handle instead of a ValueError."""
import pytest

import synth

torch = pytest.importorskip("torch")


@pytest.fixture
def part():
    from paper_1811_06965_amd.runtime import Partition
    p = object.__new__(Partition)
    p.cfg = synth.PartitionConfig("dec", layers=2, d_model=32, d_ff=64, heads=2, seq=8, batch=4, micro=2, dtype="f32",
                                  kind="decoder", loss="xent_ls", vocab=40, mem_seq=6)
    p.M, p.tdtype, p.h, p._lane, p.device = 2, torch.float32, None, None, torch.device("cuda", 0)
    return p


def good(device):
    return dict(x=torch.zeros(2, 8, 32, device=device), tokens=torch.zeros(2, 8, dtype=torch.int32, device=device),
                mem=torch.zeros(2, 6, 32, device=device))


def test_scoring_of_tensors_on_the_host(part):
    with pytest.raises(ValueError, match="cuda:0"):
        part.score(**good("cpu"))


@pytest.mark.parametrize("name", ["x", "tokens", "mem"])
def test_scoring_with_one_tensor_elsewhere(part, name):
    part.device = torch.device("cpu")  # the others are where the partition is
    kw = good("cpu")
    kw[name] = kw[name].to("meta")
    with pytest.raises(ValueError, match=name):
        part.score(**kw)


@pytest.mark.parametrize("kw", [dict(top=-1), dict(top=33), dict(top=41)])
def test_alternatives_out_of_range(part, kw):
    part.device = torch.device("cpu")
    with pytest.raises(ValueError, match="top"):
        part.score(**good("cpu"), **kw)


@pytest.mark.parametrize("device,name", [("cuda", "dy"), ("cpu", "dlogp"), ("cpu", "dentropy")])
def test_token_weights_on_another_device(part, device, name, monkeypatch):
    """Nothing on the partition's device, and one of the weights elsewhere."""
    refused(part, device, name, monkeypatch, dict(dlogp=torch.zeros(4, 8), dentropy=torch.zeros(4, 8)), name)


@pytest.mark.parametrize("name,bad", [("dy", torch.zeros(4, 8, dtype=torch.int64)), ("dlogp", torch.zeros(4, 9)),
                                      ("dentropy", torch.zeros(4, 8).double()), ("dlogp", torch.zeros(8, 4).t())])
def test_token_weights_of_another_type_or_shape(part, name, bad, monkeypatch):
    refused(part, "cpu", name, monkeypatch, {"dlogp": torch.zeros(4, 8), name: bad})


def refused(part, device, name, monkeypatch, kw, elsewhere=None):
    from paper_1811_06965_amd import gp
    part.device = torch.device(device, 0) if device == "cuda" else torch.device(device)
    stream = type("S", (), {"cuda_stream": 0})()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: stream)
    monkeypatch.setattr(gp, "gp_forward_microbatch", lambda *a: pytest.fail("a forward was issued"))
    if elsewhere in kw:
        kw[elsewhere] = kw[elsewhere].to("meta")
    dy = kw.pop("dy", torch.zeros(4, 8, dtype=torch.int32))
    with pytest.raises(ValueError, match=name):
        part.step(torch.zeros(4, 8, 32), torch.zeros(4, 6, 32), dy, fwd_streams=1, bwd_streams=1, **kw)
