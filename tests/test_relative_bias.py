"""A relative bias is made for one number of buckets and one furthest distance: what the kernels would read its map of
distances with cannot be another's.  Without a GPU: tensors stay on the host, and a call that reaches the device fails the test."""
import types

import pytest

torch = pytest.importorskip("torch")

HEADS, BUCKETS, DISTANCE = 2, 32, 128


@pytest.fixture
def ops(monkeypatch):
    import os
    from paper_1811_06965_amd import build, gp, ops as o
    if not os.path.exists(gp.LIB_PATH):
        build.build()

    def reached(*_):
        raise AssertionError("the call went on to the device")
    monkeypatch.setattr(o, "_gpu", lambda t: t.device)
    monkeypatch.setattr(o, "_on", reached)
    return o


@pytest.fixture
def bias(ops, monkeypatch):
    b = ops.RelativeBias(torch.zeros(HEADS, BUCKETS), DISTANCE)
    monkeypatch.setattr(ops, "_gpu", lambda t: types.SimpleNamespace(index=t.get_device()))
    return b


def calls(ops, bias):
    q = torch.zeros(1, 4, HEADS, 64)
    lse = torch.zeros(1, HEADS, 4)
    return [lambda: ops.attention(q, q, q, bias=bias), lambda: ops.attention_backward(q, q, q, q, lse, q, bias=bias)]


def test_taken_as_it_was_made(ops, bias):
    with pytest.raises(AssertionError, match="went on"):
        calls(ops, bias)[0]()
    assert bias.max_distance == DISTANCE and bias.bidirectional is True and bias.bucket_of.numel() == 2 * DISTANCE + 1


@pytest.mark.parametrize("name,value", [("max_distance", 1000), ("max_distance", 5), ("bidirectional", False),
                                        ("bucket_of", torch.zeros(3, dtype=torch.int32))])
def test_what_the_map_was_made_for_stays(bias, name, value):
    with pytest.raises(AttributeError):
        setattr(bias, name, value)


@pytest.mark.parametrize("length", [1, 5, 2 * DISTANCE, 2 * DISTANCE + 3])
def test_a_map_of_another_length(ops, bias, length):
    bias.bucket_of.resize_(length)
    for call in calls(ops, bias):
        with pytest.raises(ValueError, match="bucket_of"):
            call()


@pytest.mark.parametrize("table", [torch.zeros(HEADS, BUCKETS - 1), torch.zeros(HEADS, BUCKETS + 1), torch.zeros(HEADS + 1, BUCKETS),
                                   torch.zeros(HEADS * BUCKETS), torch.zeros(HEADS, BUCKETS).double(), torch.zeros(BUCKETS, HEADS).t()])
def test_a_table_of_another_shape(ops, bias, table):
    bias.table = table
    for call in calls(ops, bias):
        with pytest.raises(ValueError, match="table"):
            call()


def test_another_table_of_the_same_shape(ops, bias):
    bias.table = torch.ones(HEADS, BUCKETS)
    with pytest.raises(AssertionError, match="went on"):
        calls(ops, bias)[0]()
