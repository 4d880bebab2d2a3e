"""Adapters and gradients on different devices are refused: the kernels of a call run on one.  No GPU: torch's CPU and meta devices stand for two."""
import pytest
import torch


@pytest.fixture
def bd(monkeypatch):
    from paper_2402_10193_amd import binding
    monkeypatch.setattr(binding, "_dev", lambda t, *a: t)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: type("S", (), {"cuda_stream": 0}))
    return binding


def _h(shape, device="cpu", dtype=torch.float16):
    return torch.zeros(shape, dtype=dtype, device=device)


def test_adapters_of_a_table_are_on_one_device(bd):
    table = bd.LoraTable([_h((4, 32)), None, _h((8, 32))], [_h((16, 4)), None, _h((16, 8))], [1.0, 1.0, 1.0])
    assert table.ranks == [4, 0, 8]
    for a, b in (("meta", "cpu"), ("cpu", "meta"), ("meta", "meta")):
        with pytest.raises(ValueError, match="one device"):
            bd.LoraTable([_h((4, 32)), None, _h((8, 32), a)], [_h((16, 4)), None, _h((16, 8), b)], [1.0, 1.0, 1.0])


def test_gradients_are_where_their_matrix_is(bd):
    table = bd.LoraTable([_h((4, 32)), None], [_h((16, 4)), None], [1.0, 1.0])
    f = lambda shape, device="cpu": _h(shape, device, torch.float32)
    bd.LoraGrads(table, [f((4, 32)), None], [f((16, 4)), None])
    with pytest.raises(ValueError, match="is on"):
        bd.LoraGrads(table, [f((4, 32), "meta"), None], [f((16, 4)), None])
    with pytest.raises(ValueError, match="is on"):
        bd.LoraGrads(table, [f((4, 32)), None], [f((16, 4), "meta"), None])
