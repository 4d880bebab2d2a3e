"""Device memory that the binding makes for itself (an AdamW plan's copy, adapters' scales) and a call that reads it on another stream than the
one it belongs to: the allocator has to hear of it.  No GPU: the library and the tensors' checks are stand-ins."""
import ctypes
import types

import pytest
import torch


class Memory:
    """What a call reads, belonging to stream 1."""

    def __init__(self):
        self.told = []

    def record_stream(self, stream):
        self.told.append(stream)

    def data_ptr(self):
        return 0x1000

    def get_device(self):
        return 0

    def numel(self):
        return 4


@pytest.fixture
def bd(monkeypatch):
    from paper_2402_10193_amd import binding
    call = lambda *a: 0
    monkeypatch.setattr(binding, "lib", lambda: types.SimpleNamespace(bd_adamw=call, bd_lora_multitenant=call, bd_lora_multitenant_group=call,
                                                                      bd_lora_multitenant_backward=call))
    monkeypatch.setattr(binding, "_dev", lambda t, *a: t)
    monkeypatch.setattr(binding, "_here", lambda *a: None)
    monkeypatch.setattr(binding, "_device_of", lambda t, what: 0)
    monkeypatch.setattr(binding, "_arg", lambda *a: 0)
    monkeypatch.setattr(binding, "_stream", lambda s: 1 if s is None else int(s))
    monkeypatch.setattr(binding, "_stream_of", lambda s, dev: 1 if s is None else int(s))
    monkeypatch.setattr(binding, "_memory_of", lambda s, dev: pytest.fail("nothing is to be allocated"))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda s, device=None: s)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: 1)
    return binding


def _table(bd):
    t = bd.LoraTable.__new__(bd.LoraTable)
    t.a, t.b, t.shape, t.ranks, t.max_rank, t.n_tenants, t.device, t.scale = [None], [None], (8, 32), [0], 0, 1, 0, Memory()
    t.a_ptrs = t.b_ptrs = (ctypes.c_void_p * 1)()
    t.rank_arr, t.streams = (ctypes.c_int32 * 1)(), {1}
    return t


def _calls(bd):
    x, y, ws = torch.zeros((1, 32), dtype=torch.float16), torch.zeros((1, 8), dtype=torch.float16), torch.zeros(256, dtype=torch.uint8)
    table, grouped, one = _table(bd), _table(bd), torch.zeros(1)
    group = bd.LoraGroup([grouped], [8])
    plan = bd.AdamWGroup.__new__(bd.AdamWGroup)
    plan.n, plan.bytes, plan.plan, plan.plan_device, plan.keep, plan.streams, plan.device = 1, 8, None, Memory(), [[one]], {1}, torch.device("cuda", 0)
    return [(table.scale, lambda s: bd.lora_multitenant(x, table, [0], y=y, workspace=ws, stream=s)),
            (table.scale, lambda s: bd.lora_multitenant_backward(y, None, None, table, [0], None, dx=x, workspace=ws, stream=s)),
            (grouped.scale, lambda s: bd.lora_multitenant_group(x, group, [0], ys=[y], workspace=ws, stream=s)),
            (plan.plan_device, lambda s: bd.adamw(plan, one, one, stream=s))]


@pytest.mark.parametrize("which", range(4))
def test_memory_read_on_another_stream_is_reported(bd, which):
    memory, call = _calls(bd)[which]
    call(None)
    call(1)
    assert memory.told == []                            # its own stream
    call(7)
    call(9)
    call(7)
    assert memory.told == [7, 9]                        # once for each
