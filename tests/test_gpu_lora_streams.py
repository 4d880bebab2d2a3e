"""Memory that tables and plans keep for themselves stays theirs while a call on another stream still needs it, also where they are dropped."""
import pytest
import torch

import lora_ref as ref64

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def bd():
    from paper_2402_10193_amd import binding
    return binding


def _not_handed_on(address, nbytes):
    """Tensors of that size, of the current stream: none at that address."""
    taken = [torch.empty(nbytes, dtype=torch.uint8, device=DEV) for _ in range(16)]
    return all(not (t.data_ptr() <= address < t.data_ptr() + t.numel()) for t in taken)


def _busy(side):
    """A stream that will not come to the next call for some milliseconds."""
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)


def test_a_plan_dropped_after_a_step_on_another_stream(bd):
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    n = 5000
    start = torch.randn(n, generator=g, device=DEV)
    grad = torch.randn(n, generator=g, device=DEV)
    lr, step = torch.full((1,), 1e-2, device=DEV), torch.ones((1,), dtype=torch.int64, device=DEV)
    results = []
    side = torch.cuda.Stream()
    for raw in (None, side, side.cuda_stream):
        p, m, v = start.clone(), torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
        group = bd.AdamWGroup([p], [grad], [m], [v])
        address, nbytes = group.plan_device.data_ptr(), group.plan_device.numel()
        if raw is not None:
            _busy(side)
        bd.adamw(group, lr, step, stream=raw)
        del group
        if raw is not None:
            assert _not_handed_on(address, nbytes)
        torch.cuda.synchronize()
        results.append((p, m, v))
    for other in results[1:]:
        assert all(torch.equal(t, u) for t, u in zip(results[0], other))


@pytest.mark.parametrize("grouped", [False, True])
def test_a_table_dropped_after_a_call_on_another_stream(bd, grouped):
    out, inn, T = 136, 64, 40
    a, b, scale, x, y0 = ref64.make([16, 20], out, inn, T, seed=3)
    scale, tok = scale.tolist(), [t % 2 for t in range(T)]
    side = torch.cuda.Stream()
    want = bd.lora_multitenant(x, bd.LoraTable(a, b, scale), tok, y0=y0)
    want_dx = bd.lora_multitenant_backward(y0, None, None, bd.LoraTable(a, b, scale), tok, None)
    for current in (False, True):
        got = []
        for backward in (False, True):
            table = bd.LoraTable(a, b, scale)
            address = table.scale.data_ptr()
            ws = bd.new_workspace(1 << 20, DEV)
            y, dx = torch.empty_like(y0), torch.empty_like(x)
            _busy(side)
            with torch.cuda.stream(side if current else torch.cuda.current_stream()):
                s = None if current else side
                if backward:
                    bd.lora_multitenant_backward(y0, None, None, table, tok, None, dx=dx, workspace=ws, stream=s)
                elif grouped:
                    bd.lora_multitenant_group(x, bd.LoraGroup([table], [out]), tok, y0s=[y0], ys=[y], workspace=ws, stream=s)
                else:
                    bd.lora_multitenant(x, table, tok, y0=y0, y=y, workspace=ws, stream=s)
            del table
            assert _not_handed_on(address, 8)
            torch.cuda.synchronize()
            got.append(dx if backward else y)
        assert torch.equal(got[0], want) and torch.equal(got[1], want_dx)
