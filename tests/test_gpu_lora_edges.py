"""Edges of the low-rank adapters' calls: gradients with infinities in tokens whose other values are far below the rest, signs of zero
of tokens without an adapter, many tenants of one token, the routes of two tokens per tenant."""
import pytest
import torch

import lora_ref as ref64

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def bd():
    from paper_2402_10193_amd import binding
    return binding


def _adapters(ranks, out, inn, gen):
    a = [(torch.randn(r, inn, generator=gen) * inn ** -0.5).half().to(DEV) if r else None for r in ranks]
    b = [(torch.randn(out, r, generator=gen) * 0.2).half().to(DEV) if r else None for r in ranks]
    return a, b


@pytest.mark.parametrize("T,rank,chunk", [(96, 8, 1), (700, 8, 1), (4000, 64, 19), (20000, 8, 19)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_gradients_keep_what_is_not_finite(bd, T, rank, chunk, bad):
    """32 tokens whose dy (and h) are zero but for one value that is not finite, beside tokens of ordinary size: that value's rows of dA
    and columns of dB are not finite, all others are those without it."""
    gen = torch.Generator().manual_seed(5)
    out, inn, first = 256, 128, 32 * chunk
    a, b = _adapters([rank], out, inn, gen)
    table = bd.LoraTable(a, b, [1.0])
    x = torch.randn(T, inn, generator=gen).half().to(DEV)
    dy = torch.randn(T, out, generator=gen).half().to(DEV) * 64
    h = torch.randn(T, rank, generator=gen).to(DEV) * 4096
    dy[first:first + 32] = 0
    h[first:first + 32] = 0
    grads = lambda: ([torch.zeros(rank, inn, device=DEV)], [torch.zeros(out, rank, device=DEV)])
    (da,), (db,) = want = grads()
    bd.lora_multitenant_backward(dy, x, h, table, [0] * T, bd.LoraGrads(table, *want), want_dx=False)
    dy2, h2 = dy.clone(), h.clone()
    dy2[first + 8, 3] = bad                                 # g of this token is not finite
    h2[first + 18, 2] = bad                                  # dB's column 2
    (da2,), (db2,) = got = grads()
    bd.lora_multitenant_backward(dy2, x, h2, table, [0] * T, bd.LoraGrads(table, *got), want_dx=False)
    assert torch.isfinite(da).all() and torch.isfinite(db).all()
    assert not torch.isfinite(da2).any()
    assert not torch.isfinite(db2[:, 2]).any() and not torch.isfinite(db2[3]).any()
    rows = [r for r in range(out) if r != 3]
    for column in (0, 1, 3, 7):
        assert torch.equal(db2[rows, column], db[rows, column])


@pytest.mark.parametrize("T", [2, 40, 600])
def test_tokens_without_an_adapter_keep_their_bits(bd, T):
    gen = torch.Generator().manual_seed(6)
    a, b = _adapters([8, 0], 136, 64, gen)
    table = bd.LoraTable(a, b, [1.0, float("nan")])
    x = torch.randn(T, 64, generator=gen).half().to(DEV)
    y0 = torch.randn(T, 136, generator=gen).half().to(DEV)
    y0[:, ::7], y0[:, 1::7] = -0.0, 0.0
    y0[1, 5], y0[1, 6] = float("inf"), -float("inf")
    tok = [t % 2 for t in range(T)]
    y = bd.lora_multitenant(x, table, tok, y0=y0)
    assert torch.equal(y[1::2].view(torch.int16), y0[1::2].view(torch.int16))
    dx0 = torch.randn(T, 64, generator=gen).half().to(DEV)
    dx0[:, ::5] = -0.0
    dx = bd.lora_multitenant_backward(y0, None, None, table, tok, None, dx0=dx0)
    assert torch.equal(dx[1::2].view(torch.int16), dx0[1::2].view(torch.int16))


@pytest.mark.parametrize("per_tenant", [1, 2, 3])
@pytest.mark.parametrize("ranks", [[16, 8], [16, 0, 5, 1], [17, 16]])
def test_many_tenants_of_few_tokens(bd, ranks, per_tenant):
    """More (tenant, matrix) pairs than one launch takes; ranks and tokens on both sides of what one launch of both products takes."""
    gen = torch.Generator().manual_seed(7)
    n, out, inn = 150, 200, 96
    ranks = [ranks[e % len(ranks)] for e in range(n)]
    T = n * per_tenant
    tok = [(7 * t) % n for t in range(T)]
    a, b = _adapters(ranks, out, inn, gen)
    scale = torch.rand(n, generator=gen) + 0.5
    table = bd.LoraTable(a, b, scale)
    x = torch.randn(T, inn, generator=gen).half().to(DEV)
    y0 = torch.randn(T, out, generator=gen).half().to(DEV)
    h = torch.full((T, max(ranks)), 7.0, device=DEV)
    y = bd.lora_multitenant(x, table, tok, y0=y0, h=h)
    want, h_of, bound = ref64.forward(x, a, b, scale, tok, y0, out)
    ref64.check(y, want, bound, "y")
    for e, (rows, want_h) in h_of.items():
        size = x[rows].double().abs() @ a[e].double().abs().t()
        ref64.check(h[rows, :ranks[e]], want_h, (inn / 8 + 16) * ref64.U32 * size, f"h of tenant {e}")
    for t, e in enumerate(tok):
        assert (h[t, ranks[e]:] == 7.0).all()


@pytest.mark.parametrize("T,n", [(2000, 2), (9000, 3), (7000, 10), (13000, 16), (6000, 200), (3000, 256), (3000, 257), (24000, 2)])
def test_order_of_many_mixed_tokens(bd, T, n):
    """Tokens of every number of tenants in any order, on both sides of what one launch sorts: the same bits as of the tokens grouped by tenant."""
    gen = torch.Generator().manual_seed(8)
    out, inn = 136, 64
    a, b = _adapters([4] * n, out, inn, gen)
    table = bd.LoraTable(a, b, torch.rand(n, generator=gen))
    tok = torch.randint(0, n, (T,), generator=gen, dtype=torch.int32)
    tok[:n] = torch.arange(n, dtype=torch.int32)
    order = torch.sort(tok, stable=True).indices
    x = torch.randn(T, inn, generator=gen).half().to(DEV)
    dy = torch.randn(T, out, generator=gen).half().to(DEV)
    here = order.to(DEV)
    grads = lambda: ([torch.empty(4, inn, device=DEV) for _ in range(n)], [torch.empty(out, 4, device=DEV) for _ in range(n)])
    results = []
    for rows in (None, here):
        xs, ys, ts = (x, dy, tok) if rows is None else (x[rows].contiguous(), dy[rows].contiguous(), tok[order])
        h = torch.empty(T, 4, device=DEV)
        y = bd.lora_multitenant(xs, table, ts, y0=ys, h=h)
        g = grads()
        dx = bd.lora_multitenant_backward(ys, xs, h, table, ts, bd.LoraGrads(table, *g), dx0=xs)
        results.append((y, h, dx, *g))
    (y, h, dx, da, db), (y2, h2, dx2, da2, db2) = results
    assert torch.equal(y[here], y2) and torch.equal(h[here], h2) and torch.equal(dx[here], dx2)
    assert all(torch.equal(p, q) for p, q in zip(da + db, da2 + db2))
    e = int(tok[5])
    rows = (tok == e).nonzero()[:, 0].to(DEV)
    want, _, bound = ref64.forward(x[rows], a, b, table.scale, [e] * len(rows), dy[rows], out)
    ref64.check(y[rows], want, bound, "y")


@pytest.mark.parametrize("out,inn,T,ranks,mixed", [
    (40, 64, 700, [40, 129, 256, 1], True), (127, 96, 600, [17, 64], False), (1, 32, 2000, [33], False), (129, 160, 900, [250, 65], True),
    (1000, 128, 1030, [256, 96], False), (300, 4096, 520, [80, 0, 24], True), (8, 32, 65535, [3, 20, 1], True), (200, 64, 65535, [16], False)])
def test_ranks_and_rows_of_many_tokens(bd, out, inn, T, ranks, mixed):
    """Over 16 ranks at once, to the largest; rows below 128 features in and out; the most tokens of a call."""
    a, b, scale, x, y0 = ref64.make(ranks, out, inn, T, seed=out + T)
    gen = torch.Generator().manual_seed(9)
    tok = torch.randint(0, len(ranks), (T,), generator=gen, dtype=torch.int32)
    tok = (tok if mixed else tok.sort().values).tolist()
    table = bd.LoraTable(a, b, scale)
    h = torch.zeros(T, max(ranks), device=DEV)
    y = bd.lora_multitenant(x, table, tok, y0=y0, h=h)
    want, h_of, bound = ref64.forward(x, a, b, scale, tok, y0, out)
    ref64.check(y, want, bound, "y")
    dy = (torch.randn(T, out, generator=gen) * 0.01).half().to(DEV)
    dx0 = torch.randn(T, inn, generator=gen).half().to(DEV)
    da = [torch.empty(r, inn, device=DEV) if r else None for r in ranks]
    db = [torch.empty(out, r, device=DEV) if r else None for r in ranks]
    dx = bd.lora_multitenant_backward(dy, x, h, table, tok, bd.LoraGrads(table, da, db), dx0=dx0)
    want_dx, dx_bound, grads = ref64.backward(dy, x, h, a, b, scale, tok, dx0)
    ref64.check(dx, want_dx, dx_bound, "dx")
    for e, (ga, ga_bound, gb, gb_bound) in grads.items():
        ref64.check(da[e], ga, ga_bound, f"dA of tenant {e}")
        ref64.check(db[e], gb, gb_bound, f"dB of tenant {e}")


@pytest.mark.parametrize("T", [2, 40, 600])
@pytest.mark.parametrize("rank", [5, 8, 20, 61])
def test_weights_that_are_not_finite_stay_in_their_row(bd, T, rank):
    """A row of B reaches its own feature of y alone, a column of A its own feature of dx: all others have the same bits."""
    out, inn, row, column = 200, 160, 130, 77
    a, b, scale, x, y0 = ref64.make([rank], out, inn, T, seed=rank)
    a2, b2 = [a[0].clone()], [b[0].clone()]
    a2[0][:, column] = float("inf")
    b2[0][row] = float("nan")
    table, with_a, with_b = bd.LoraTable(a, b, scale), bd.LoraTable(a2, b, scale), bd.LoraTable(a, b2, scale)
    tok = [0] * T
    y, z = (bd.lora_multitenant(x, t, tok, y0=y0) for t in (table, with_b))
    others = [f for f in range(out) if f != row]
    assert torch.equal(y[:, others], z[:, others]) and torch.isnan(z[:, row]).all()
    dx, dz = (bd.lora_multitenant_backward(y0, None, None, t, tok, None, dx0=x) for t in (table, with_a))
    others = [f for f in range(inn) if f != column]
    assert torch.equal(dx[:, others], dz[:, others]) and not torch.isfinite(dz[:, column]).any()


def test_memory_of_a_call_belongs_to_its_stream(bd, monkeypatch):
    """Without a workspace a call allocates one: of its own stream, not of the current one, which may hand the memory on too early."""
    a, b, scale, x, y0 = ref64.make([16, 20], 136, 64, 40, seed=3)
    table = bd.LoraTable(a, b, scale)
    tok = [t % 2 for t in range(40)]
    want = bd.lora_multitenant(x, table, tok, y0=y0)
    want_dx = bd.lora_multitenant_backward(y0, None, None, table, tok, None, dx0=x)
    torch.cuda.synchronize()
    seen, make = [], bd.new_workspace
    monkeypatch.setattr(bd, "new_workspace", lambda n, device: (seen.append(torch.cuda.current_stream().cuda_stream), make(n, device))[1])
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        y = bd.lora_multitenant(x, table, tok, y0=y0, stream=stream)
        ys = bd.lora_multitenant_group(x, bd.LoraGroup([table], [136]), tok, y0s=[y0], stream=stream)
        dx = bd.lora_multitenant_backward(y0, None, None, table, tok, None, dx0=x, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(ys[0], want) and torch.equal(dx, want_dx)
    assert seen == [side.cuda_stream] * 6
