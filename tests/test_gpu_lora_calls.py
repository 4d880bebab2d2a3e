"""Calls of the low-rank adapters that lie between the ordinary ones: gradients of some tenants only, inputs that no wanted result needs."""
import pytest
import torch

import lora_ref as ref64

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def bd():
    from paper_2402_10193_amd import binding
    return binding


def _gradients(ranks, out, inn, da=None, db=None):
    """Gradients full of 7 for the tenants in `da` and `db` (all that have an adapter where not given)."""
    some = lambda which, e: ranks[e] > 0 and (which is None or e in which)
    return ([torch.full((r, inn), 7.0, device=DEV) if some(da, e) else None for e, r in enumerate(ranks)],
            [torch.full((out, r), 7.0, device=DEV) if some(db, e) else None for e, r in enumerate(ranks)])


@pytest.mark.parametrize("T", [4, 40, 600, 5000])
@pytest.mark.parametrize("mixed", [True, False])
def test_gradients_of_some_tenants(bd, T, mixed):
    """Frozen tenants among trained ones: no A of anyone and no B of a tenant whose dA is not wanted.  The gradients are right, and the bits
    those of the same call with every weight given."""
    print(f"gradients of some tenants T={T} mixed={mixed}", flush=True)
    out, inn, ranks = 264, 128, [8, 17, 0, 16]
    a, b, scale, x, dy = ref64.make(ranks, out, inn, T, seed=T)
    tok = [(5 * t + t // 7) % 4 for t in range(T)]
    tok = tok if mixed else sorted(tok)
    h = torch.randn((T, 17), generator=torch.Generator().manual_seed(1)).to(DEV)
    table = bd.LoraTable(a, b, scale)
    _, _, want = ref64.backward(dy, x, h, a, b, scale, tok, None)
    for want_a, want_b in (([0], [1]), ([3], []), ([0, 1], [3]), ([], [0])):
        part = bd.LoraTable(a, b, scale)
        for e in range(4):
            part.a_ptrs[e] = None
            if e not in want_a:
                part.b_ptrs[e] = None
        results = []
        for weights in (part, table):
            da, db = _gradients(ranks, out, inn, want_a, want_b)
            bd.lora_multitenant_backward(dy, x if want_a else None, h if want_b else None, weights, tok, bd.LoraGrads(weights, da, db), want_dx=False)
            results.append((da, db))
        (da, db), (da2, db2) = results
        for e in want_a:
            ref64.check(da[e], want[e][0], want[e][1], f"dA of tenant {e}")
            assert torch.equal(da[e], da2[e])
        for e in want_b:
            ref64.check(db[e], want[e][2], want[e][3], f"dB of tenant {e}")
            assert torch.equal(db[e], db2[e])


@pytest.mark.parametrize("T", [2, 20, 600])
@pytest.mark.parametrize("rank", [5, 16, 40])
def test_h_alone_needs_no_scales(bd, T, rank):
    """A matrix without outputs whose h is asked for, alone and beside another one: scales, y and B may be missing."""
    print(f"h alone T={T} rank={rank}", flush=True)
    inn, out = 96, 40
    a, b, scale, x, y0 = ref64.make([rank, 8], out, inn, T, seed=T + rank)
    tok = [t % 2 for t in range(T)]
    none = bd.LoraTable(a, [torch.empty((0, t.shape[1]), dtype=torch.float16, device=DEV) for t in b], scale)
    _, h_of, _ = ref64.forward(x, a, b, scale, tok, y0, out)
    for both in (False, True):
        tables = [bd.LoraTable(a, b, scale), none] if both else [none]
        group = bd.LoraGroup(tables, [out, 0] if both else [0])
        group.scale[group.n - 1] = None
        hs = [torch.zeros((T, max(rank, 8)), device=DEV) for _ in tables]
        ys = bd.lora_multitenant_group(x, group, tok, y0s=[y0, None] if both else [None], hs=hs)
        for e, (rows, want) in h_of.items():
            size = x[rows].double().abs() @ a[e].double().abs().t()
            for h in hs:
                ref64.check(h[rows, :want.shape[1]], want, (inn / 8 + 16) * ref64.U32 * size + 1e-30, f"h of tenant {e}")
        if both:
            want, _, bound = ref64.forward(x, a, b, scale, tok, y0, out)
            ref64.check(ys[0], want, bound, "y")


@pytest.mark.parametrize("T", [60, 900])
@pytest.mark.parametrize("out", [20, 33, 160])
@pytest.mark.parametrize("ranks", [[1, 2, 3, 4, 5, 6, 7], [17, 18, 8, 33, 39, 41]])
def test_gradients_of_ranks_without_whole_pieces(bd, T, out, ranks):
    """A last block of 16 ranks with fewer than 8 in it, and no other."""
    print(f"no whole pieces T={T} out={out} ranks={ranks}", flush=True)
    inn, n = 64, len(ranks)
    a, b, scale, x, dy = ref64.make(ranks, out, inn, T, seed=T + out)
    tok = [(3 * t) % n for t in range(T)]
    h = torch.randn((T, max(ranks)), generator=torch.Generator().manual_seed(2)).to(DEV)
    table = bd.LoraTable(a, b, scale)
    da, db = _gradients(ranks, out, inn)
    dx = bd.lora_multitenant_backward(dy, x, h, table, tok, bd.LoraGrads(table, da, db))
    want, bound, grads = ref64.backward(dy, x, h, a, b, scale, tok, None)
    ref64.check(dx, want, bound, "dx")
    for e, (ga, ga_bound, gb, gb_bound) in grads.items():
        ref64.check(da[e], ga, ga_bound, f"dA of tenant {e}")
        ref64.check(db[e], gb, gb_bound, f"dB of tenant {e}")


def _same_as_formula(got, want, what):
    """Infinities where the formula in 64 bits has them, with their signs, NaN where it has them, and no other."""
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN at {int(torch.isnan(got).sum())} places, {int(torch.isnan(want).sum())} by the formula"
    for bad in (float("inf"), -float("inf")):
        assert torch.equal(got == bad, want == bad), f"{what}: {bad} at {int((got == bad).sum())} places, {int((want == bad).sum())} by the formula"


@pytest.mark.parametrize("T,at", [(5, 3), (32, 0), (33, 32), (96, 70), (128, 127), (129, 128), (700, 699), (4200, 4199)])
@pytest.mark.parametrize("rank", [8, 24, 64])
def test_infinite_operands_of_the_gradients(bd, T, at, rank):
    """An infinity of h makes its column of dB infinite, one of g its row of dA: with the formula's sign, however many tiles of tokens there are."""
    print(f"infinite operands T={T} at={at} rank={rank}", flush=True)
    out, inn = 136, 160
    a, b, scale, x, dy = ref64.make([rank], out, inn, T, seed=T)
    h = torch.randn((T, rank), generator=torch.Generator().manual_seed(3)).to(DEV)
    h[at, 2], h[at, rank - 1] = float("inf"), -float("inf")
    table = bd.LoraTable(a, b, scale)
    _, db = _gradients([rank], out, inn)
    bd.lora_multitenant_backward(dy, None, h, table, [0] * T, bd.LoraGrads(table, [None], db), want_dx=False)
    _same_as_formula(db[0], float(scale[0]) * (dy.double().t() @ h.double()), "dB")
    dy[at, 7] = float("inf")                             # g of this token, all ranks, by the sign of B
    da, _ = _gradients([rank], out, inn)
    bd.lora_multitenant_backward(dy, x, None, table, [0] * T, bd.LoraGrads(table, da, [None]), want_dx=False)
    g = float(scale[0]) * (dy.double() @ b[0].double())
    _same_as_formula(da[0], g.t() @ x.double(), "dA")


@pytest.mark.parametrize("T", [20, 300, 3000])
@pytest.mark.parametrize("ranks", [[8], [16, 40], [64, 5, 130]])
@pytest.mark.parametrize("stride", [1, 3])
def test_ranks_of_very_different_size(bd, T, ranks, stride):
    """Every row of dA and column of dB by its own size: ranks up to 2^-30 of the strongest one in g, up to 2^-60 in h.  A value of g or h is kept to
    2^-22 of itself (two of the sums' 2^-23), or to 2^-38 of its rank's largest; the rest as in lora_ref."""
    print(f"ranks of very different size T={T} ranks={ranks}", flush=True)
    out, inn, n = 200, 96, len(ranks)
    a, b, scale, x, dy = ref64.make(ranks, out, inn, T, seed=T + n)
    b = [(t.float() * 2.0 ** (10 - 10 * (torch.arange(t.shape[1], device=DEV) % 4))).half() for t in b]
    h = torch.randn((T, max(ranks)), generator=torch.Generator().manual_seed(4)).to(DEV)
    h = h * 2.0 ** (20 - 20.0 * (torch.arange(max(ranks), device=DEV) % 4))
    tok = [(stride * t) % n for t in range(T)]
    table = bd.LoraTable(a, b, scale)
    da, db = _gradients(ranks, out, inn)
    bd.lora_multitenant_backward(dy, x, h, table, tok, bd.LoraGrads(table, da, db), want_dx=False)
    for e in sorted(set(tok)):
        r = ranks[e]
        rows = ref64.rows_of(tok, e, DEV)
        d, X, H, B, s = dy[rows].double(), x[rows].double(), h[rows, :r].double(), b[e].double(), float(scale[e])
        g, g_size, adds = s * (d @ B), abs(s) * (d.abs() @ B.abs()), len(rows) / 4 + 32
        bound = (out / 8 + 16 + adds) * ref64.U32 * (g_size.t() @ X.abs()) + 2.0 ** -38 * g.abs().amax(0)[:, None] * X.abs().sum(0)[None, :]
        ref64.check(da[e], g.t() @ X, bound, f"dA of tenant {e}")
        bound = adds * ref64.U32 * abs(s) * (d.abs().t() @ H.abs()) + 2.0 ** -38 * abs(s) * H.abs().amax(0)[None, :] * d.abs().sum(0)[:, None]
        ref64.check(db[e], s * (d.t() @ H), bound, f"dB of tenant {e}")


@pytest.mark.parametrize("T", [1, 2, 3, 40, 600])
@pytest.mark.parametrize("rank", [5, 8, 20, 61])
def test_infinite_inputs_give_what_the_formula_gives(bd, T, rank):
    """An infinity of A, B, x or dy meets finite values of both signs, some of them whole binary16 numbers: infinities with the formula's sign, by
    one launch, by tiles of 16 tokens and of 64, forward and backward."""
    print(f"infinite inputs T={T} rank={rank}", flush=True)
    out, inn, inf = 200, 160, float("inf")
    a, b, scale, x, dy = ref64.make([rank], out, inn, T, seed=rank + T)
    x[:, 1:] = 0                                         # h and g are products of two binary16 numbers, some of one
    x[::2, 0], a[0][::2, 0] = 1.0, 0.5
    a[0][a[0] == 0] = 0.25
    tok, s = [0] * T, float(scale[0])
    h = x.double() @ a[0].double().t()
    bad = b[0].clone()
    bad[130, rank - 1], bad[7, 0] = inf, -inf
    y = bd.lora_multitenant(x, bd.LoraTable(a, [bad], scale), tok, out=out)
    _same_as_formula(y, s * (h @ bad.double().t()), "y")
    g = s * (dy.double() @ b[0].double())
    bad = a[0].clone()
    bad[rank - 1, 130], bad[0, 7] = -inf, inf
    dx = bd.lora_multitenant_backward(dy, None, None, bd.LoraTable([bad], b, scale), tok, None)
    _same_as_formula(dx, g @ bad.double(), "dx")
    table = bd.LoraTable(a, b, scale)
    da, db = _gradients([rank], out, inn)
    bad = x.clone()
    bad[T - 1, 11], bad[0, 150] = inf, -inf
    bd.lora_multitenant_backward(dy, bad, None, table, tok, bd.LoraGrads(table, da, [None]), want_dx=False)
    _same_as_formula(da[0], g.t() @ bad.double(), "dA")
    bad = dy.clone()
    bad[T - 1, 199], bad[0, 100] = inf, -inf
    bd.lora_multitenant_backward(bad, None, h.float(), table, tok, bd.LoraGrads(table, [None], db), want_dx=False)
    _same_as_formula(db[0], s * (bad.double().t() @ h), "dB")


@pytest.mark.parametrize("T", [2, 40, 600])
@pytest.mark.parametrize("out", [5, 136])
def test_every_bit_of_tokens_without_an_adapter(bd, T, out):
    """All 65536 binary16 patterns among them, NaN of every kind, in y and in dx; the other tenant's tokens take part."""
    inn = 64
    a, b, scale, x, dy = ref64.make([8, 0], out, inn, T, seed=T)
    table, tok = bd.LoraTable(a, b, scale), [t % 2 for t in range(T)]
    for first in range(0, 65536, (T + 1) // 2 * out) if T > 2 else (0x0000, 0x7BFD, 0x7C00, 0x7D00, 0x7E01, 0xFBFF, 0xFC01, 0xFE55):
        y0 = ((torch.arange(T * out, device=DEV) + first) & 0xFFFF).to(torch.int32).to(torch.int16).view(torch.float16).view(T, out)
        y = bd.lora_multitenant(x, table, tok, y0=y0)
        assert torch.equal(y[1::2].view(torch.int16), y0[1::2].view(torch.int16)), f"y from {first:#x}"
    dx0 = torch.full((T, inn), 0x7C01, dtype=torch.int16, device=DEV).view(torch.float16)
    dx = bd.lora_multitenant_backward(dy, None, None, table, tok, None, dx0=dx0)
    assert torch.equal(dx[1::2].view(torch.int16), dx0[1::2].view(torch.int16))
