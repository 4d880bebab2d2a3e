"""Low-rank adapters of many tenants at once (bd_lora_multitenant, _group, _backward) against the formula in 64 bits: ranks from 1 to
the largest, odd sizes, one token to several thousand, sorted and mixed batches, tenants without an adapter or without a token,
infinities, captured and replayed calls, and the calls together as a training step uses them."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

import lora_ref as ref64                                # noqa: E402
from gpu_util import TiledProblem                       # noqa: E402
from paper_2402_10193_amd import binding as bd          # noqa: E402

DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    bd.lib()


def _tokens(T, n, order, seed=5):
    rng = random.Random(seed)
    tok = [rng.randrange(n) for _ in range(T)]
    if order == "grouped":
        return sorted(tok)
    if order == "reversed":
        return sorted(tok, reverse=True)
    return tok


# (out, in, T, ranks of the tenants, order of the tokens)
FORWARD = [
    (64, 32, 1, [1], "mixed"),
    (1, 32, 3, [2, 0], "mixed"),
    (7, 64, 5, [3, 8], "mixed"),
    (130, 96, 16, [16], "grouped"),
    (128, 256, 17, [16], "grouped"),
    (513, 160, 33, [5, 17, 0, 31], "mixed"),
    (1000, 1024, 64, [8, 12, 24, 33], "reversed"),
    (257, 992, 100, [64, 1], "mixed"),
    (96, 4096, 130, [256, 200], "mixed"),
    (640, 2048, 512, [16] * 40, "mixed"),               # several pairs of launches
    (300, 512, 512, [20], "grouped"),                   # one tenant fills 32 tiles
    (777, 224, 513, [16, 40, 0, 9], "mixed"),           # records are jobs, order table
    (777, 224, 700, [16, 40, 0, 9], "grouped"),         # ... no table
    (512, 1024, 2100, [64, 129], "reversed"),
    (264, 96, 1500, [4] * 90, "mixed"),                 # more jobs than records
    (40, 11008, 600, [16, 16], "grouped"),
    (4104, 320, 4500, [30], "grouped"),
]


@pytest.mark.parametrize("case", FORWARD, ids=lambda c: f"{c[0]}x{c[1]}_T{c[2]}_n{len(c[3])}_{c[4]}")
@pytest.mark.parametrize("with_y0", [True, False])
def test_forward(case, with_y0):
    out, inn, T, ranks, order = case
    print(f"forward {case} y0={with_y0}", flush=True)
    a, b, scale, x, y0 = ref64.make(ranks, out, inn, T, seed=out + T)
    tok = _tokens(T, len(ranks), order)
    table = bd.LoraTable(a, b, scale)
    h = torch.full((T, max(ranks) + 3), 7.0, dtype=torch.float32, device=DEV)
    y = torch.full((T, out), float("nan"), dtype=torch.float16, device=DEV)
    got = bd.lora_multitenant(x, table, tok, y0=y0 if with_y0 else None, y=y, h=h)
    want, h_of, bound = ref64.forward(x, a, b, scale, tok, y0 if with_y0 else None, out)
    assert got is y
    ref64.check(y, want, bound, "y")
    untouched = torch.ones_like(h, dtype=torch.bool)
    for e, (rows, hh) in h_of.items():
        r = hh.shape[1]
        size = x[rows].double().abs() @ a[e].double().abs().t()
        ref64.check(h[rows, :r], hh, (inn / 8 + 16) * ref64.U32 * size + 1e-30, "h")
        untouched[rows, :r] = False
    assert (h[untouched] == 7.0).all()                  # nothing behind a token's rank
    again = bd.lora_multitenant(x, table, torch.tensor(tok, dtype=torch.int32), y0=y0 if with_y0 else None)
    assert torch.equal(again, y)                        # the same bits, from a CPU tensor of tenants too
    if with_y0:                                         # in place
        z = y0.clone()
        assert bd.lora_multitenant(x, table, tok, y0=z, y=z) is z
        assert torch.equal(z, y)


@pytest.mark.parametrize("T,order", [(1, "mixed"), (16, "mixed"), (70, "mixed"), (600, "mixed"), (900, "grouped")])
def test_group(T, order):
    outs, inn, ranks = [256, 61, 1100], 384, [[16, 0, 5, 33], [16, 4, 0, 1], [8, 0, 0, 70]]
    tok = _tokens(T, 4, order)
    mats = [ref64.make(r, o, inn, T, seed=31 + m) for m, (r, o) in enumerate(zip(ranks, outs))]
    x = mats[0][3]
    for n in (2, 3):
        group = bd.LoraGroup([bd.LoraTable(*m[:3]) for m in mats[:n]], outs[:n])
        hs = [torch.zeros((T, 70), dtype=torch.float32, device=DEV) for _ in range(n)]
        ys = bd.lora_multitenant_group(x, group, tok, y0s=[m[4] if i != 1 else None for i, m in enumerate(mats[:n])], hs=hs)
        for i in range(n):
            a, b, scale, _, y0 = mats[i]
            want, h_of, bound = ref64.forward(x, a, b, scale, tok, y0 if i != 1 else None, outs[i])
            ref64.check(ys[i], want, bound, f"y of matrix {i}")
            for e, (rows, hh) in h_of.items():
                size = x[rows].double().abs() @ a[e].double().abs().t()
                ref64.check(hs[i][rows, :hh.shape[1]], hh, (inn / 8 + 16) * ref64.U32 * size + 1e-30, "h")


def test_group_with_an_empty_matrix_and_h_alone():
    """A matrix without outputs gives its h all the same."""
    T, inn = 20, 64
    a, b, scale, x, y0 = ref64.make([3, 5], 40, inn, T, seed=3)
    tok = _tokens(T, 2, "mixed")
    empty = [torch.empty((0, t.shape[1]), dtype=torch.float16, device=DEV) for t in b]
    group = bd.LoraGroup([bd.LoraTable(a, b, scale), bd.LoraTable(a, empty, scale)], [40, 0])
    hs = [torch.zeros((T, 5), dtype=torch.float32, device=DEV) for _ in range(2)]
    ys = bd.lora_multitenant_group(x, group, tok, y0s=[y0, None], hs=hs)
    want, _, bound = ref64.forward(x, a, b, scale, tok, y0, 40)
    ref64.check(ys[0], want, bound, "y")
    assert ys[1].shape == (T, 0) and torch.equal(hs[0], hs[1])


def test_forward_edges():
    """No token, an empty reduction, no adapter anywhere, scales of adapters that are not there."""
    a, b, scale, x, y0 = ref64.make([4, 0], 24, 32, 6, seed=1)
    table = bd.LoraTable(a, b, scale)
    assert bd.lora_multitenant(x[:0], table, [], y0=y0[:0]).shape == (0, 24)
    none = bd.LoraTable([None, None], [None, None], torch.full((2,), float("nan"), device=DEV))
    assert torch.equal(bd.lora_multitenant(x, none, [0, 1, 0, 1, 1, 1], y0=y0), y0)
    assert torch.equal(bd.lora_multitenant(x, none, [0, 1, 0, 1, 1, 1], out=24), torch.zeros_like(y0))
    a0, b0 = [torch.empty((4, 0), dtype=torch.float16, device=DEV)], [b[0]]
    h = torch.ones((6, 4), dtype=torch.float32, device=DEV)
    y = bd.lora_multitenant(x[:, :0].contiguous(), bd.LoraTable(a0, b0, scale[:1]), [0] * 6, y0=y0, h=h)
    assert torch.equal(y, y0) and (h == 0).all()


def test_range_of_h():
    """h far beyond binary16, and far below it, in one tile; infinities stay with their token."""
    out, inn, T = 200, 256, 40
    a, b, scale, x, _ = ref64.make([16], out, inn, T, seed=9)
    a = [(a[0].float() * 1000).half()]                  # h up to 1e9
    size = torch.logspace(-6, 4.5, T, device=DEV)[:, None]
    x = (x.float() * size).half()
    small = [(b[0].float() * 1e-4).half()]
    y = bd.lora_multitenant(x, bd.LoraTable(a, small, scale), [0] * T, out=out)
    want, _, bound = ref64.forward(x, a, small, scale, [0] * T, None, out)
    keep = want.abs().amax(1) < 60000                   # what binary16 can hold
    assert keep.sum() > T // 2
    ref64.check(y[keep], want[keep], bound[keep], "y")
    x[3, 5] = float("inf")
    x[7, 0] = float("nan")
    z = bd.lora_multitenant(x, bd.LoraTable(a, small, scale), [0] * T, out=out)
    same = torch.tensor([t for t in range(T) if t not in (3, 7)], device=DEV)
    assert torch.equal(z[same].view(torch.int16), y[same].view(torch.int16)) and not torch.isfinite(z[3]).any() and torch.isnan(z[7]).all()


# (out, in, T, ranks, order)
BACKWARD = [
    (1, 32, 1, [1], "mixed"),
    (7, 64, 5, [3, 8], "mixed"),
    (130, 96, 31, [16], "grouped"),
    (513, 160, 33, [5, 17, 0, 31], "mixed"),
    (1003, 1024, 100, [8, 64, 24, 33], "reversed"),
    (129, 992, 300, [256, 200], "mixed"),
    (96, 128, 512, [7] * 70, "mixed"),                  # more jobs than records
    (777, 224, 700, [16, 40, 0, 9], "mixed"),
    (264, 2048, 1300, [64, 129], "grouped"),            # tokens in parts
    (1000, 96, 5000, [16], "grouped"),
    (40, 4096, 2500, [3, 2], "mixed"),
]


def _run_backward(case, dx0_given=True, accumulate=False, seed=0):
    out, inn, T, ranks, order = case
    a, b, scale, x, dy = ref64.make(ranks, out, inn, T, seed=out + T + seed)
    tok = _tokens(T, len(ranks), order, seed=seed)
    dy = (dy.float() * 0.01).half()
    dx0 = (torch.flip(x, (0,)).float() * 0.02).half() if dx0_given else None
    h = torch.full((T, max(ranks) + 1), 3.0, dtype=torch.float32, device=DEV)
    table = bd.LoraTable(a, b, scale)
    bd.lora_multitenant(x, table, tok, y0=torch.zeros((T, out), dtype=torch.float16, device=DEV), h=h)
    fill = 0.25 if accumulate else float("nan")
    da = [torch.full(w.shape, fill, dtype=torch.float32, device=DEV) if w is not None else None for w in a]
    db = [torch.full(w.shape, fill, dtype=torch.float32, device=DEV) if w is not None else None for w in b]
    dx = bd.lora_multitenant_backward(dy, x, h, table, tok, bd.LoraGrads(table, da, db), dx0=dx0, accumulate=accumulate)
    return a, b, scale, x, dy, tok, dx0, h, table, da, db, dx


@pytest.mark.parametrize("case", BACKWARD, ids=lambda c: f"{c[0]}x{c[1]}_T{c[2]}_n{len(c[3])}_{c[4]}")
@pytest.mark.parametrize("dx0_given,accumulate", [(True, False), (False, True)])
def test_backward(case, dx0_given, accumulate):
    print(f"backward {case} {dx0_given} {accumulate}", flush=True)
    a, b, scale, x, dy, tok, dx0, h, table, da, db, dx = _run_backward(case, dx0_given, accumulate)
    want, bound, grads = ref64.backward(dy, x, h, a, b, scale, tok, dx0)
    ref64.check(dx, want, bound, "dx")
    start = 0.25 if accumulate else 0.0
    for e in range(len(a)):
        if a[e] is None:
            continue
        if e not in grads:                              # no token: zeros, or what was there
            assert (da[e] == start).all() and (db[e] == start).all()
            continue
        ga, ga_bound, gb, gb_bound = grads[e]
        extra = 2.0 ** -23 * (0.25 + ga.abs()) if accumulate else 0.0
        ref64.check(da[e], ga + start, ga_bound + extra, f"dA of tenant {e}")
        extra = 2.0 ** -23 * (0.25 + gb.abs()) if accumulate else 0.0
        ref64.check(db[e], gb + start, gb_bound + extra, f"dB of tenant {e}")


def test_backward_parts_wanted():
    """Any of dx, dA and dB alone, absent gradients of single tenants, dx in place, and the same bits each way."""
    case = (264, 256, 900, [16, 20, 0, 4], "mixed")
    a, b, scale, x, dy, tok, dx0, h, table, da, db, dx = _run_backward(case)
    n = len(a)
    assert torch.equal(bd.lora_multitenant_backward(dy, None, None, table, tok, None, dx0=dx0), dx)
    z = dx0.clone()
    bd.lora_multitenant_backward(dy, None, None, table, tok, None, dx0=z, dx=z)
    assert torch.equal(z, dx)
    one = [torch.full_like(da[1], float("nan")) if e == 1 else None for e in range(n)]
    assert bd.lora_multitenant_backward(dy, x, None, table, tok, bd.LoraGrads(table, one, [None] * n), want_dx=False) is None
    assert torch.equal(one[1], da[1])
    other = [torch.full_like(db[3], float("nan")) if e == 3 else None for e in range(n)]
    bd.lora_multitenant_backward(dy, None, h, table, tok, bd.LoraGrads(table, [None] * n, other), want_dx=False)
    assert torch.equal(other[3], db[3])


def test_backward_without_tokens():
    a, b, scale, x, y0 = ref64.make([4, 9], 24, 32, 1, seed=1)
    table = bd.LoraTable(a, b, scale)
    da, db = ([torch.ones(w.shape, dtype=torch.float32, device=DEV) for w in ws] for ws in (a, b))
    grads = bd.LoraGrads(table, da, db)
    e = torch.empty((0, 24), dtype=torch.float16, device=DEV)
    bd.lora_multitenant_backward(e, x[:0], None, table, [], grads, accumulate=True)
    assert all((t == 1).all() for t in da + db)
    bd.lora_multitenant_backward(e, x[:0], None, table, [], grads)
    assert all((t == 0).all() for t in da + db)


def test_gradients_of_small_and_large_losses():
    """dy where g leaves binary16 on either side; a single token among zeros."""
    for size in (1e-7, 6e4):
        a, b, scale, x, dy = ref64.make([16, 5], 300, 128, 200, seed=77, b_std=0.05 if size < 1 else 3.0)
        dy = torch.zeros_like(dy) if size < 1 else dy.clamp(-1, 1)
        dy = (dy.float() * size).half() if size > 1 else dy
        dy[17] = size
        tok = _tokens(200, 2, "mixed")
        table = bd.LoraTable(a, b, scale)
        h = torch.zeros((200, 16), dtype=torch.float32, device=DEV)
        bd.lora_multitenant(x, table, tok, out=300, h=h)
        da, db = ([torch.empty(w.shape, dtype=torch.float32, device=DEV) for w in ws] for ws in (a, b))
        bd.lora_multitenant_backward(dy, x, h, table, tok, bd.LoraGrads(table, da, db), want_dx=False)
        _, _, grads = ref64.backward(dy, x, h, a, b, scale, tok, None)
        for e, (ga, ga_bound, gb, gb_bound) in grads.items():
            ref64.check(da[e], ga, ga_bound, f"dA {size}")
            ref64.check(db[e], gb, gb_bound, f"dB {size}")


def test_gradients_against_differences():
    """L = sum c y is linear in A, in B and in x: its central difference along any direction is the derivative, up to the rounding
    of y to binary16, at most 2^-11 of |c| |y| each way (and what binary32 adds, far below it)."""
    out, inn, T, ranks = 96, 160, 50, [6, 11]
    a, b, scale, x, dy = ref64.make(ranks, out, inn, T, seed=123)
    tok = _tokens(T, 2, "mixed")
    table = bd.LoraTable(a, b, scale)
    h = torch.zeros((T, 11), dtype=torch.float32, device=DEV)
    bd.lora_multitenant(x, table, tok, out=out, h=h)
    da, db = ([torch.empty(w.shape, dtype=torch.float32, device=DEV) for w in ws] for ws in (a, b))
    dx = bd.lora_multitenant_backward(dy, x, h, table, tok, bd.LoraGrads(table, da, db))

    def loss(xx, aa, bb):
        y = bd.lora_multitenant(xx, bd.LoraTable(aa, bb, scale), tok, out=out).double()
        return float((y * dy.double()).sum()), float((y.abs() * dy.double().abs()).sum())

    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    like = lambda t, std: (torch.empty(t.shape, device=DEV).normal_(0.0, std, generator=g)).half()
    for what in ("x", "a", "b"):
        d = [like(x, 1.0)] if what == "x" else [like(t, 0.1) for t in (a if what == "a" else b)]
        up, down = [], []
        for sign, to in ((1, up), (-1, down)):
            move = lambda ts: [(t.float() + sign * v.float()).half() for t, v in zip(ts, d)]
            to += [move([x])[0] if what == "x" else x, move(a) if what == "a" else a, move(b) if what == "b" else b]
        # the step that was really taken, after the rounding of the moved tensors
        step = [(p.double() - q.double()) / 2 for p, q in (zip(up[1], down[1]) if what == "a" else zip(up[2], down[2]) if what == "b" else [(up[0], down[0])])]
        grad = {"x": [dx], "a": da, "b": db}[what]
        derivative = sum(float((s * t.double()).sum()) for s, t in zip(step, grad))
        (l1, m1), (l0, m0) = loss(*up), loss(*down)
        slack = 2.0 ** -11 * (m1 + m0) / 2 + (2.0 ** -11 * sum(float((s.abs() * t.double().abs()).sum()) for s, t in zip(step, grad)) if what == "x" else 0.0)
        assert abs((l1 - l0) / 2 - derivative) <= 1.02 * slack, what
        assert abs(derivative) > 0.01 * slack


def _capture(run):
    run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    return graph


@pytest.mark.parametrize("T,order", [(6, "mixed"), (300, "mixed"), (900, "mixed"), (900, "grouped")])
def test_replayed_from_a_graph(T, order):
    """Forward and backward in one graph with a workspace each, replayed with new inputs between eager calls on workspaces of their own."""
    out, inn, ranks = 264, 512, [16, 5, 33, 0]
    a, b, scale, x, y0 = ref64.make(ranks, out, inn, T, seed=8)
    tok = torch.tensor(_tokens(T, 4, order), dtype=torch.int32)
    table = bd.LoraTable(a, b, scale)
    y, dx, h = torch.empty_like(y0), torch.empty_like(x), torch.zeros((T, 33), dtype=torch.float32, device=DEV)
    da, db = ([torch.empty(w.shape, dtype=torch.float32, device=DEV) if w is not None else None for w in ws] for ws in (a, b))
    grads = bd.LoraGrads(table, da, db)
    ws = [bd.new_workspace(bd.lora_workspace_bytes(T, 1, 33), DEV), bd.new_workspace(bd.lora_backward_workspace_bytes(T, out, inn, 4, 33), DEV)]

    def run():
        bd.lora_multitenant(x, table, tok, y0=y0, y=y, h=h, workspace=ws[0])
        bd.lora_multitenant_backward(y, x, h, table, tok, grads, dx=dx, workspace=ws[1])
    graph = _capture(run)
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    for rep in range(4):
        x.copy_(torch.empty_like(x, dtype=torch.float32).normal_(0.0, 1.0, generator=g))
        y0.copy_(torch.empty_like(y0, dtype=torch.float32).normal_(0.0, 1.0, generator=g))
        for t in [y, dx, h] + [v for v in da + db if v is not None]:
            t.fill_(float("nan"))
        for w in ws:
            w.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in [y, dx] + [v for v in da + db if v is not None]]
        h2 = torch.zeros_like(h)
        y2 = bd.lora_multitenant(x, table, tok, y0=y0, h=h2)
        da2, db2 = ([torch.empty_like(t) if t is not None else None for t in ts] for ts in (da, db))
        dx2 = bd.lora_multitenant_backward(y2, x, h2, table, tok, bd.LoraGrads(table, da2, db2))
        torch.cuda.synchronize()
        for u, v in zip(got, [y2, dx2] + [v for v in da2 + db2 if v is not None]):
            assert torch.equal(u, v), f"replay {rep}"


def test_two_streams_at_once():
    """Two calls at once on streams and workspaces of their own."""
    out, inn, T = 512, 1024, 300
    streams = [torch.cuda.Stream() for _ in range(2)]
    sets = []
    for k in range(2):
        a, b, scale, x, y0 = ref64.make([16, 8, 40], out, inn, T, seed=50 + k)
        sets.append((x, bd.LoraTable(a, b, scale), _tokens(T, 3, "mixed", seed=k), y0, torch.empty_like(y0),
                     bd.new_workspace(bd.lora_workspace_bytes(T, 1, 40), DEV)))
    want = [bd.lora_multitenant(x, t, tok, y0=y0) for x, t, tok, y0, _, _ in sets]
    torch.cuda.synchronize()
    for _ in range(20):
        for k, (x, t, tok, y0, y, ws) in enumerate(sets):
            bd.lora_multitenant(x, t, tok, y0=y0, y=y, workspace=ws, stream=streams[k])
    torch.cuda.synchronize()
    for k in range(2):
        assert torch.equal(sets[k][4], want[k])


def test_training_steps_beside_the_shared_projection(ref):
    """Two steps as a program makes them: the projection with its 1-bit deltas, the adapters on top of it in place, two micro-batches
    of gradients added up, AdamW on all of them at once, whose fp16 copies are the adapters of the next step."""
    out, inn, n = 272, 512, 3
    prob = TiledProblem(ref, out, inn, n, tag=("lora", "step"))
    ranks = [8, 16, 5]
    a, b, scale, _, _ = ref64.make(ranks, out, inn, 1, seed=21)
    table = bd.LoraTable(a, b, scale)
    p16 = a + b
    p32 = [t.float() for t in p16]
    grads32 = [torch.empty_like(t) for t in p32]
    m, v = ([torch.zeros_like(t) for t in p32] for _ in range(2))
    adam = bd.AdamWGroup(p32, grads32, m, v, params_f16=p16)
    grads = bd.LoraGrads(table, grads32[:n], grads32[n:])
    lr, step = torch.full((1,), 1e-2, device=DEV), torch.zeros((1,), dtype=torch.int64, device=DEV)
    m64, v64, p64 = ([t.double() for t in ts] for ts in (m, v, p32))
    for it in range(2):
        want = None
        for micro in range(2):
            T = (40, 23)[micro]
            tok = _tokens(T, n, "mixed", seed=10 * it + micro)
            x = prob.x(T, tag=("step", it, micro))
            y = bd.linear_multitenant_tiled(x, prob.w_tiled, out, prob.ttable, tok)
            base = y.clone()
            h = torch.zeros((T, 16), dtype=torch.float32, device=DEV)
            bd.lora_multitenant(x, table, tok, y0=y, y=y, h=h)
            w64, _, bound = ref64.forward(x, a, b, scale, tok, base, out)
            ref64.check(y, w64, bound, "y")
            dy = (y.float() * 1e-2).half()              # of the loss 0.005 sum y^2
            bd.lora_multitenant_backward(dy, x, h, table, tok, grads, want_dx=False, accumulate=micro > 0)
            _, _, g64 = ref64.backward(dy, x, h, a, b, scale, tok, None)
            part = [g64[e][0] for e in range(n)] + [g64[e][2] for e in range(n)]
            limit = [g64[e][1] for e in range(n)] + [g64[e][3] for e in range(n)]
            want = part if want is None else [u + w for u, w in zip(want, part)]
            total = limit if micro == 0 else [u + w for u, w in zip(total, limit)]
        for k in range(2 * n):
            ref64.check(grads32[k], want[k], total[k] + 2.0 ** -23 * want[k].abs(), f"gradient {k}")
        step += 1
        bd.adamw(adam, lr, step)
        t = it + 1
        for k in range(2 * n):
            g = grads32[k].double()
            m64[k] = 0.9 * m64[k] + 0.1 * g
            v64[k] = 0.999 * v64[k] + 0.001 * g * g
            move = 1e-2 / (1 - 0.9 ** t) * m64[k] / ((v64[k] / (1 - 0.999 ** t)).sqrt() + 1e-8)
            p64[k] = p64[k] * (1 - 1e-4) - move
            # 8 roundings of the move, 4 of the parameter; the second step carries the first one's on
            ref64.check(p32[k], p64[k], t * 2.0 ** -23 * (4 * p64[k].abs() + 16 * move.abs() + 0.2), f"parameter {k}")
            assert torch.equal(p16[k], p32[k].half())
