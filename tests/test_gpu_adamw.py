"""AdamW over many tensors at once (bd_adamw) against the formula in 64 bits: binary32 and 8-bit states, binary32 and binary16
gradients, tensors of one element to several workgroups, a skipped step, overflowed gradients, captured and replayed steps."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2402_10193_amd import binding as bd          # noqa: E402

DEV = "cuda"
U = 2.0 ** -24
SIZES = [1, 3, 4, 255, 256, 257, 1023, 4096, 4097, 10001, 0, 65536, 70003]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    bd.lib()


def code_values(fraction_bits):
    top = 1 << fraction_bits
    return [float(f) if e == 0 else float((top + f) << (e - 1)) for e in range(8) for f in range(top)]


M_VALUES = torch.tensor(code_values(4) + [-v for v in code_values(4)], dtype=torch.float64)
V_VALUES = torch.tensor(code_values(5), dtype=torch.float64)


def drawn(n, step):
    k = (np.arange(n, dtype=np.uint64) + np.uint64(step * 0x9E3779B9)) & np.uint64(0xFFFFFFFF)
    mask = np.uint64(0xFFFFFFFF)
    k = (k * np.uint64(0xD1B54A33)) & mask
    k = ((k ^ (k >> np.uint64(15))) * np.uint64(0xB5297A4D)) & mask
    k = ((k ^ (k >> np.uint64(16))) * np.uint64(0x9E3779B9)) & mask
    return torch.from_numpy((k >> np.uint64(14)).astype(np.float64) / 2 ** 18)


def blocks(n):
    return -(-n // 256)


def per_element(scales, n):
    return scales.repeat_interleave(256)[:n]


class Problem:
    def __init__(self, sizes, bits, grad, seed, copies=True):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        normal = lambda n, std: torch.empty(n, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=g)
        self.sizes, self.bits = sizes, bits
        self.p = [normal(n, 0.05) for n in sizes]
        self.g = [normal(n, 1e-2).to(torch.float16 if grad == "f16" else torch.float32) for n in sizes]
        self.p16 = [torch.full((n,), float("nan"), dtype=torch.float16, device=DEV) if copies and i % 3 != 2 else None for i, n in enumerate(sizes)]
        if bits == 32:
            self.m, self.v = [normal(n, 1e-3) for n in sizes], [normal(n, 1e-2).square() for n in sizes]
            self.ms = self.vs = None
        else:
            byte = lambda n: torch.randint(0, 256, (n,), dtype=torch.uint8, device=DEV, generator=g)
            self.m, self.v = [byte(n) for n in sizes], [byte(n) for n in sizes]
            self.ms = [normal(blocks(n), 1e-6).abs() for n in sizes]
            self.vs = [normal(blocks(n), 3e-6).abs() for n in sizes]
        self.group = bd.AdamWGroup(self.p, self.g, self.m, self.v, params_f16=self.p16 if copies else None, exp_avg_scales=self.ms,
                                   exp_avg_sq_scales=self.vs)

    def states(self, i):
        """m and v of tensor i in 64 bits, on the CPU."""
        m, v = self.m[i].cpu(), self.v[i].cpu()
        if self.bits == 32:
            return m.double(), v.double()
        n = self.sizes[i]
        return M_VALUES[m.long()] * per_element(self.ms[i].cpu().double(), n), (V_VALUES[v.long()] * per_element(self.vs[i].cpu().double(), n)) ** 2


def one(v, dtype=torch.float32):
    return torch.full((1,), v, dtype=dtype, device=DEV)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "f16"])
@pytest.mark.parametrize("step,scaled", [(1, False), (7, True), (100000, True)])
def test_step(bits, grad, step, scaled):
    print(f"adamw bits={bits} grad={grad} step={step}", flush=True)
    prob = Problem(SIZES, bits, grad, seed=step % 97)
    lr, b1, b2, eps, wd = 3e-3, 0.9, 0.99, 1e-8, 0.05
    b1f, b2f = (float(np.float32(b)) for b in (b1, b2))
    before = [(p.cpu().double(), *prob.states(i)) for i, p in enumerate(prob.p)]
    grads = [g.cpu().double() * (0.125 if scaled else 1.0) for g in prob.g]
    bd.adamw(prob.group, one(lr), one(step, torch.int64), beta1=b1, beta2=b2, eps=eps, weight_decay=wd, grad_scale=one(0.125) if scaled else None)
    torch.cuda.synchronize()
    for i, n in enumerate(SIZES):
        p, m, v = before[i]
        g = grads[i]
        # binary32: the constants are rounded (2^-24 each), then 3 roundings; 8 bits: the values read have 2 more
        m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        m_size = b1 * m.abs() + (1 - b1) * g.abs()
        m_off, v_off = 6 * U * m_size, 8 * U * v1
        denominator = v1.sqrt() / np.sqrt(1 - b2 ** step) + eps
        rate = float(np.float32(lr)) / (1 - b1 ** step)
        move = rate * m1 / denominator
        p1 = p * (1 - float(np.float32(lr)) * wd) - move
        # the square root halves v's error; 8 more roundings of the move, 4 of the parameter
        off = U * (4 * p.abs() + 14 * move.abs()) + rate * m_off / denominator
        assert ((prob.p[i].cpu().double() - p1).abs() <= off).all(), f"p of tensor {i} ({n})"
        if prob.p16[i] is not None:
            assert torch.equal(prob.p16[i], prob.p[i].half()), f"copy of tensor {i}"
        if n == 0:
            continue
        if bits == 32:
            assert ((prob.m[i].cpu().double() - m1).abs() <= m_off).all() and ((prob.v[i].cpu().double() - v1).abs() <= v_off).all()
            continue
        pad = blocks(n) * 256 - n
        top = torch.nn.functional.pad(m1.abs(), (0, pad)).view(-1, 256).amax(1) / 1984
        root = torch.nn.functional.pad(v1.sqrt(), (0, pad)).view(-1, 256).amax(1) / 4032
        assert ((prob.ms[i].cpu().double() - top).abs() <= 16 * U * top).all() and ((prob.vs[i].cpu().double() - root).abs() <= 16 * U * root).all()
        # the codes, wherever u is not so near a border that 2^-20 of it decides
        u = m1.abs() / per_element(top, n)
        cell = torch.exp2((torch.floor(torch.log2(u.clamp(min=1))) - 4).clamp(min=0))
        clear = ((u / cell) % 1 - 0.5).abs() > 2.0 ** -18 * 32
        got = M_VALUES[prob.m[i].cpu().long()]
        want = torch.round(u / cell) * cell * torch.sign(m1)
        assert clear.double().mean() > 0.99 and (got[clear] == want[clear]).all(), f"m codes of tensor {i}"
        assert ((got.abs() - u).abs() <= cell / 2 * (1 + 1e-3)).all()
        u = v1.sqrt() / per_element(root, n)
        cell = torch.exp2((torch.floor(torch.log2(u.clamp(min=1))) - 5).clamp(min=0))
        at = u / cell + drawn(n, step)
        clear = torch.minimum(at % 1, 1 - at % 1) > 2.0 ** -18 * 64
        got = V_VALUES[prob.v[i].cpu().long()]
        want = (torch.floor(at) * cell).clamp(1, 4032)
        assert clear.double().mean() > 0.99 and (got[clear] == want[clear]).all(), f"v codes of tensor {i}"
        assert ((got - u).abs() <= cell * (1 + 1e-3)).all()


def test_many_tensors():
    sizes = [(37 * i) % 900 + 1 for i in range(131)]
    for bits in (32, 8):
        prob = Problem(sizes, bits, "f32", seed=5, copies=False)
        before = [(p.cpu().double(), *prob.states(i)) for i, p in enumerate(prob.p)]
        bd.adamw(prob.group, one(1e-3), one(3, torch.int64), weight_decay=0.0)
        for i in range(len(sizes)):
            p, m, v = before[i]
            g = prob.g[i].cpu().double()
            m, v = 0.9 * m + 0.1 * g, 0.999 * v + 0.001 * g * g
            move = 1e-3 / (1 - 0.9 ** 3) * m / (v.sqrt() / np.sqrt(1 - 0.999 ** 3) + 1e-8)
            assert ((prob.p[i].cpu().double() - (p - move)).abs() <= 2.0 ** -20 * (p.abs() + move.abs() + 1e-3)).all(), i


def test_skip_and_empty():
    prob = Problem([300, 5], 8, "f32", seed=1)
    keep = [t.clone() for t in prob.p + prob.m + prob.v + prob.ms + prob.vs]
    bd.adamw(prob.group, one(1e-3), one(1, torch.int64), skip=one(1, torch.int32))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(keep, prob.p + prob.m + prob.v + prob.ms + prob.vs))
    bd.adamw(prob.group, one(1e-3), one(1, torch.int64), skip=one(0, torch.int32))
    assert not torch.equal(keep[0], prob.p[0])
    bd.adamw(bd.AdamWGroup([], [], [], []), one(1e-3), one(1, torch.int64))


def test_zero_state_and_zero_gradients():
    """The state before the first step is all zeros; elements whose gradient is zero stay where they are but for the decay."""
    n = 700
    p = torch.linspace(-1, 1, n, device=DEV)
    g = torch.zeros(n, device=DEV)
    g[256:300] = 0.5
    m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    ms, vs = (torch.zeros(3, device=DEV) for _ in range(2))
    start = p.clone()
    bd.adamw(bd.AdamWGroup([p], [g], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs]), one(0.1), one(1, torch.int64), weight_decay=0.0)
    assert torch.equal(p[:256], start[:256]) and torch.equal(p[300:], start[300:])
    assert ((start - p)[256:300] - 0.1).abs().max() < 1e-5
    assert (ms[[0, 2]] == 0).all() and (vs[[0, 2]] == 0).all() and (m[:256] == 0).all() and (v[300:] == 0).all()
    assert (m[256:300] == 127).all() and (v[256:300] == 255).all()


def test_not_finite():
    """An infinity or NaN: its element where states are binary32, its block of 256 where they are in 8 bits; nothing else."""
    for bad in (float("inf"), float("nan"), -float("inf")):
        for bits in (32, 8):
            prob, clean = Problem([1024], bits, "f32", seed=2), Problem([1024], bits, "f32", seed=2)
            prob.g[0][300] = bad
            for q in (prob, clean):
                bd.adamw(q.group, one(1e-3), one(2, torch.int64))
            other = torch.ones(1024, dtype=torch.bool, device=DEV)
            other[300] = False
            assert torch.equal(prob.p[0][other], clean.p[0][other]) and not torch.isfinite(prob.p[0][300])
            if bits == 8:
                other[256:512] = False
                m, v = prob.states(0)
                assert torch.isnan(m[256:512]).all() and torch.isnan(v[256:512]).all()
            assert torch.equal(prob.m[0][other], clean.m[0][other]) and torch.equal(prob.v[0][other], clean.v[0][other])


def test_blocks_of_tiny_states():
    n = 512
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    g[:256], g[256:] = 2.0 ** -120, 2.0 ** -40         # m below 2^-100, v underflows; both regular
    m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    ms, vs = (torch.zeros(2, device=DEV) for _ in range(2))
    bd.adamw(bd.AdamWGroup([p], [g], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs]), one(1e-3), one(1, torch.int64))
    assert float(ms[0]) == 0 and float(vs[0]) == 0 and (m[:256] == 0).all() and (v[:256] == 0).all()
    assert (m[256:] == 127).all() and (v[256:] == 255).all() and torch.isfinite(p).all()


def test_second_moment_follows_small_changes():
    """Gradients of constant size: v tends to g^2 although a step moves it by far less than a code step.  Rounding up with the
    fraction's probability keeps sqrt(v) right on average; squaring adds the variance: at most (1/32)^2 of v where it moves a whole
    step, in proportion to what it moves (0.05 % a step against 1.6 % at least), so at most 2^-10 * 0.0005 * 64 = 3e-5 a step against
    the 1e-3 a step by which v returns: 3 %.  4096 elements leave less than 1 % of chance."""
    n, steps = 4096 + 256, 2500
    p, g = torch.zeros(n, device=DEV), torch.full((n,), 1e-2, device=DEV)
    g[::256] = 0.1                                      # a large one in every block
    m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    ms, vs = (torch.zeros(blocks(n), device=DEV) for _ in range(2))
    group = bd.AdamWGroup([p], [g], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs])
    lr, step = one(0.0), torch.zeros((1,), dtype=torch.int64, device=DEV)
    for _ in range(steps):
        step += 1
        bd.adamw(group, lr, step)
    values = ((V_VALUES[v.cpu().long()] * per_element(vs.cpu().double(), n)) ** 2).view(-1, 256)[:, 1:]
    want = 1e-4 * (1 - 0.999 ** steps)
    assert abs(float(values.mean()) / want - 1) < 0.05


def test_replayed_from_a_graph():
    """A captured step counts on: the number of the step and the rate are read when it runs."""
    for bits in (32, 8):
        prob, eager = Problem([5000, 33], bits, "f32", seed=4), Problem([5000, 33], bits, "f32", seed=4)
        lr, step = one(1e-3), torch.zeros((1,), dtype=torch.int64, device=DEV)
        other = torch.zeros_like(step)
        bd.adamw(prob.group, lr, step, skip=one(1, torch.int32))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step += 1
            bd.adamw(prob.group, lr, step)
        step.zero_()
        for rep in range(4):
            for q in (prob, eager):
                for t in q.g:
                    t.mul_(0.9)
            lr.fill_(1e-3 * (rep + 1))
            graph.replay()
            torch.cuda.synchronize()
            other += 1
            bd.adamw(eager.group, lr, other)
            torch.cuda.synchronize()
            for u, w in zip(prob.p + prob.p16 + prob.m + prob.v, eager.p + eager.p16 + eager.m + eager.v):
                assert u is None or torch.equal(u, w), f"replay {rep}"


def test_values_of_codes():
    """Every code, both states, and lengths that are not whole."""
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).to(DEV)
    assert torch.equal(bd.adamw_values(codes, False).cpu().double(), M_VALUES) and torch.equal(bd.adamw_values(codes, True).cpu().double(), V_VALUES)
    for n in (1, 7, 8, 9, 2049, 100003):
        c = torch.randint(0, 256, (n,), dtype=torch.uint8, device=DEV)
        for second, table in ((False, M_VALUES), (True, V_VALUES)):
            assert torch.equal(bd.adamw_values(c, second).cpu().double(), table[c.cpu().long()]), n
    assert bd.adamw_values(codes[:0], True).numel() == 0
