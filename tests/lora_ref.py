"""Low-rank adapters in 64 bits, tenant by tenant, and how far the library may be from them.

Bounds: a product of two binary16 numbers is exact in binary32; every addition of a sum rounds by at most 2^-23 of what has been
added up in magnitude so far (2^-24, twice that where the adder truncates).  A sum over n elements runs in eight wavefronts or
more, so that an element takes part in at most n / 8 + 16 additions; the value h (or g) that goes on into the next product is
kept to 2^-22 of itself, or to 2^-39 of the largest of its group.  A result in binary16 is rounded once: half a step, 2^-11 of the
value, or 2^-25 among the subnormal numbers.
"""
import torch

U32, U16 = 2.0 ** -23, 2.0 ** -11
TINY16 = 2.0 ** -25


def rows_of(tok, e, device):
    return torch.tensor([t for t, k in enumerate(tok) if k == e], dtype=torch.int64, device=device)


def make(ranks, out, inn, T, seed, device="cuda", x_std=1.0, b_std=0.05):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    n = lambda shape, std: torch.empty(shape, dtype=torch.float32, device=device).normal_(0.0, std, generator=g).half()
    a = [n((r, inn), inn ** -0.5 if inn else 1.0) if r else None for r in ranks]
    b = [n((out, r), b_std) if r else None for r in ranks]
    scale = torch.linspace(0.5, 2.0, max(len(ranks), 1), device=device)[:len(ranks)]
    return a, b, scale, n((T, inn), x_std), n((T, out), 1.0)


def forward(x, a, b, scale, tok, y0, out):
    """y, h (a list by tenant) and the bound of y, all in 64 bits."""
    T = x.shape[0]
    y = y0.double() if y0 is not None else torch.zeros((T, out), dtype=torch.float64, device=x.device)
    y = y.clone()
    size, h_of = y.abs(), {}
    count = 0
    for e in sorted(set(tok)):
        if a[e] is None:
            continue
        rows, A, B, s = rows_of(tok, e, x.device), a[e].double(), b[e].double(), float(scale[e])
        h = x[rows].double() @ A.t()
        h_of[e] = (rows, h)
        y[rows] += s * (h @ B.t())
        size[rows] += abs(s) * ((x[rows].double().abs() @ A.abs().t()) @ B.abs().t())
        count = max(count, A.shape[1] / 8 + 2 * (A.shape[0] + 16) + 32)
    return y, h_of, U16 * y.abs() + TINY16 + count * U32 * size


def check(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    over = (got - want).abs() > bound
    assert torch.isfinite(got).all(), f"{what}: not finite"
    assert not over.any(), f"{what}: {int(over.sum())} of {over.numel()} outside, worst {float(((got - want).abs() / bound).max()):.3g} times the bound"


def backward(dy, x, h, a, b, scale, tok, dx0):
    """dx and {tenant: (dA, dB)} with their bounds, in 64 bits; h: [T, >= rank] as the forward call left it."""
    T, inn, out = dy.shape[0], x.shape[1], dy.shape[1]
    dx = dx0.double().clone() if dx0 is not None else torch.zeros((T, inn), dtype=torch.float64, device=dy.device)
    size, grads = dx.abs(), {}
    count = 0.0
    for e in sorted(set(tok)):
        if a[e] is None:
            continue
        rows, A, B, s, r = rows_of(tok, e, dy.device), a[e].double(), b[e].double(), float(scale[e]), a[e].shape[0]
        d, X, H = dy[rows].double(), x[rows].double(), h[rows, :r].double()
        g, g_size = s * (d @ B), abs(s) * (d.abs() @ B.abs())
        dx[rows] += g @ A
        size[rows] += g_size @ A.abs()
        count = max(count, out / 8 + 16 + 2 * (r + 16) + 16)
        adds = len(rows) / 4 + 32
        da, db = g.t() @ X, s * (d.t() @ H)
        da_bound = (out / 8 + 16 + adds) * U32 * (g_size.t() @ X.abs()) + 2.0 ** -38 * g.abs().max() * X.abs().sum(0)[None, :]
        db_bound = adds * U32 * abs(s) * (d.abs().t() @ H.abs()) + 2.0 ** -38 * abs(s) * H.abs().max() * d.abs().sum(0)[:, None]
        grads[e] = (da, da_bound + 1e-30, db, db_bound + 1e-30)
    return dx, U16 * dx.abs() + TINY16 + count * U32 * size, grads
