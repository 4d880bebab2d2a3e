"""CPU-side checks of the low-rank adapters and of AdamW: every bad argument is found on the host before anything is enqueued (fake
addresses, never dereferenced; no GPU needed)."""
import ctypes
import os

import pytest

A = 0x100000                                            # a fake, 256-byte aligned device address; multiples of it lie apart


@pytest.fixture(scope="module")
def bd():
    from paper_2402_10193_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2402_10193_amd import build
        build.build_library()
    binding.lib()
    return binding


def _i32(*v):
    return (ctypes.c_int32 * max(len(v), 1))(*v)


def _ptrs(*v):
    return (ctypes.c_void_p * max(len(v), 1))(*v)


def test_workspace_sizes(bd):
    f, b = bd.lora_workspace_bytes, bd.lora_backward_workspace_bytes
    # the order of the tokens, then up to 8 partial sums of h in rows of whole 16 ranks, each rounded up to 256 bytes
    assert f(1, 1, 1) == 256 + 8 * 16 * 4
    assert f(100, 3, 17) == 512 + 8 * 3 * 100 * 32 * 4
    assert f(65535, 1, 256) == 262144 + 65535 * 256 * 4
    assert f(0, 1, 8) == 0 and f(1, 4, 8) == 0 and f(1, 0, 8) == 0 and f(1, 1, 0) == 0 and f(1, 1, 257) == 0 and f(65536, 1, 1) == 0
    # g and h as operands (2 KB per 16 ranks and chunk of 32 tokens; 3 chunks and one more per tenant), a number per chunk, and 3 parts
    # of the gradients of one adapter (one for 32 tokens, 32 at most)
    assert b(100, 40, 64, 5, 17) == 512 + 8 * 100 * 32 * 4 + 2 * (8 * 2 * 2048 + 256) + 3 * 32 * (40 + 64) * 4
    assert b(0, 40, 64, 1, 17) == 0 and b(1, 40, 65, 1, 17) == 0 and b(1, -1, 64, 1, 1) == 0 and b(1, 40, 64, 1, 0) == 0 and b(1, 40, 64, 0, 1) == 0


def test_forward_argument_errors(bd):
    L = bd.lib()
    need = bd.lora_workspace_bytes(3, 1, 16)

    def call(x=A, a=_ptrs(2 * A, 3 * A), b=_ptrs(4 * A, 5 * A), r=_i32(16, 8), s=6 * A, tok=_i32(0, 1, 1), y0=7 * A, y=8 * A, h=9 * A, ld=16,
             T=3, out=40, inn=64, nt=2, ws=10 * A, nb=need):
        return L.bd_lora_multitenant(x, a, b, r, s, tok, y0, y, h, ld, T, out, inn, nt, ws, nb, 0)

    assert call(T=-1) == 2 and call(T=65536) == 2 and call(out=-1) == 2 and call(inn=48) == 2 and call(inn=-32) == 2 and call(nt=-1) == 2
    assert call(out=(1 << 24) + 1) == 2 and call(inn=(1 << 24) + 32) == 2
    assert call(r=_i32(257, 8)) == 2 and call(r=_i32(16, -1)) == 2 and call(ld=15) == 2
    assert call(x=0) == 1 and call(a=None) == 1 and call(b=None) == 1 and call(r=None) == 1 and call(s=0) == 1 and call(tok=None) == 1 and call(y=0) == 1
    assert call(a=_ptrs(2 * A, None)) == 1 and call(b=_ptrs(None, 5 * A)) == 1
    assert call(x=A + 8) == 3 and call(y=8 * A + 2) == 3 and call(y0=7 * A + 8) == 3 and call(a=_ptrs(2 * A + 8, 3 * A)) == 3
    assert call(b=_ptrs(4 * A, 5 * A + 2)) == 3 and call(h=9 * A + 2) == 3 and call(s=6 * A + 1) == 3
    assert call(tok=_i32(0, 2, 1)) == 4 and call(tok=_i32(-1, 0, 1)) == 4
    assert call(ws=0) == 5 and call(nb=need - 1) == 5 and call(ws=10 * A + 16) == 5
    assert call(y=A + 16) == 8 and call(y=2 * A) == 8 and call(y=5 * A + 32) == 8          # over x, an A, a B
    assert call(y=7 * A + 16) == 8                                                          # over y0, but not y0 itself
    assert call(h=8 * A) == 8 and call(h=7 * A + 16) == 8 and call(h=A) == 8 and call(h=4 * A) == 8
    assert call(y=6 * A) == 8 and call(h=6 * A + 4) == 8                                    # over the scales
    assert call(T=0, x=0, a=None, y=0) == 0
    # only tenants with tokens count: the other's rank and pointers are not looked at, and what is not needed may be missing
    assert call(r=_i32(999, 8), a=_ptrs(None, None), tok=_i32(1, 1, 1)) == 1
    # no adapter in the call: nothing but y0 and y is needed, and in place nothing is done
    assert call(r=_i32(0, 0), a=_ptrs(None, None), b=_ptrs(None, None), x=0, s=0, h=0, ws=0, nb=0, y0=8 * A) == 0


def test_forward_group_argument_errors(bd):
    L = bd.lib()
    need = bd.lora_workspace_bytes(2, 2, 16)
    sizes = (ctypes.c_int64 * 3)(40, 48, 56)

    def call(n=2, a=_ptrs(2 * A, 3 * A), b=_ptrs(4 * A, 5 * A), r=_i32(16, 16), s=_ptrs(6 * A, 6 * A + 64), y0=_ptrs(7 * A, None), y=_ptrs(8 * A, 9 * A),
             h=_ptrs(11 * A, 12 * A), ld=16, out=sizes, ws=10 * A, nb=need):
        return L.bd_lora_multitenant_group(n, A, a, b, r, s, _i32(0, 0), y0, y, h, ld, 2, out, 64, 1, ws, nb, 0)

    assert call(n=0) == 2 and call(n=4) == 2 and call(out=None) == 1 and call(s=None) == 1 and call(y=None) == 1
    assert call(y=_ptrs(8 * A, None)) == 1 and call(s=_ptrs(6 * A, None)) == 1
    assert call(y=_ptrs(8 * A, 8 * A + 16)) == 8 and call(y=_ptrs(8 * A, 7 * A)) == 8       # one y over another, over another's y0
    assert call(h=_ptrs(11 * A, 11 * A)) == 8 and call(h=_ptrs(11 * A, 8 * A)) == 8
    assert call(nb=need - 1) == 5 and call(ld=15) == 2


def test_backward_argument_errors(bd):
    L = bd.lib()
    need = bd.lora_backward_workspace_bytes(3, 40, 64, 2, 16)

    def call(dy=A, x=2 * A, h=3 * A, ld=16, a=_ptrs(4 * A, 5 * A), b=_ptrs(6 * A, 7 * A), r=_i32(16, 8), s=8 * A, tok=_i32(0, 1, 1), dx0=9 * A,
             dx=10 * A, da=_ptrs(11 * A, 12 * A), db=_ptrs(13 * A, 14 * A), acc=0, T=3, out=40, inn=64, nt=2, ws=15 * A, nb=need):
        return L.bd_lora_multitenant_backward(dy, x, h, ld, a, b, r, s, tok, dx0, dx, da, db, acc, T, out, inn, nt, ws, nb, 0)

    assert call(T=-1) == 2 and call(T=65536) == 2 and call(out=-1) == 2 and call(inn=40) == 2 and call(nt=-1) == 2
    assert call(r=_i32(257, 8)) == 2 and call(r=_i32(16, -1)) == 2 and call(ld=15) == 2
    assert call(dy=0) == 1 and call(x=0) == 1 and call(h=0) == 1 and call(s=0) == 1 and call(r=None) == 1 and call(tok=None) == 1
    assert call(a=None) == 1 and call(b=_ptrs(6 * A, None)) == 1 and call(a=_ptrs(None, 5 * A)) == 1
    for name, at in (("dy", 1), ("x", 2), ("dx0", 9), ("dx", 10)):
        assert call(**{name: at * A + 8}) == 3, name
    assert call(h=3 * A + 2) == 3 and call(s=8 * A + 2) == 3 and call(da=_ptrs(11 * A + 2, 12 * A)) == 3 and call(db=_ptrs(13 * A, 14 * A + 2)) == 3
    assert call(a=_ptrs(4 * A + 8, 5 * A)) == 3 and call(b=_ptrs(6 * A, 7 * A + 2)) == 3
    assert call(tok=_i32(0, 2, 1)) == 4 and call(tok=_i32(0, -1, 1)) == 4
    assert call(ws=0) == 5 and call(nb=need - 1) == 5 and call(ws=15 * A + 128) == 5
    # what is written over what is read, or over something else that is written: the same gradient for two tenants among it
    assert call(dx=A) == 8 and call(dx=2 * A + 32) == 8 and call(dx=9 * A + 16) == 8 and call(dx=4 * A) == 8 and call(dx=6 * A) == 8
    assert call(da=_ptrs(11 * A, 11 * A)) == 8 and call(da=_ptrs(11 * A, 11 * A + 16 * 64 * 4 - 16)) == 8 and call(db=_ptrs(11 * A, 14 * A)) == 8
    assert call(da=_ptrs(10 * A, 12 * A)) == 8 and call(da=_ptrs(3 * A, 12 * A)) == 8 and call(db=_ptrs(2 * A, 14 * A)) == 8
    assert call(dx=8 * A) == 8 and call(da=_ptrs(8 * A + 4, 12 * A)) == 8                   # over the scales
    # the gradients of a tenant without a token are checked too: they are set to zero
    one = _i32(1, 1, 1)
    assert call(tok=one, da=_ptrs(12 * A, 12 * A)) == 8 and call(tok=one, r=_i32(300, 8)) == 2 and call(tok=one, da=_ptrs(11 * A + 2, 12 * A)) == 3
    assert call(T=0, dy=0, x=0, h=0, a=None, b=None, da=None, db=None, ws=0, nb=0, dx=0, dx0=0) == 0


def test_adamw_argument_errors(bd):
    L = bd.lib()
    numel = lambda *v: (ctypes.c_int64 * max(len(v), 1))(*v)
    size_of = L.bd_adamw_plan_bytes
    nbytes = size_of(2, numel(300, 7))
    assert size_of(2, numel(30000, 7)) > nbytes > size_of(1, numel(300)) > size_of(0, None) > 0
    assert size_of(-1, None) == 0 and size_of(1048577, None) == 0 and size_of(1, None) == 0
    assert size_of(1, numel(-1)) == 0 and size_of(1, numel((1 << 35) + 1)) == 0 and size_of(200, numel(*([1 << 35] * 200))) == 0
    plan = (ctypes.c_uint64 * (nbytes // 8 + 1))()

    def make(to=plan, size=nbytes, n=2, p=_ptrs(A, 2 * A), p16=_ptrs(3 * A, None), g=_ptrs(4 * A, 5 * A), m=_ptrs(6 * A, 7 * A), v=_ptrs(8 * A, 9 * A),
             ms=_ptrs(10 * A, 11 * A), vs=_ptrs(12 * A, 13 * A), count=numel(300, 7)):
        return L.bd_adamw_plan(to, size, n, p, p16, g, 0, m, v, ms, vs, count)

    assert make() == 0 and make(ms=None, vs=None) == 0 and make(p16=None) == 0
    assert make(n=-1) == 2 and make(count=numel(300, -1)) == 2 and make(count=numel(300, (1 << 35) + 1)) == 2
    assert make(to=None) == 1 and make(p=None) == 1 and make(g=None) == 1 and make(m=None) == 1 and make(v=None) == 1 and make(count=None) == 1
    assert make(ms=None) == 1 and make(vs=None) == 1 and make(p=_ptrs(A, None)) == 1 and make(g=_ptrs(None, 5 * A)) == 1
    assert make(m=_ptrs(None, 7 * A)) == 1 and make(v=_ptrs(8 * A, None)) == 1 and make(vs=_ptrs(12 * A, None)) == 1
    assert make(p=_ptrs(A + 4, 2 * A)) == 3 and make(g=_ptrs(4 * A, 5 * A + 8)) == 3 and make(m=_ptrs(6 * A + 1, 7 * A)) == 3
    assert make(p16=_ptrs(3 * A + 2, None)) == 3 and make(ms=_ptrs(10 * A + 2, 11 * A)) == 3
    assert make(size=nbytes - 1) == 5
    assert make(p=_ptrs(A, A)) == 8 and make(m=_ptrs(6 * A, 6 * A + 256)) == 8 and make(g=_ptrs(A + 512, 5 * A)) == 8
    assert make(p16=_ptrs(3 * A, 4 * A)) == 8 and make(vs=_ptrs(10 * A + 4, 13 * A)) == 8
    assert make(g=_ptrs(4 * A, 4 * A)) == 0                                                 # read twice is no overlap
    assert make(p=_ptrs(None, 2 * A), g=_ptrs(None, 5 * A), count=numel(0, 7)) == 0         # nothing of an empty tensor is looked at

    step = lambda p=plan, size=nbytes, dev=16 * A, lr=14 * A, t=15 * A, gs=0, skip=0, b1=0.9, b2=0.999, eps=1e-8, wd=0.0: L.bd_adamw(p, size, dev, lr, t, gs, skip, b1, b2, eps, wd, 0)
    assert make() == 0
    assert step(p=None) == 1 and step(dev=0) == 1 and step(dev=16 * A + 8) == 3 and step(lr=0) == 1 and step(t=0) == 1
    assert step(lr=14 * A + 2) == 3 and step(t=15 * A + 4) == 3 and step(gs=A + 1) == 3 and step(skip=A + 2) == 3
    assert step(size=8) == 9 and step(size=nbytes - 8) == 9
    junk = (ctypes.c_uint64 * 64)(*([7] * 64))
    assert step(p=junk, size=512) == 9
    nan = float("nan")
    for bad in (dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=nan), dict(eps=-1e-8), dict(eps=nan), dict(wd=-1.0), dict(b1=nan), dict(wd=nan)):
        assert step(**bad) == 7, bad
    assert make(n=0) == 0 and step(lr=0, t=0) == 0


def test_binding_refusals(bd):
    """What the binding finds without the library: wrong devices, types and shapes."""
    import torch
    h = lambda *s: torch.zeros(s, dtype=torch.float16)
    with pytest.raises(ValueError):
        bd.LoraTable([h(4, 32)], [h(8, 4)], [1.0])                     # not on a device
    with pytest.raises(ValueError):
        bd.LoraTable([None], [h(8, 4)], [1.0])
    with pytest.raises(ValueError):
        bd.LoraTable([None, None], [None], [1.0, 1.0])
    with pytest.raises(ValueError):
        bd.lora_multitenant(h(1, 32), None, [0])
    with pytest.raises(ValueError):
        bd.AdamWGroup([torch.zeros(4)], [torch.zeros(4)], [torch.zeros(4)], [torch.zeros(4)])
    with pytest.raises(ValueError):
        bd.AdamWGroup([], [], [], [], exp_avg_scales=[])
    with pytest.raises(TypeError):
        bd._tok_pointer(torch.zeros(3, dtype=torch.int64), 3)
    with pytest.raises(ValueError):
        bd._tok_pointer([0, 1], 3)


def test_adamw_values_argument_errors(bd):
    f = bd.lib().bd_adamw_values
    assert f(A, -1, 0, 2 * A, 0) == 2 and f(A, (1 << 35) + 1, 0, 2 * A, 0) == 2
    assert f(0, 8, 0, 2 * A, 0) == 1 and f(A, 8, 0, 0, 0) == 1 and f(A + 8, 8, 0, 2 * A, 0) == 3 and f(A, 8, 0, 2 * A + 8, 0) == 3
    assert f(A, 64, 0, A + 32, 0) == 8 and f(0, 0, 0, 0, 0) == 0
