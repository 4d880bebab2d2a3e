"""What the launches of the low-rank adapters would read, call by call, without a GPU: the host side built with stand-ins for the
launches (lora_records.cpp), fake addresses that nothing reads."""
import ctypes
import os
import subprocess

import pytest

A = 0x100000                                            # a fake, 256-byte aligned device address; multiples of it lie apart
SHRINK, EXPAND, OPERANDS, GRADIENTS, DECODE = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    from paper_2402_10193_amd import build
    here = os.path.dirname(os.path.abspath(__file__))
    lib = str(tmp_path_factory.mktemp("lora") / "lora_records.so")
    subprocess.run([build._hipcc(), "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", os.path.join(build.ROOT, "include"),
                    "-I", build.CSRC, os.path.join(here, "lora_records.cpp"), "-o", lib], check=True, capture_output=True, timeout=110)
    L = ctypes.CDLL(lib)
    i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
    L.lora_records.restype = i64
    L.bd_lora_backward_workspace_bytes.restype = sz
    L.bd_lora_backward_workspace_bytes.argtypes = [i64, i64, i64, i32, i32]
    L.bd_lora_multitenant_backward.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i64, i64, i64, i32, vp, sz, vp]
    return L


def _records(L, kind):
    to = (ctypes.c_int64 * (7 * 4096))()
    n = L.lora_records(to, 4096)
    assert n <= 4096
    return [r for r in (tuple(to[7 * i:7 * i + 7]) for i in range(n)) if r[0] in kind]


def _backward(L, T, ranks, a, b, da, db, dx, dx0=None, out=40, inn=64, tok=None):
    n = len(ranks)
    ptrs = lambda v: None if v is None else (ctypes.c_void_p * n)(*v)
    tok = tok if tok is not None else [t % n for t in range(T)]
    L.lora_records(None, 0)
    return L.bd_lora_multitenant_backward(A, 2 * A, 3 * A, max(ranks), ptrs(a), ptrs(b), (ctypes.c_int32 * n)(*ranks), 4 * A, (ctypes.c_int32 * T)(*tok),
                                          dx0, dx, ptrs(da), ptrs(db), 0, T, out, inn, n, 5 * A,
                                          L.bd_lora_backward_workspace_bytes(T, out, inn, n, max(ranks)), None)


@pytest.mark.parametrize("T", [3, 40, 600])
@pytest.mark.parametrize("sorted_tokens", [True, False])
def test_weights_of_tenants_without_a_wanted_gradient_are_not_read(host, T, sorted_tokens):
    """dx is not wanted, dA of tenant 0 only: the B of the others may be missing, and no launch reads it, nor what it would have given."""
    tok = [t % 3 for t in range(T)]
    tok = sorted(tok) if sorted_tokens else tok
    b0, wanted, other = 20 * A, 30 * A, 31 * A
    assert _backward(host, T, [8, 17, 16], None, [b0, None, None], [wanted, None, None], [None, other, None], None, tok=tok) == 0
    every = _records(host, {SHRINK, OPERANDS, GRADIENTS})
    shrink = [r for r in every if r[0] == SHRINK]
    assert shrink and all(r[1] == 0 and r[3] == b0 for r in shrink)
    sides = [r[4] for r in every if r[0] == OPERANDS]     # by tenant: g for tenant 0, h for tenant 1, none for tenant 2
    assert sides == [1, 2, 0]
    assert [(r[1], r[5], r[6]) for r in every if r[0] == GRADIENTS and (r[5] or r[6])] == [(0, wanted, 0), (1, 0, other)]
    # a missing B whose gradient of A is wanted is refused, and so is any where dx is wanted
    assert _backward(host, T, [8, 17, 16], None, [None, b0, b0], [wanted, None, None], None, None, tok=tok) == 1
    assert _backward(host, T, [8, 17, 16], [21 * A] * 3, [b0, None, b0], [wanted, None, None], None, 32 * A, tok=tok) == 1


@pytest.mark.parametrize("T", [3, 40, 600])
def test_all_of_g_is_prepared_where_dx_is_wanted(host, T):
    """dx adds up the parts of g where no launch before it has: with any dA wanted, g is whole for all tenants that have an adapter."""
    a, b, da = [21 * A, 22 * A, None], [20 * A, 23 * A, None], [None, 30 * A, None]
    assert _backward(host, T, [8, 17, 0], a, b, da, None, 32 * A) == 0
    every = _records(host, {SHRINK, EXPAND, OPERANDS, GRADIENTS})
    assert {r[1] for r in every if r[0] == SHRINK} == {0, 1} and {r[1] for r in every if r[0] == EXPAND} == {0, 1, 2}
    assert [r[4] for r in every if r[0] == OPERANDS] == [1, 1]
    assert all(r[3] for r in every if r[0] in (SHRINK, EXPAND) and r[2] > 0)
