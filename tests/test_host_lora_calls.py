"""CPU-side checks of calls of the low-rank adapters that lie between the ordinary ones: fake addresses, never dereferenced."""
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


@pytest.mark.parametrize("ld", [0, -1, -16, 15])
def test_an_h_narrower_than_the_ranks_is_refused(bd, ld):
    """Rows of h that do not hold a token's ranks, rows of no element among them: of one matrix, of a group, of decode and larger calls."""
    L = bd.lib()
    for T, rank in ((1, 16), (3, 16), (3, 17), (600, 16)):
        need = bd.lora_workspace_bytes(T, 2, rank)
        tok = _i32(*([0] * T))
        assert L.bd_lora_multitenant(A, _ptrs(2 * A), _ptrs(3 * A), _i32(rank), 4 * A, tok, None, 5 * A, 6 * A, ld, T, 40, 64, 1, 7 * A, need, 0) == 2
        out = (ctypes.c_int64 * 2)(40, 40)
        for h in (_ptrs(6 * A, None), _ptrs(None, 6 * A)):
            assert L.bd_lora_multitenant_group(2, A, _ptrs(2 * A, 8 * A), _ptrs(3 * A, 9 * A), _i32(rank, rank), _ptrs(4 * A, 4 * A), tok, None,
                                               _ptrs(5 * A, 10 * A), h, ld, T, out, 64, 1, 7 * A, need, 0) == 2


def test_a_negative_width_of_h_is_refused_without_ranks_too(bd):
    call = lambda ld: bd.lib().bd_lora_multitenant(A, _ptrs(None), _ptrs(None), _i32(0), None, _i32(0, 0), 5 * A, 5 * A, 6 * A, ld, 2, 40, 64, 1, None, 0, 0)
    assert call(-1) == 2 and call(0) == 0                # (in place without an adapter: nothing to do)
