"""How dense attention deals its calls to blocks: on the host, without a GPU.

Every call that the header allows has to fit a block's shared memory, 160 KB with the kernels' own arrays.  The planners are
internal functions of the library, called here by their symbols.
"""
import ctypes
import itertools
import os

import pytest

F32, BF16 = 0, 1
LDS = 160 * 1024
WIDEST = 4993  # of a grid of several rows with a bias


class Call(ctypes.Structure):  # scram::DenseCall
    _fields_ = [("Q", ctypes.c_void_p), ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("bias_rows", ctypes.c_int),
                ("lengths", ctypes.c_void_p), ("grid", ctypes.c_int * 6), ("key_slices", ctypes.c_int), ("scale", ctypes.c_float),
                ("causal", ctypes.c_bool), ("first", ctypes.c_int), ("origin", ctypes.c_void_p)]


class Needs(ctypes.Structure):  # scram::DenseNeeds
    _fields_ = [("blocks", ctypes.c_uint64), ("lds", ctypes.c_size_t)]


@pytest.fixture(scope="module")
def L():
    from paper_1905_10308_amd import binding

    if not os.path.exists(binding.LIB_PATH):
        from paper_1905_10308_amd import build

        build.build()
    L = binding.lib()
    for name in ("_ZN5scram11dense_needsEiRKNS_9DenseCallE", "_ZN5scram20dense_backward_needsEiRKNS_9DenseCallE"):
        f = getattr(L, name)
        f.argtypes, f.restype = [ctypes.c_int, ctypes.POINTER(Call)], Needs
    window = L._ZN5scram17dense_bias_windowEii
    window.argtypes, window.restype = [ctypes.c_int, ctypes.c_int], ctypes.c_int64
    size = L._ZN5scram21dense_workspace_bytesEiRKNS_9DenseCallE
    size.argtypes, size.restype = [ctypes.c_int, ctypes.POINTER(Call)], ctypes.c_size_t
    return L


def call(S, Sk, Hq, Wq, Hk, Wk, d, bias=1, causal=False):
    return Call(bias=16 if bias else None, bias_rows=bias, grid=(S, Hq, Wq, Hk, Wk, d), key_slices=Sk, scale=1.0, causal=causal)


def needs(L, dtype, c):
    return (L._ZN5scram11dense_needsEiRKNS_9DenseCallE(dtype, c), L._ZN5scram20dense_backward_needsEiRKNS_9DenseCallE(dtype, c))


def test_the_structure_is_the_library_s(L):
    for c in ((32, 16, 1, 1, 64, 64, 64), (6, 3, 9, 40, 9, 40, 128), (4, 4, 1, 1, 30, 31, 16)):
        for dtype in (F32, BF16):
            assert L._ZN5scram21dense_workspace_bytesEiRKNS_9DenseCallE(dtype, call(*c)) == L.scram_dense_attend_workspace_bytes(*c, dtype, 1)


def test_the_widest_grid(L):
    most = 10240  # places of two runs of 128
    assert L._ZN5scram17dense_bias_windowEii(2, WIDEST) <= most < L._ZN5scram17dense_bias_windowEii(2, WIDEST + 1)
    assert all(L._ZN5scram17dense_bias_windowEii(2, w) <= most for w in range(1, WIDEST))
    assert L._ZN5scram17dense_bias_windowEii(1, 1 << 30) <= most


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("c", [
    (1, 1, 2, 3400, 2, 3400, 128), (1, 1, 2, 2950, 2, 2950, 128), (1, 1, 1, 1, 2, 3600, 128), (1, 1, 2, 3600, 2, 3600, 128),
    (10, 1, 1, 1, 70, 70, 128), (10, 1, 1, 3, 70, 70, 128), (300, 300, 2, 1450, 2, 1450, 128), (130, 130, 2, 1500, 2, 1500, 128),
    (1, 1, 2, WIDEST, 2, WIDEST, 128)], ids=lambda c: "x".join(map(str, c)))
def test_wide_grids_fit(L, c, dtype):
    for n in needs(L, dtype, call(*c)):
        assert 0 < n.lds <= LDS and n.blocks > 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
def test_every_call_fits(L, d, dtype):
    """Over widths up to the widest, few and many slices and queries, shared keys, with and without a bias and the mask."""
    widths = [*range(1, 70, 3), *range(70, 200, 13), *range(200, WIDEST, 61), WIDEST]
    worst = 0
    for S, share, Hk, Wk, run in itertools.product((1, 33, 300), (1, 2, 10), (1, 2, 3, 70), widths, (0, 1, 3, 200)):
        if run > Hk * Wk:
            continue
        shape = (S * share, S, 1 if run else Hk, run or Wk, Hk, Wk, d)
        for bias, causal in ((1, False), (1, True), (0, False)):
            if bias or Wk % 7 == 0:
                worst = max(worst, *(n.lds for n in needs(L, dtype, call(*shape, bias, causal))))
    assert worst <= LDS
