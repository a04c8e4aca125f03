"""Argument checks of the invariant layers' C entry points: every refusal is made before device work."""
import ctypes as ct

import pytest

from paper_2609_35099_amd import e3mi

P = ct.c_void_p(4096)      # never dereferenced: the calls below are refused first
ODD = ct.c_void_p(4097)
HALF = ct.c_void_p(4098)   # aligned for bfloat16 only
F32, BF16 = 0, 1
OK, INVALID, SMALL = 0, 1, 4


@pytest.fixture(scope="module")
def L():
    return e3mi.lib()


def test_pack8_refusals(L):
    for fn in (L.e3_pack8, L.e3_unpack8):
        def call(dtype=F32, a=P, ld=8, b=P, c=P, rows=4, cols=8):
            return fn(dtype, a, ld, b, c, rows, cols, None) if fn is L.e3_pack8 else fn(dtype, b, c, a, ld, rows, cols,
                                                                                        None)
        for kw in ({"dtype": 2}, {"dtype": -1}, {"ld": 7}, {"rows": -1}, {"cols": 0}, {"cols": (1 << 20) + 1, "ld": 1 << 21},
                   {"a": None}, {"b": None}, {"c": None}, {"a": ODD}, {"a": HALF}, {"dtype": BF16, "a": ODD},
                   {"rows": (1 << 40) + 1}):
            assert call(**kw) == INVALID, kw
        assert call(rows=0, a=None, b=None, c=None) == OK


def test_layer_norm_refusals(L):
    def fwd(dtype=F32, x=P, ldx=8, g=P, b=P, eps=1e-5, y=P, ldy=8, mean=None, rstd=None, xq=None, xc=None, yq=None,
            yc=None, rows=4, cols=8):
        return L.e3_layer_norm_fwd(dtype, x, ldx, g, b, eps, y, ldy, mean, rstd, xq, xc, yq, yc, rows, cols, None)
    for kw in ({"dtype": 9}, {"x": None}, {"y": None}, {"ldx": 7}, {"ldy": 7}, {"eps": -1e-9}, {"eps": float("nan")},
               {"xq": P}, {"xc": P}, {"yq": P}, {"g": ODD}, {"b": HALF}, {"mean": HALF}, {"rstd": ODD}, {"rows": -2},
               {"cols": 0}):
        assert fwd(**kw) == INVALID, kw
    assert fwd(rows=0, x=None, y=None) == OK

    n = ct.c_size_t()
    assert L.e3_layer_norm_workspace_size(F32, 100, 33, ct.byref(n)) == OK and n.value >= 2 * 33 * 4
    assert L.e3_layer_norm_workspace_size(F32, 0, 33, ct.byref(n)) == OK and n.value == 0
    assert L.e3_layer_norm_workspace_size(F32, 1, 33, None) == INVALID
    assert L.e3_layer_norm_workspace_size(F32, -1, 33, ct.byref(n)) == INVALID
    L.e3_layer_norm_workspace_size(F32, 4, 8, ct.byref(n))

    def bwd(dtype=F32, x=P, ldx=8, xq=None, xc=None, g=P, dy=P, lddy=8, mean=P, rstd=P, dx=P, lddx=8, dg=P, db=P, ws=P,
            nb=n.value, rows=4, cols=8):
        return L.e3_layer_norm_bwd(dtype, x, ldx, xq, xc, g, dy, lddy, mean, rstd, dx, lddx, dg, db, ws, nb, rows, cols,
                                   None)
    for kw in ({"x": None}, {"xq": P, "xc": P}, {"x": None, "xq": P}, {"dy": None}, {"mean": None}, {"rstd": None},
               {"ldx": 7}, {"lddy": 7}, {"lddx": 7}, {"ws": None}, {"g": ODD}, {"dx": HALF}, {"dg": HALF}, {"db": ODD},
               {"cols": -1}):
        assert bwd(**kw) == INVALID, kw
    assert bwd(nb=n.value - 1) == SMALL
    assert bwd(dx=None, dg=None, db=None, ws=None, nb=0) == OK          # nothing asked for
    assert bwd(rows=0, x=None, dy=None, mean=None, rstd=None, dg=None, db=None, ws=None, nb=0) == OK


def test_dense_refusals(L):
    f, b = ct.c_size_t(), ct.c_size_t()
    assert L.e3_dense_workspace_size(F32, 16, 8, 8, ct.byref(f), ct.byref(b)) == OK
    for args in ((3, 1, 1, 1), (F32, -1, 1, 1), (F32, 1, 0, 1), (F32, 1, 1, 0), (F32, 1, 1, (1 << 20) + 1)):
        assert L.e3_dense_workspace_size(*args, ct.byref(f), ct.byref(b)) == INVALID
    assert L.e3_dense_workspace_size(F32, 1, 1, 1, None, ct.byref(b)) == INVALID
    # zero rows need no scratch, and no size of a call needs a petabyte
    assert L.e3_dense_workspace_size(BF16, 0, 64, 64, ct.byref(f), ct.byref(b)) == OK and f.value == b.value == 0

    def fwd(dtype=F32, x=P, ldx=8, W=P, bias=P, r=P, ldr=8, act=0, y=P, ldy=8, z=None, ldz=8, zq=None, zc=None, yq=None,
            yc=None, M=4, K=8, N=8):
        return L.e3_dense_fwd(dtype, x, ldx, W, bias, r, ldr, act, y, ldy, z, ldz, zq, zc, yq, yc, P, 1 << 40, M, K, N,
                              None)
    for kw in ({"x": None}, {"W": None}, {"y": None}, {"ldx": 7}, {"ldr": 7}, {"ldy": 7}, {"z": P, "ldz": 7}, {"act": 4},
               {"act": -1}, {"zq": P}, {"yc": P}, {"x": HALF}, {"W": ODD}, {"bias": HALF}, {"r": HALF}, {"y": ODD},
               {"z": HALF}, {"K": 0}, {"N": 0}, {"M": -1}, {"dtype": 7}):
        assert fwd(**kw) == INVALID, kw
    assert fwd(M=0, x=None, y=None) == OK

    L.e3_dense_workspace_size(F32, 4, 8, 8, ct.byref(f), ct.byref(b))

    def bwd(dtype=F32, x=P, ldx=8, xq=None, xc=None, W=P, z=P, ldz=8, zq=None, zc=None, act=2, dy=P, lddy=8, dx=P, lddx=8,
            dW=P, db=P, ws=P, nb=b.value, M=4, K=8, N=8):
        return L.e3_dense_bwd(dtype, x, ldx, xq, xc, W, z, ldz, zq, zc, act, dy, lddy, dx, lddx, dW, db, ws, nb, M, K, N,
                              None)
    for kw in ({"x": None}, {"xq": P, "xc": P}, {"xq": P}, {"W": None}, {"z": None}, {"zq": P, "zc": P}, {"zc": P},
               {"dy": None}, {"act": 5}, {"ldx": 7}, {"ldz": 7}, {"lddy": 7}, {"lddx": 7}, {"dx": ODD}, {"dW": HALF},
               {"db": HALF}, {"K": 0}, {"M": -1}):
        assert bwd(**kw) == INVALID, kw
    if b.value:
        assert bwd(nb=b.value - 1) == SMALL
        assert bwd(ws=None) == INVALID


def _sizes(L, *args):
    f, b = ct.c_size_t(), ct.c_size_t()
    assert L.e3_dense_workspace_size(*args, ct.byref(f), ct.byref(b)) == OK
    return f.value, b.value


@pytest.mark.parametrize("dtype,M,K,N", [(F32, 16, 1000, 500), (BF16, 16, 1000, 500), (F32, 300, 4100, 300), (BF16, 3001, 4099, 2051)])
def test_dense_forward_scratch_refusals(L, dtype, M, K, N):
    """Sizes whose reduction is split: less scratch than asked for, none, or misaligned."""
    need = _sizes(L, dtype, M, K, N)[0]
    assert need >= 2 * M * N * 4                    # two splits at least

    def fwd(ws, nb):
        return L.e3_dense_fwd(dtype, P, K, P, None, None, N, 0, P, N, None, N, None, None, None, None, ws, nb, M, K, N, None)
    assert fwd(P, need - 1) == SMALL and fwd(P, 0) == SMALL and fwd(None, 0) == SMALL
    for ws in (None, ODD, HALF):
        assert fwd(ws, need) == INVALID, ws


@pytest.mark.parametrize("dtype,M,K,N", [(F32, 64, 300, 40), (BF16, 64, 300, 40), (F32, 5000, 64, 64), (BF16, 40000, 128, 256)])
def test_dense_backward_scratch_refusals(L, dtype, M, K, N):
    """Sizes that write dz (K = 300) or split the sum over rows."""
    need = _sizes(L, dtype, M, K, N)[1]
    assert need > 0

    def bwd(ws, nb):
        return L.e3_dense_bwd(dtype, P, K, None, None, P, P, N, None, None, 2, P, N, P, K, P, P, ws, nb, M, K, N, None)
    assert bwd(P, need - 1) == SMALL and bwd(P, 0) == SMALL and bwd(None, 0) == SMALL
    for ws in (None, ODD, HALF, ct.c_void_p(4096 + 8)):       # 16-byte alignment
        assert bwd(ws, need) == INVALID, ws


def test_dense_scratch_stays_near_the_tensors(L):
    """No size asks for more than a small multiple of what it works on: 256 splits are taken only where the
    outputs are few, dz is as large as dy."""
    for dtype, e in ((F32, 4), (BF16, 2)):
        for M in (1, 9, 100, 4097, 1_000_003):
            for K in (1, 17, 300, 4099, 1 << 20):
                for N in (1, 8, 65, 1027, 1 << 20):
                    f, b = _sizes(L, dtype, M, K, N)
                    tensors = e * (M * K + K * N + M * N)
                    assert f <= 16 * tensors + (64 << 20), (dtype, M, K, N, f)
                    assert b <= 16 * tensors + (64 << 20), (dtype, M, K, N, b)
