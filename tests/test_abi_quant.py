"""The refusals of the 8-bit calls on the CPU: every argument is checked before any HIP call
(made-up device addresses, never read; a made-up handle of a 96 x 64 weight)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2407_02068_amd", "liblpv.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="liblpv.so not built")

OK, INVALID, SHAPE, DTYPE, BLOCK, ALIAS, ALLOC = 0, -1, -2, -3, -4, -5, -6
FAKE = 0x7f0000000000
G = 1 << 32


class Handle(ctypes.Structure):
    """The leading members of an lpv_quant."""
    _fields_ = [("N", ctypes.c_int64), ("K", ctypes.c_int64), ("rest", ctypes.c_char * 512)]


HANDLE = Handle(96, 64)
H_PTR = ctypes.addressof(HANDLE)


@pytest.fixture(scope="module")
def L():
    from paper_2407_02068_amd import lpv
    return lpv.lib()


def rows(L, call, x=FAKE, ldx=40, y=FAKE + G, ldy=40, M=5, D=40, dt=2, gamma=FAKE + 2 * G,
         beta=FAKE + 3 * G, eps=1e-6, S=FAKE + 4 * G, lds=40, q=FAKE + 5 * G, ldq=40, scale=FAKE + 6 * G):
    params = {"lpv_quant_rows": (), "lpv_add_rmsnorm_quant": (gamma, eps),
              "lpv_add_layernorm_quant": (gamma, beta, eps)}[call]
    return getattr(L, call)(x, ldx, y, ldy, M, D, dt, *params, S, lds, q, ldq, scale, None)


ROWS = ["lpv_quant_rows", "lpv_add_rmsnorm_quant", "lpv_add_layernorm_quant"]


@pytest.mark.parametrize("call", ROWS)
@pytest.mark.parametrize("kw,want", [
    (dict(dt=3), DTYPE), (dict(dt=-1), DTYPE), (dict(D=0), SHAPE), (dict(D=-8), SHAPE),
    (dict(D=32769, ldx=40000), SHAPE), (dict(M=-1), SHAPE), (dict(M=1 << 31), SHAPE),
    (dict(ldx=39), INVALID), (dict(ldy=39), INVALID), (dict(lds=39), INVALID), (dict(ldq=39), INVALID),
    (dict(ldx=(1 << 22) + 1), INVALID), (dict(ldq=(1 << 22) + 1), INVALID), (dict(ldx=-40), INVALID),
    (dict(x=0), INVALID), (dict(q=0), INVALID), (dict(scale=0), INVALID), (dict(x=FAKE + 1), INVALID),
    (dict(y=FAKE + G + 1), INVALID), (dict(S=FAKE + 4 * G + 1), INVALID), (dict(scale=FAKE + 6 * G + 2), INVALID),
    (dict(x=FAKE + 2, dt=0), INVALID),
    # S: x or y itself, or apart from them
    (dict(S=FAKE + 2), ALIAS), (dict(S=FAKE + 80), ALIAS), (dict(S=FAKE, lds=48), ALIAS),
    (dict(S=FAKE + G + 80), ALIAS), (dict(S=FAKE, y=FAKE + 80), ALIAS),
    # codes and scales apart from everything
    (dict(q=FAKE + 8), ALIAS), (dict(q=FAKE + G), ALIAS), (dict(q=FAKE + 4 * G + 399), ALIAS),
    (dict(q=FAKE + 6 * G - 199), ALIAS), (dict(scale=FAKE + 396), ALIAS), (dict(scale=FAKE + 4 * G), ALIAS),
    (dict(scale=FAKE + G), ALIAS),
])
def test_rows_refuse(L, call, kw, want):
    assert rows(L, call, **kw) == want
    assert L.lpv_last_error().decode() != ""


@pytest.mark.parametrize("call", ROWS[1:])
@pytest.mark.parametrize("kw,want", [
    (dict(gamma=0), INVALID), (dict(gamma=FAKE + 1), INVALID), (dict(eps=-1e-9), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(q=FAKE + 2 * G + 64), ALIAS),
    (dict(scale=FAKE + 2 * G + 76), ALIAS), (dict(S=FAKE + 2 * G - 380), ALIAS),
])
def test_norms_refuse(L, call, kw, want):
    assert rows(L, call, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(beta=0), INVALID), (dict(beta=FAKE + 3), INVALID), (dict(q=FAKE + 3 * G), ALIAS),
    (dict(S=FAKE + 3 * G + 16), ALIAS)])
def test_layernorm_refuses(L, kw, want):
    assert rows(L, "lpv_add_layernorm_quant", **kw) == want


@pytest.mark.parametrize("call", ROWS)
def test_no_rows_is_a_noop(L, call):
    assert rows(L, call, M=0, x=0, y=0, S=0, q=0, scale=0) == OK
    assert rows(L, call, M=0, D=0) == SHAPE  # (its other arguments are still checked)


def pack(L, W=FAKE, ldw=64, N=96, K=64, scale=FAKE + G, b_r=32, b_c=32, mask=FAKE + 2 * G):
    out = ctypes.c_void_p(123)
    st = L.lpv_quant_pack(W, ldw, N, K, scale, b_r, b_c, mask, None, ctypes.byref(out))
    if st != OK:
        assert out.value is None
    return st


@pytest.mark.parametrize("kw,want", [
    (dict(b_r=8), BLOCK), (dict(b_c=128), BLOCK), (dict(b_r=0), BLOCK), (dict(b_c=-16), BLOCK),
    (dict(N=112), SHAPE), (dict(K=80, ldw=80), SHAPE), (dict(N=0), SHAPE), (dict(K=-32), SHAPE),
    (dict(N=65568), SHAPE), (dict(K=65568, ldw=65568), SHAPE),
    (dict(mask=0, N=104), SHAPE), (dict(mask=0, K=24, ldw=32), SHAPE),  # dense: multiples of 16
    (dict(W=0), INVALID), (dict(W=FAKE + 8), INVALID), (dict(ldw=48), INVALID), (dict(ldw=72), INVALID),
    (dict(ldw=(1 << 22) + 16), INVALID), (dict(scale=0), INVALID), (dict(scale=FAKE + G + 2), INVALID),
])
def test_pack_refuses(L, kw, want):
    assert pack(L, **kw) == want
    assert L.lpv_last_error().decode() != ""


def test_pack_null_out_and_allocation(L, monkeypatch):
    assert L.lpv_quant_pack(FAKE, 64, 96, 64, FAKE + G, 32, 32, FAKE + 2 * G, None, None) == INVALID
    monkeypatch.setenv("LPV_FAULT_INJECT", "alloc")
    assert pack(L) == ALLOC and pack(L, mask=0) == ALLOC
    assert "allocation" in L.lpv_last_error().decode()


def linear(L, h=H_PTR, X=FAKE, ldx=64, xscale=FAKE + G, M=7, bias=FAKE + 2 * G, Y=FAKE + 3 * G, ldy=96, dt=2,
           epi=0):
    return L.lpv_quant_linear(h, X, ldx, xscale, M, bias, Y, ldy, dt, epi, None)


@pytest.mark.parametrize("kw,want", [
    (dict(h=None), INVALID), (dict(dt=3), DTYPE), (dict(dt=-1), DTYPE), (dict(M=-1), SHAPE),
    (dict(M=1 << 31), SHAPE), (dict(epi=2), INVALID), (dict(epi=-1), INVALID),
    (dict(ldx=48), INVALID), (dict(ldx=72), INVALID), (dict(ldx=(1 << 22) + 16), INVALID),
    (dict(ldy=88), INVALID), (dict(ldy=100), INVALID), (dict(ldy=98, dt=0), INVALID),
    (dict(ldy=(1 << 22) + 8), INVALID),
    (dict(X=0), INVALID), (dict(Y=0), INVALID), (dict(xscale=0), INVALID), (dict(X=FAKE + 8), INVALID),
    (dict(Y=FAKE + 3 * G + 8), INVALID), (dict(bias=FAKE + 8), INVALID), (dict(xscale=FAKE + G + 1), INVALID),
    (dict(Y=FAKE), ALIAS), (dict(Y=FAKE + 432), ALIAS), (dict(Y=FAKE + G - 1328), ALIAS),
    (dict(Y=FAKE + 2 * G + 176), ALIAS), (dict(Y=FAKE + 2 * G + 352, dt=0), ALIAS),
])
def test_linear_refuses(L, kw, want):
    assert linear(L, **kw) == want
    assert L.lpv_last_error().decode() != ""


def test_linear_of_no_tokens_and_null_handles(L):
    assert linear(L, M=0, X=0, Y=0, xscale=0) == OK
    assert L.lpv_quant_info_get(None, None) == INVALID
    from paper_2407_02068_amd.lpv import QuantInfo
    assert L.lpv_quant_info_get(None, ctypes.byref(QuantInfo())) == INVALID
    assert L.lpv_quant_info_get(H_PTR, None) == INVALID
    L.lpv_quant_destroy(None)
