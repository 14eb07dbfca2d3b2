"""The finetuning calls' refusals on the CPU: every argument is checked before any HIP call
(made-up device addresses, never read; a made-up handle of 49 tokens and 169 buckets)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2407_02068_amd", "liblpv.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="liblpv.so not built")

OK, INVALID, SHAPE, DTYPE, ALIAS, ALLOC = 0, -1, -2, -3, -5, -6
FAKE = 0x7f0000000000
G = 1 << 32


class Handle(ctypes.Structure):
    """The leading members of an lpv_relpos."""
    _fields_ = [("T", ctypes.c_int32), ("nt", ctypes.c_int32), ("n_buckets", ctypes.c_int32),
                ("n_segs", ctypes.c_int32), ("device", ctypes.c_int32), ("rest", ctypes.c_char * 256)]


HANDLE = Handle(49, 2, 169, 169, 0)
H_PTR = ctypes.addressof(HANDLE)


@pytest.fixture(scope="module")
def L():
    from paper_2407_02068_amd import lpv
    return lpv.lib()


def create(L, index=FAKE, T=49, n=169):
    out = ctypes.c_void_p(123)
    st = L.lpv_relpos_create(index, T, n, None, ctypes.byref(out))
    assert out.value is None
    return st


def test_relpos_create_refuses(L):
    assert L.lpv_relpos_create(FAKE, 49, 169, None, None) == INVALID
    assert create(L, index=0) == INVALID and create(L, index=FAKE + 2) == INVALID
    assert create(L, T=0) == SHAPE and create(L, T=2049) == SHAPE and create(L, T=-1) == SHAPE
    assert create(L, n=0) == SHAPE and create(L, n=65536) == SHAPE
    assert L.lpv_last_error().decode() != ""
    L.lpv_relpos_destroy(None)


def test_relpos_workspace_size(L):
    b = ctypes.c_size_t(0)
    size = lambda p=H_PTR, n=4, H=3, grad=0: L.lpv_relpos_workspace_size(p, n, H, grad, ctypes.byref(b))
    assert size(p=None) == INVALID and L.lpv_relpos_workspace_size(H_PTR, 4, 3, 0, None) == INVALID
    assert size(H=0) == SHAPE and size(H=65) == SHAPE and size(n=-1) == SHAPE
    assert size(n=1 << 31) == SHAPE and size(n=1 << 27) == SHAPE and size(n=1 << 62) == SHAPE
    assert size() == OK and size(grad=1) == OK and b.value > 0
    assert size(n=0, grad=1) == OK


def attention(L, p=H_PTR, table=FAKE, qkv=FAKE + G, ldq=288, n=4, H=3, hd=32, dt=2, region=0, nr=0,
              out=FAKE + 2 * G, ldo=96, lse=0, ws=FAKE + 3 * G, wsb=0):
    return L.lpv_relpos_attention(p, table, qkv, ldq, n, H, hd, dt, region, nr, out, ldo, lse, ws, wsb,
                                  None)


COMMON = [
    (dict(p=None), INVALID), (dict(dt=0), DTYPE), (dict(dt=9), DTYPE), (dict(hd=48), SHAPE),
    (dict(hd=128), SHAPE), (dict(H=0), SHAPE), (dict(H=65), SHAPE), (dict(n=-1), SHAPE),
    (dict(n=1 << 31), SHAPE), (dict(n=1 << 27), SHAPE), (dict(n=(1 << 62) + 1), SHAPE),
    (dict(table=0), INVALID), (dict(table=FAKE + 1), INVALID), (dict(qkv=0), INVALID),
    (dict(qkv=FAKE + G + 8), INVALID), (dict(out=0), INVALID), (dict(out=FAKE + 2 * G + 4), INVALID),
    (dict(ldq=280), INVALID), (dict(ldq=292), INVALID), (dict(ldq=(1 << 22) + 8), INVALID),
    (dict(ldo=88), INVALID), (dict(ldo=100), INVALID), (dict(region=FAKE + 4 * G, nr=0), INVALID),
    (dict(region=FAKE + 4 * G + 2, nr=1), INVALID), (dict(region=FAKE + 4 * G, nr=-3), INVALID),
]


@pytest.mark.parametrize("kw,want", COMMON + [
    (dict(out=FAKE + G + 1024), ALIAS), (dict(lse=FAKE + G), ALIAS), (dict(lse=FAKE + 2 * G + 16), ALIAS),
    (dict(lse=FAKE + 5 * G + 2), INVALID)])
def test_relpos_attention_refuses(L, kw, want):
    assert attention(L, **kw) == want
    assert L.lpv_last_error().decode() != ""


def test_relpos_attention_without_sequences(L):
    assert attention(L, n=0, qkv=0, out=0, ws=0) == OK


def grad(L, p=H_PTR, table=FAKE, qkv=FAKE + G, ldq=288, n=4, H=3, hd=32, dt=2, region=0, nr=0,
         out=FAKE + 2 * G, ldo=96, lse=FAKE + 5 * G, dout=FAKE + 6 * G, ldg=96, dqkv=FAKE + 7 * G,
         lddq=288, dtable=FAKE + 8 * G, ws=FAKE + 3 * G, wsb=64):
    return L.lpv_relpos_attention_grad(p, table, qkv, ldq, n, H, hd, dt, region, nr, out, ldo, lse, dout,
                                       ldg, dqkv, lddq, dtable, ws, wsb, None)


@pytest.mark.parametrize("kw,want", COMMON + [
    (dict(lse=0), INVALID), (dict(lse=FAKE + 5 * G + 1), INVALID), (dict(dout=0), INVALID),
    (dict(dout=FAKE + 6 * G + 8), INVALID), (dict(dqkv=0), INVALID), (dict(dqkv=FAKE + 7 * G + 2), INVALID),
    (dict(dtable=0), INVALID), (dict(dtable=FAKE + 8 * G + 1), INVALID), (dict(ldg=88), INVALID),
    (dict(ldg=98), INVALID), (dict(lddq=96), INVALID), (dict(lddq=290), INVALID),
    (dict(dqkv=FAKE + G), ALIAS), (dict(dqkv=FAKE + 2 * G + 64), ALIAS), (dict(dqkv=FAKE + 6 * G), ALIAS),
    (dict(dqkv=FAKE + 5 * G), ALIAS), (dict(dtable=FAKE + 7 * G), ALIAS), (dict(dtable=FAKE + 5 * G), ALIAS),
    (dict(dtable=FAKE + 2 * G), ALIAS), (dict(wsb=16), INVALID), (dict(ws=0, wsb=1 << 40), INVALID),
    (dict(ws=FAKE + 3 * G + 8, wsb=1 << 40), INVALID)])
def test_relpos_grad_refuses(L, kw, want):
    assert grad(L, **kw) == want
    assert L.lpv_last_error().decode() != ""


def distill(L, z=FAKE, ldz=1008, M=10, V=1000, dt=2, ids=FAKE + G, t=FAKE + 2 * G, ldt=16, k=16, tau=1.0,
            g=0, loss=FAKE + 3 * G, d=FAKE + 4 * G, ldd=1008, Vd=1008, ws=0, wsb=0):
    return L.lpv_distill(z, ldz, M, V, dt, ids, t, ldt, k, ctypes.c_double(tau), g, loss, d, ldd, Vd, ws,
                         wsb, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dt=3), DTYPE), (dict(dt=-1), DTYPE), (dict(M=-1), SHAPE), (dict(M=1 << 31), SHAPE),
    (dict(V=0), SHAPE), (dict(V=(1 << 22) + 1), SHAPE), (dict(k=0), SHAPE), (dict(k=1025), SHAPE),
    (dict(tau=0.0), INVALID), (dict(tau=-1.0), INVALID), (dict(tau=float("nan")), INVALID),
    (dict(tau=1e4), INVALID), (dict(tau=float("inf")), INVALID), (dict(ldz=999), INVALID),
    (dict(ldz=1004), INVALID), (dict(ldz=(1 << 22) + 8), INVALID), (dict(ldd=1000), INVALID),
    (dict(ldd=1012), INVALID), (dict(Vd=999), INVALID), (dict(ldt=15), INVALID), (dict(z=0), INVALID),
    (dict(z=FAKE + 8), INVALID), (dict(d=FAKE + 4 * G + 8), INVALID), (dict(ids=0), INVALID),
    (dict(t=0), INVALID), (dict(loss=0), INVALID), (dict(loss=FAKE + 3 * G + 2), INVALID),
    (dict(g=FAKE + 5 * G + 1), INVALID), (dict(ids=FAKE + G + 3), INVALID), (dict(d=FAKE + 16), ALIAS),
    (dict(d=FAKE, ldd=1016), ALIAS), (dict(loss=FAKE + 64), ALIAS), (dict(loss=FAKE + G + 4), ALIAS),
    (dict(loss=FAKE + 4 * G), ALIAS), (dict(d=FAKE + 2 * G - 16), ALIAS),
    (dict(g=FAKE + 3 * G + 4), ALIAS), (dict(g=FAKE + 4 * G + 400), ALIAS),
    # few long rows need a workspace
    (dict(M=2, V=100000, ldz=100000, ldd=100000, Vd=100000), INVALID),
    (dict(M=2, V=100000, ldz=100000, ldd=100000, Vd=100000, ws=FAKE + 6 * G, wsb=8), INVALID),
    (dict(M=2, V=100000, ldz=100000, ldd=100000, Vd=100000, ws=FAKE + 6 * G + 8, wsb=1 << 20), INVALID)])
def test_distill_refuses(L, kw, want):
    assert distill(L, **kw) == want
    assert L.lpv_last_error().decode() != ""


def test_distill_without_rows_and_its_workspace(L):
    assert distill(L, M=0, z=0, ids=0, t=0, loss=0, d=0) == OK
    b = ctypes.c_size_t(0)
    size = lambda M, V, k=16, dt=2: L.lpv_distill_workspace_size(M, V, k, dt, ctypes.byref(b))
    assert size(256, 1000) == OK and b.value == 0
    assert size(2, 100000) == OK and 0 < b.value <= 2 * (100000 // 8 // 256 * 8 + 4)
    assert size(0, 100000) == OK and b.value == 0
    assert size(2, 0) == SHAPE and size(-1, 5) == SHAPE and size(2, 5, 0) == SHAPE and size(2, 5, 4, 7) == DTYPE
    assert L.lpv_distill_workspace_size(2, 5, 4, 2, None) == INVALID


# 49 tokens x 4 windows of labels; 169 buckets x 3 heads of 2 bytes
REGION = dict(region=FAKE + 4 * G, nr=4)


@pytest.mark.parametrize("kw", [
    dict(out=FAKE), dict(out=FAKE - 4 * 49 * 96 * 2 + 16), dict(lse=FAKE + 169 * 6 - 6),
    dict(out=FAKE + 4 * G, **REGION), dict(out=FAKE + 4 * G + 4 * 49 * 4 - 16, **REGION),
    dict(lse=FAKE + 4 * G + 4 * 49 * 4 - 4, **REGION)])
def test_relpos_attention_refuses_outputs_over_what_it_reads(L, kw):
    assert attention(L, **kw) == ALIAS


@pytest.mark.parametrize("kw", [
    dict(dtable=FAKE), dict(dtable=FAKE + 169 * 6 - 2), dict(dtable=FAKE - 169 * 6 + 2),
    dict(dtable=FAKE, n=0), dict(dtable=FAKE + 4 * G + 4 * 49 * 4 - 4, **REGION),
    dict(dqkv=FAKE + 4 * G, **REGION), dict(dqkv=FAKE + 4 * G + 4 * 49 * 4 - 16, **REGION), dict(dqkv=FAKE)])
def test_relpos_grad_refuses_outputs_over_what_it_reads(L, kw):
    assert grad(L, **kw) == ALIAS


def test_neighbours_are_not_overlaps(L):
    """Right beside the table or the labels: not ALIAS (what refuses is the missing workspace)."""
    table = dict(dtable=FAKE + 169 * 6)
    labels = dict(dqkv=FAKE + 4 * G + 4 * 49 * 4, **REGION)
    assert (4 * 49 * 4) % 16 == 0
    for kw in (table, labels, dict(dtable=FAKE + 4 * G + 4 * 49 * 4, **REGION)):
        assert grad(L, wsb=16, **kw) == INVALID
