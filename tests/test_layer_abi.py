"""C-ABI checks of the layer operators that need no GPU: every call below must
be refused (or be a no-op) by the argument checks, before any CUDA call."""
import ctypes

import pytest

from paper_2506_08520_gb300 import binding as nb
from paper_2506_08520_gb300 import build as nbuild

OK, EINVAL, EDTYPE = nb.NYSTRA_OK, nb.NYSTRA_EINVAL, nb.NYSTRA_EDTYPE
MB = 1 << 20  # pointers that are never dereferenced, 16 MB apart
A, B, C, D, E, F, G, H, I, J, K = (i * 16 * MB for i in range(1, 12))
BIG = 1 << 62


@pytest.fixture(scope="module")
def lib():
    nbuild.build()
    return nb.lib()


def s3(*v):
    return (ctypes.c_longlong * 3)(*v)


def s2(*v):
    return (ctypes.c_longlong * 2)(*v)


def norm(L, x=A, xs=64, w=B, b=C, y=D, ys=64, m=E, r=F, rows=4, cols=64, eps=1e-5, dt=1, wdt=0):
    return L.nystra_layer_norm(x, xs, w, b, y, ys, m, r, rows, cols, eps, dt, wdt, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=3), EDTYPE), (dict(wdt=2), EDTYPE), (dict(dt=0, wdt=1), EDTYPE),
    (dict(rows=-1), EINVAL), (dict(cols=-1), EINVAL), (dict(eps=-1e-9), EINVAL), (dict(eps=float("nan")), EINVAL),
    (dict(eps=float("inf")), EINVAL), (dict(x=0), EINVAL), (dict(y=0), EINVAL), (dict(x=A + 1), EINVAL),
    (dict(w=B + 2), EINVAL), (dict(m=E + 2), EINVAL), (dict(ys=63), EINVAL), (dict(ys=-64), EINVAL),
    (dict(xs=-64), EINVAL), (dict(xs=BIG), EINVAL), (dict(y=A + 2), EINVAL), (dict(y=A, ys=65), EINVAL),
    (dict(y=B - 128), EINVAL), (dict(m=D), EINVAL), (dict(m=F + 4), EINVAL), (dict(r=A), EINVAL),
    (dict(rows=0, x=0, y=0), OK), (dict(cols=0, x=0, y=0), OK)])
def test_layer_norm(lib, kw, code):
    assert norm(lib, **kw) == code


def norm_bwd(L, dy=A, ds=64, x=B, xs=64, m=C, r=D, w=E, dx=F, dxs=64, dw=G, db=H, rows=4, cols=64, dt=1, wdt=0, ws=I,
             wb=None):
    wb = L.nystra_layer_norm_workspace(max(rows, 0), max(cols, 0)) if wb is None else wb
    return L.nystra_layer_norm_backward(dy, ds, x, xs, m, r, w, dx, dxs, dw, db, rows, cols, dt, wdt, ws, wb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=7), EDTYPE), (dict(wdt=2), EDTYPE), (dict(rows=-1), EINVAL), (dict(cols=-2), EINVAL), (dict(dy=0), EINVAL),
    (dict(x=0), EINVAL), (dict(dx=0), EINVAL), (dict(m=0), EINVAL), (dict(r=0), EINVAL), (dict(ws=0), EINVAL),
    (dict(wb=16), EINVAL), (dict(ws=I + 8), EINVAL), (dict(dw=G + 2), EINVAL), (dict(dx=A + 2), EINVAL),
    (dict(dx=B, dxs=70), EINVAL), (dict(dxs=10), EINVAL), (dict(dw=E), EINVAL), (dict(db=G + 4), EINVAL),
    (dict(dw=A), EINVAL), (dict(ws=B), EINVAL), (dict(ws=E), EINVAL), (dict(dx=C - 128), EINVAL),
    (dict(cols=0), OK), (dict(rows=0, dw=0, db=0, ws=0), OK), (dict(rows=0, ws=0), EINVAL)])
def test_layer_norm_backward(lib, kw, code):
    assert norm_bwd(lib, **kw) == code


def test_layer_norm_workspace(lib):
    assert lib.nystra_layer_norm_workspace(-1, 4) < 0 and lib.nystra_layer_norm_workspace(4, -1) < 0
    assert lib.nystra_layer_norm_workspace(0, 64) >= 2 * 64 * 4
    for rows in (1, 100, 10 ** 9):  # bounded, however many rows
        assert 0 < lib.nystra_layer_norm_workspace(rows, 4096) < 64 << 20


def rot(L, q=A, qs=(1024, 256, 64), qo=B, qos=(1024, 256, 64), hq=4, k=C, ks=(512, 256, 64), ko=D, kos=(512, 256, 64),
        hk=2, f=E, r=64, pos=F, bits=64, ps=4, amp=1.0, n=2, N=4, d=64, layout=0, inv=0, dt=1):
    return L.nystra_rotary(q, s3(*qs) if qs else None, qo, s3(*qos) if qos else None, hq, k, s3(*ks) if ks else None,
                           ko, s3(*kos) if kos else None, hk, f, r, pos, bits, ps, amp, n, N, d, layout, inv, dt, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=-1), EDTYPE), (dict(n=-1), EINVAL), (dict(N=-1), EINVAL), (dict(hq=-1), EINVAL), (dict(d=0), EINVAL),
    (dict(d=257), EINVAL), (dict(r=66), EINVAL), (dict(r=7), EINVAL), (dict(r=-2), EINVAL), (dict(layout=2), EINVAL),
    (dict(inv=2), EINVAL), (dict(amp=float("inf")), EINVAL), (dict(f=0), EINVAL), (dict(f=E + 4), EINVAL),
    (dict(bits=16), EINVAL), (dict(pos=F + 4), EINVAL), (dict(ps=-1), EINVAL), (dict(q=0), EINVAL),
    (dict(qs=None), EINVAL), (dict(kos=None), EINVAL), (dict(qs=(-1, 256, 64)), EINVAL), (dict(qs=(BIG, 1, 1)), EINVAL),
    (dict(qo=A + 128), EINVAL), (dict(qo=A, qos=(1024, 64, 256)), EINVAL), (dict(qos=(0, 256, 64)), EINVAL),
    (dict(qos=(1024, 256, 32)), EINVAL), (dict(qo=C), EINVAL), (dict(qo=D), EINVAL), (dict(ko=A), EINVAL),
    (dict(qo=E - 64), EINVAL), (dict(ko=F - 64), EINVAL),
    (dict(q=A, qo=A, k=A, ko=A, ks=(1024, 256, 64), kos=(1024, 256, 64)), EINVAL),
    (dict(n=0, q=0), OK), (dict(N=0, q=0), OK), (dict(hq=0, hk=0, q=0, k=0), OK)])
def test_rotary(lib, kw, code):
    assert rot(lib, **kw) == code


ST = (4096, 2048, 32)  # n = 2, heads = 2, N = 64, d = 32


def lin(L, q=A, qs=ST, k=B, ks=ST, v=C, vs=ST, o=D, os=ST, ld=E, ln=F, si=G, so=H, scale=1.0, n=2, h=2, N=64, dk=32,
        dv=32, dt=1, ws=None, wb=0):
    return L.nystra_linear_attention(q, s3(*qs) if qs else None, k, s3(*ks) if ks else None, v, s3(*vs) if vs else None,
                                     o, s3(*os) if os else None, ld, ln, si, so, scale, n, h, N, dk, dv, dt, ws, wb,
                                     None)


BAD_LINEAR = [
    (dict(dt=3), EDTYPE), (dict(n=-1), EINVAL), (dict(h=-1), EINVAL), (dict(N=-1), EINVAL), (dict(N=(1 << 24) + 1), EINVAL),
    (dict(dk=0), EINVAL), (dict(dk=129), EINVAL), (dict(dv=0), EINVAL), (dict(dv=129), EINVAL),
    (dict(n=1 << 20, h=1 << 10), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(q=0), EINVAL), (dict(v=0), EINVAL),
    (dict(ld=0), EINVAL), (dict(ld=E + 2), EINVAL), (dict(ln=F + 1), EINVAL), (dict(qs=None), EINVAL),
    (dict(ks=(4096, -1, 32)), EINVAL), (dict(vs=(BIG, BIG, 1)), EINVAL), (dict(q=A + 1), EINVAL), (dict(si=G + 2), EINVAL)]


@pytest.mark.parametrize("kw,code", BAD_LINEAR + [
    (dict(o=0), EINVAL), (dict(os=(4096, 2048, 16)), EINVAL), (dict(os=(0, 2048, 32)), EINVAL), (dict(o=A), EINVAL),
    (dict(o=C + 64), EINVAL), (dict(o=E - 8), EINVAL), (dict(o=G), EINVAL), (dict(o=H), EINVAL), (dict(so=G + 64), EINVAL),
    (dict(so=B), EINVAL), (dict(so=E), EINVAL), (dict(ws=I + 4, wb=1 << 20), EINVAL),
    (dict(n=0, q=0), OK), (dict(h=0, q=0), OK), (dict(N=0, q=0, so=0), OK)])
def test_linear_attention(lib, kw, code):
    assert lin(lib, **kw) == code


def lin_bwd(L, do=A, dos=ST, q=B, qs=ST, k=C, ks=ST, v=D, vs=ST, ld=E, ln=F, si=G, ds=H, dq=I, dqs=ST, dk_=J, dks=ST,
            dv_=K, dvs=ST, di=12 * 16 * MB, scale=1.0, n=2, h=2, N=64, dk=32, dv=32, dt=1, ws=None, wb=0):
    p = lambda s: s3(*s) if s else None  # noqa: E731
    return L.nystra_linear_attention_backward(do, p(dos), q, p(qs), k, p(ks), v, p(vs), ld, ln, si, ds, dq, p(dqs), dk_,
                                              p(dks), dv_, p(dvs), di, scale, n, h, N, dk, dv, dt, ws, wb, None)


@pytest.mark.parametrize("kw,code", BAD_LINEAR + [
    (dict(do=0), EINVAL), (dict(dq=0), EINVAL), (dict(dk_=0), EINVAL), (dict(dv_=0), EINVAL), (dict(dq=A), EINVAL),
    (dict(dv_=J + 64), EINVAL), (dict(dqs=(4096, 0, 32)), EINVAL), (dict(di=H), EINVAL), (dict(di=G), EINVAL),
    (dict(di=A), EINVAL), (dict(dk_=H - 64), EINVAL), (dict(dvs=None), EINVAL),
    (dict(n=0, q=0), OK), (dict(N=0, q=0, di=0), OK)])
def test_linear_attention_backward(lib, kw, code):
    assert lin_bwd(lib, **kw) == code


def test_linear_attention_workspace(lib):
    W = lib.nystra_linear_attention_workspace
    for bad in ((-1, 1, 1, 8, 8, 0, 0), (1, -1, 1, 8, 8, 0, 0), (1, 1, -1, 8, 8, 0, 0), (1, 1, 1, 0, 8, 0, 0),
                (1, 1, 1, 8, 129, 0, 0), (1, 1, 1, 8, 8, 5, 0)):
        assert W(*bad) < 0
    assert W(0, 4, 100, 8, 8, 1, 0) == 0 and W(1, 4, 0, 8, 8, 1, 1) == 0
    for dt in (0, 1, 2):
        for back in (0, 1):
            need = W(1, 2, 1 << 20, 64, 64, dt, back)  # one long sequence: split, into a bounded number of segments
            assert 0 < need < 1 << 30
            call = lin_bwd if back else lin
            assert call(lib, n=1, N=1 << 20, dk=64, dv=64, dt=dt, ws=64 * 16 * MB, wb=need - 1) == EINVAL


def step(L, q=A, qs=(64, 32), k=B, ks=(64, 32), v=C, vs=(64, 32), o=D, os=(64, 32), ld=E, si=G, so=H, scale=1.0, n=2,
         h=2, dk=32, dv=32, dt=1):
    return L.nystra_linear_attention_step(q, s2(*qs) if qs else None, k, s2(*ks) if ks else None, v,
                                          s2(*vs) if vs else None, o, s2(*os) if os else None, ld, si, so, scale, n, h,
                                          dk, dv, dt, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=3), EDTYPE), (dict(n=-1), EINVAL), (dict(dk=0), EINVAL), (dict(dv=129), EINVAL), (dict(q=0), EINVAL),
    (dict(so=0), EINVAL), (dict(ld=0), EINVAL), (dict(qs=None), EINVAL), (dict(os=(0, 32)), EINVAL),
    (dict(os=(64, 16)), EINVAL), (dict(ks=(-1, 32)), EINVAL), (dict(o=A), EINVAL), (dict(so=G + 64), EINVAL),
    (dict(so=C - 64), EINVAL), (dict(o=H), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(si=G + 1), EINVAL),
    (dict(n=0, q=0), OK)])
def test_linear_attention_step(lib, kw, code):
    assert step(lib, **kw) == code


@pytest.mark.parametrize("cols", [(1 << 30) + 1, (1 << 31) - 600, (1 << 31) - 1])
def test_layer_norm_rows_too_long(lib, cols):
    """Rows whose columns, or the two sums per column, would leave 32-bit indexes."""
    far = dict(xs=1 << 31, ys=1 << 31)
    wide = {k: i << 40 for i, k in enumerate("xwbymr", 1)}
    assert norm(lib, cols=cols, **far, **wide) == EINVAL
    assert lib.nystra_layer_norm_workspace(4, cols) == EINVAL
    wide = {k: i << 40 for i, k in enumerate(("dy", "x", "m", "r", "w", "dx", "dw", "db", "ws"), 1)}
    for grads in ({}, dict(dw=0, db=0, ws=0)):
        assert norm_bwd(lib, cols=cols, ds=1 << 31, xs=1 << 31, dxs=1 << 31, wb=1 << 40, **{**wide, **grads}) == EINVAL
    assert lib.nystra_layer_norm_workspace(4, 1 << 30) > 0


# q and k [2, heads, 5, d = 64] in one buffer, k `at` elements behind q, which share elements
@pytest.mark.parametrize("qs,ks,at,hq,hk", [
    ((3840, 64, 768), (3840, 64, 768), 64, 4, 4),     # a fused projection [n, N, 3, heads, d], k one head on
    ((3840, 64, 768), (3840, 64, 768), 192, 4, 2),    # three heads on
    ((3840, 64, 768), (3840, 64, 768), 768, 4, 4),    # one token on
    ((3840, 64, 768), (3840, 64, 768), 3840, 4, 4),   # one sequence on
    ((3840, 64, 768), (3840, 64, 768), 2, 4, 4),      # one pair of features on
    ((3840, 64, 768), (3840, 64, 768), 254, 4, 4),    # one pair of features short of the next place
    ((3840, 64, 768), (3840, 64, 768), 0, 4, 4),
    ((3840, 64, 768), (3840, 64, 768), 0, 4, 1),
    ((2560, 64, 512), (2560, 64, 512), 384, 4, 4),    # q's heads of the next token
    ((1280, 64, 256), (1280, 256, 64), 256, 4, 4),    # other strides
])
def test_rotary_in_place_on_shared_elements(lib, qs, ks, at, hq, hk):
    """Turned in place, q and k may be slices of one buffer, but each element turns once: refused, whichever comes
    first, and also where only one of them is turned in place and the other one reads."""
    k = A + 2 * at
    a = dict(q=A, qo=A, qs=qs, qos=qs, hq=hq, k=k, ko=k, ks=ks, kos=ks, hk=hk)
    b = dict(q=k, qo=k, qs=ks, qos=ks, hq=hk, k=A, ko=A, ks=qs, kos=qs, hk=hq)
    for args in (a, b):
        for other in ({}, dict(qo=C), dict(ko=C)):
            assert rot(lib, n=2, N=5, pos=None, f=K, **{**args, **other}) == EINVAL
