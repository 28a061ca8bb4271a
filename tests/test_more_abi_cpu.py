"""Host-side checks of the 8-bit floating-point projection, the norm and rotation of heads and the bookkeeping: they answer before any
CUDA call."""
import ctypes

import pytest

OK, INVALID, UNSUPPORTED = 0, 1, 2
P = ctypes.c_void_p
FAKE = P(1 << 20)  # never dereferenced: the checks fail first
ODD = P((1 << 20) + 4)
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def J():
    from paper_2609_34866_gb300 import binding, build
    build.build()
    binding._LIB = None
    binding.lib()
    return binding


def _cache(J, heads=2, dh=64, bits=8, page=16, pages=4, ptr=1 << 20):
    return J._KvCacheDesc(heads, dh, bits, page, pages, ptr, ptr, ptr, ptr)


def _how(J, norm=1, eps=1e-6, qw=None, kw=None, pos=1 << 20, cos=1 << 20, sin=1 << 20, length=8, dim=64, inter=0):
    return J._NormRope(norm, eps, qw, kw, pos, cos, sin, length, dim, inter)


def test_fp8_refusals(J):
    L = J.lib()

    def quant(M=4, K=64, x=FAKE, t=1, ld=64, rows=128, c=FAKE, s=FAKE):
        return L.jab_fp8_quantize(M, K, x, t, ld, rows, c, s, None)

    def call(M=4, N=128, K=64, x=FAKE, xt=1, ldx=64, w=FAKE, s=FAKE, rows=1, y=FAKE, yt=1, ldy=128, ws=FAKE, nb=1 << 40):
        return L.jab_fp8_linear(M, N, K, x, xt, ldx, w, s, rows, y, yt, ldy, ws, nb, None)

    assert quant(M=0, x=None) == OK and call(M=0, x=None) == OK
    for bad in (dict(x=None), dict(c=None), dict(s=None), dict(M=-1), dict(K=0), dict(t=3), dict(ld=56), dict(ld=65), dict(x=ODD), dict(c=ODD), dict(rows=64),
                dict(rows=0)):
        assert quant(**bad) == INVALID, bad
    for bad in (dict(x=None), dict(w=None), dict(s=None), dict(y=None), dict(ws=None), dict(M=-1), dict(N=0), dict(K=0), dict(xt=3), dict(yt=-1),
                dict(ldx=48), dict(ldx=65), dict(ldy=127), dict(x=ODD), dict(w=ODD), dict(ws=ODD), dict(nb=100), dict(rows=2)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(K=24, ldx=24), dict(K=131088, ldx=131088)):
        assert call(**bad) == UNSUPPORTED, bad
    assert quant(K=24, ld=24) == UNSUPPORTED
    assert J.jab_fp8_linear_workspace_size(4, 128, 24) == 0
    assert J.jab_fp8_linear_workspace_size(8, 128, 64) >= 8 * 64
    assert J.jab_fp8_linear_workspace_size(0, 128, 64) > 0


def test_norm_rope_refusals(J):
    L = J.lib()

    def write(c=None, n=3, hq=2, x=FAKE, t=0, ld=6 * 64, slots=FAKE, q=FAKE, how=None):
        return L.jab_kv_write_norm_rope(ctypes.byref(c or _cache(J)), n, hq, x, t, ld, slots, ctypes.byref(how or _how(J)), q, None)

    def rows(n=3, hq=2, hk=1, dh=64, x=FAKE, t=0, ld=192, how=None, q=FAKE, ldq=128, k=FAKE, ldk=64):
        return L.jab_qk_norm_rope(n, hq, hk, dh, x, t, ld, ctypes.byref(how or _how(J)), q, ldq, k, ldk, None)

    def back(n=3, hq=2, hk=1, dh=64, x=FAKE, t=0, ld=192, how=None, q=FAKE, ldq=128, k=FAKE, ldk=64, dx=FAKE, lddx=192, wq=FAKE, wk=FAKE, ws=FAKE,
             nb=1 << 30):
        return L.jab_qk_norm_rope_backward(n, hq, hk, dh, x, t, ld, ctypes.byref(how or _how(J)), q, ldq, k, ldk, dx, lddx, wq, wk, ws, nb, None)

    assert write(n=0) == OK and rows(n=0) == OK and back(n=0, wq=None, wk=None) == OK
    hows = [dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(qw=(1 << 20) + 4), dict(kw=8), dict(pos=None), dict(cos=None), dict(sin=None),
            dict(length=0), dict(dim=0), dict(dim=80), dict(dim=128), dict(cos=(1 << 20) + 8)]
    for f in (write, rows, back):
        for bad in hows:
            assert f(how=_how(J, **bad)) == INVALID, (f, bad)
        assert f(how=_how(J, dim=24)) == UNSUPPORTED
        for bad in (dict(x=None), dict(x=ODD), dict(n=-1), dict(hq=-1), dict(t=7), dict(ld=184), dict(ld=385)):
            assert f(**bad) == INVALID, (f, bad)
    assert write(slots=None) == INVALID and write(q=ODD) == INVALID
    assert write(_cache(J, dh=96)) == UNSUPPORTED and write(_cache(J, ptr=0)) == INVALID
    for f in (rows, back):
        for bad in (dict(q=None), dict(k=None), dict(q=ODD), dict(ldq=120), dict(ldk=56), dict(ldk=65), dict(hq=0, hk=0), dict(hk=-1)):
            assert f(**bad) == INVALID, (f, bad)
        for bad in (dict(dh=96), dict(hq=4096), dict(n=(1 << 31) + 1)):
            assert f(**bad) == UNSUPPORTED, (f, bad)
    for bad in (dict(dx=None), dict(lddx=184), dict(ws=None), dict(nb=1000), dict(ws=ODD), dict(how=_how(J, norm=0))):
        assert back(**bad) == INVALID, bad
    size = L.jab_qk_norm_rope_backward_workspace_size
    assert size(3, 2, 1, 64) > 0 and size(3, 0, 0, 64) == 0 and size(3, 2, 1, 96) == 0 and size(-1, 2, 1, 64) == 0
    assert L.jab_kv_write_norm_rope(ctypes.byref(_cache(J)), 3, 2, FAKE, 0, 384, FAKE, None, FAKE, None) == INVALID


def test_table_refusals(J):
    L = J.lib()

    def call(length=8, dim=64, theta=1e4, cos=FAKE, sin=FAKE, **k):
        s = dict(kind=2, factor=4.0, original=4096.0, low=1.0, high=32.0, attention=1.0)
        s.update(k)
        return L.jab_rope_table_scaled(length, dim, theta, ctypes.byref(J._RopeScaling(*s.values())), cos, sin, None)

    for bad in (dict(length=0), dict(dim=0), dict(theta=0.0), dict(theta=NAN), dict(cos=None), dict(sin=ODD), dict(kind=3), dict(kind=-1), dict(factor=0.5),
                dict(factor=NAN), dict(original=0.0), dict(low=-1.0), dict(low=32.0), dict(high=INF), dict(attention=0.0), dict(attention=NAN)):
        assert call(**bad) == INVALID, bad
    assert call(dim=24) == UNSUPPORTED and call(dim=256) == UNSUPPORTED


def test_bookkeeping_refusals(J):
    L = J.lib()

    def plan(c=None, B=2, n=4, lens=FAKE, counts=FAKE, pages=FAKE, mp=4, free=FAKE, cap=4, nf=FAKE, nl=FAKE, nn=FAKE, qs=FAKE, slots=FAKE, pos=FAKE):
        return L.jab_kv_plan(ctypes.byref(c or _cache(J)), B, n, lens, counts, pages, mp, free, cap, nf, nl, nn, qs, slots, pos, None)

    def release(c=None, B=2, lens=FAKE, ended=FAKE, pages=FAKE, mp=4, sh=0, free=FAKE, cap=4, nf=FAKE, nl=FAKE, nn=FAKE):
        return L.jab_kv_release(ctypes.byref(c or _cache(J)), B, lens, ended, pages, mp, sh, free, cap, nf, nl, nn, None)

    for f in (plan, release):
        for bad in (dict(B=0), dict(mp=0), dict(lens=None), dict(pages=None), dict(free=None), dict(cap=-1), dict(nf=None), dict(nl=None), dict(nn=None),
                    dict(lens=P((1 << 20) + 2))):
            assert f(**bad) == INVALID, (f, bad)
        for bad in (dict(B=8193), dict(mp=1 << 27)):
            assert f(**bad) == UNSUPPORTED, (f, bad)
        assert f(_cache(J, page=24)) == UNSUPPORTED and f(_cache(J, pages=0)) == INVALID
    for bad in (dict(n=-1), dict(counts=None), dict(qs=None), dict(slots=None), dict(pos=None), dict(slots=ODD)):
        assert plan(**bad) == INVALID, bad
    assert plan(n=1 << 30) == UNSUPPORTED
    assert release(ended=None) == INVALID and release(sh=-16) == INVALID and release(sh=80) == INVALID and release(sh=8) == UNSUPPORTED


def test_binding_refuses_wrong_tensors(J):
    import torch
    x = torch.zeros((2, 128))
    with pytest.raises(ValueError):
        J.jab_fp8_quantize(x, torch.zeros((2, 128), dtype=torch.float8_e4m3fn), torch.zeros((1, 1)))
    with pytest.raises(ValueError):
        J.jab_qk_norm_rope(x, 1, 1, 64, x[:, :64], x[:, 64:], norm_eps=1e-6)
    with pytest.raises(ValueError):
        J._norm_rope(2, 64, None, None, False, None, x, None)
    with pytest.raises(ValueError):
        J._norm_rope(2, 64, None, (x, x), False, None, None, None)


def test_binding_refuses_missing_heads(J):
    import torch
    x = torch.zeros((2, 128))
    assert J._heads(None, 2, 0, 64, x, "q") == (None, 0)
    for name in ("q", "k", "dq", "dk"):
        with pytest.raises(ValueError, match=f"{name} is needed"):
            J._heads(None, 2, 1, 64, x, name)


def test_binding_refuses_unknown_kinds_of_tables(J):
    import torch
    with pytest.raises(ValueError, match="kind must be one of"):
        J.jab_rope_table_scaled(torch.zeros((4, 32)), torch.zeros((4, 32)), 1e4, kind="other")
