"""Host-side checks of the serving entry points: they answer before any CUDA call."""
import ctypes

import pytest

OK, INVALID, UNSUPPORTED = 0, 1, 2
P = ctypes.c_void_p
FAKE = P(1 << 20)  # never dereferenced: the checks fail first
ODD = P((1 << 20) + 4)


@pytest.fixture(scope="module")
def J():
    from paper_2609_34866_gb300 import binding, build
    build.build()
    binding._LIB = None
    binding.lib()
    return binding


def _cache(J, heads=2, dh=64, bits=8, page=16, pages=4, ptr=1 << 20):
    return J._KvCacheDesc(heads, dh, bits, page, pages, ptr, ptr, ptr, ptr)


def test_quantized_linear_refusals(J):
    L = J.lib()

    def call(M=4, N=128, K=64, x=FAKE, xt=1, ldx=64, w=FAKE, s=FAKE, y=FAKE, yt=1, ldy=128, ws=FAKE, nb=1 << 40):
        return L.jab_quantized_linear(M, N, K, x, xt, ldx, w, s, y, yt, ldy, ws, nb, None)

    assert call(M=0) == OK and call(M=0, x=None) == OK
    for bad in (dict(x=None), dict(w=None), dict(s=None), dict(y=None), dict(ws=None), dict(M=-1), dict(N=0), dict(K=0), dict(xt=3), dict(yt=-1),
                dict(ldx=48), dict(ldx=65), dict(ldy=127), dict(x=ODD), dict(w=ODD), dict(ws=ODD), dict(nb=100)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(K=24, ldx=24), dict(K=131088, ldx=131088), dict(xt=2)):
        assert call(**bad) == UNSUPPORTED, bad
    assert J.jab_quantized_linear_workspace_size(4, 128, 24) == 0
    assert J.jab_quantized_linear_workspace_size(8, 128, 64) >= 8 * 64 * 2
    assert J.jab_quantized_linear_workspace_size(0, 128, 64) > 0


def test_cache_refusals(J):
    L = J.lib()

    def write(c, n=3, hq=2, x=FAKE, t=0, ld=6 * 64, slots=FAKE, pos=None, cos=None, sin=None, rl=0, q=FAKE):
        return L.jab_kv_write(ctypes.byref(c), n, hq, x, t, ld, slots, pos, cos, sin, rl, q, None)

    good = _cache(J)
    assert write(good, n=0) == OK
    for bad in (dict(x=None), dict(x=ODD), dict(slots=None), dict(n=-1), dict(hq=-1), dict(t=7), dict(ld=6 * 64 - 8), dict(ld=6 * 64 + 4), dict(q=ODD),
                dict(pos=FAKE), dict(pos=FAKE, cos=FAKE, sin=FAKE, rl=0), dict(cos=FAKE, sin=FAKE, rl=8)):
        assert write(good, **bad) == INVALID, bad
    for c in (_cache(J, heads=0), _cache(J, page=0), _cache(J, pages=0), _cache(J, ptr=0), _cache(J, ptr=(1 << 20) + 8)):
        assert write(c) == INVALID
    for c in (_cache(J, dh=96), _cache(J, bits=6), _cache(J, page=24), _cache(J, page=8192)):
        assert write(c) == UNSUPPORTED
    assert L.jab_kv_write(None, 3, 2, FAKE, 0, 384, FAKE, None, None, None, 0, None, None) == INVALID

    def read(c, B=2, pages=FAKE, mp=3, starts=None, counts=FAKE, T=5, k=FAKE, v=FAKE, t=0):
        return L.jab_kv_read(ctypes.byref(c), B, pages, mp, starts, counts, T, k, v, t, None)

    assert read(good, B=0) == OK and read(good, T=0) == OK
    for bad in (dict(pages=None), dict(counts=None), dict(k=None), dict(v=None), dict(k=ODD), dict(mp=0), dict(B=-1), dict(T=-1), dict(t=3)):
        assert read(good, **bad) == INVALID, bad
    assert L.jab_rope_table(0, 64, 10000.0, FAKE, FAKE, None) == INVALID
    assert L.jab_rope_table(8, 64, -1.0, FAKE, FAKE, None) == INVALID
    assert L.jab_rope_table(8, 80, 10000.0, FAKE, FAKE, None) == UNSUPPORTED


def test_attention_refusals(J):
    L = J.lib()

    def call(c, B=2, n=2, hq=4, q=FAKE, t=0, ldq=256, qs=FAKE, pages=FAKE, mp=4, lens=FAKE, mq=1, ml=64, sh=0, win=0, sc=0.0, o=FAKE, ldo=256, lse=None,
             ws=FAKE, nb=1 << 40):
        return L.jab_kv_attention(ctypes.byref(c), B, n, hq, q, t, ldq, qs, pages, mp, lens, mq, ml, sh, win, sc, o, ldo, lse, ws, nb, None)

    good = _cache(J)
    assert call(good, n=0) == OK
    for bad in (dict(q=None), dict(q=ODD), dict(qs=None), dict(pages=None), dict(lens=None), dict(o=None), dict(ws=None), dict(ws=ODD), dict(nb=64), dict(B=0),
                dict(n=-1), dict(hq=0), dict(mq=0), dict(ml=-1), dict(sh=-16), dict(sh=80), dict(win=-1), dict(sc=float("nan")), dict(ldq=248), dict(ldo=260),
                dict(mp=0), dict(t=9)):
        assert call(good, **bad) == INVALID, bad
    for bad in (dict(t=2), dict(hq=3), dict(sh=8), dict(B=5000), dict(mp=1 << 27)):
        assert call(good, **bad) == UNSUPPORTED, bad
    assert call(_cache(J, dh=32)) == UNSUPPORTED
    size = lambda **k: L.jab_kv_attention_workspace_size(ctypes.byref(good), 2, k.get("n", 2), k.get("hq", 4), k.get("mq", 1), 64, k.get("sh", 0))  # noqa: E731
    assert size() > 0 and size(hq=3) == 0 and size(n=-1) == 0 and size(sh=8) == 0
    assert size(mq=64, n=128) >= size()


def test_binding_refuses_wrong_tensors(J):
    import torch
    x = torch.zeros((2, 64))
    with pytest.raises(ValueError):
        J.jab_quantized_linear(x, torch.zeros((8, 64), dtype=torch.int8), torch.zeros(8), torch.zeros((2, 8)), torch.zeros(8, dtype=torch.uint8))
    with pytest.raises(ValueError):
        J.KvCache(2, 64, 6, 16, 4, device="cpu")
