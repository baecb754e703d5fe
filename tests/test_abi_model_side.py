"""Host checks of the model side of a step: refusals before anything is enqueued, scratch sizes, and the tensors a binding refuses.  No GPU is
needed, no pointer is dereferenced."""
import ctypes

import pytest
import torch

P = Bd = L = None


@pytest.fixture(scope="module", autouse=True)
def _library():
    """Imported here and not above: the oracle's pins are collected on machines without the library."""
    global P, Bd, L
    import __graft_entry__
    __graft_entry__.ensure_built()
    import paper_2509_24328_amd
    from paper_2509_24328_amd import binding
    P, Bd, L = paper_2509_24328_amd, binding, binding.lib


p = ctypes.c_void_p(256 * 1024)                       # non-NULL, aligned, never dereferenced
p2 = ctypes.c_void_p(512 * 1024)
odd = ctypes.c_void_p(256 * 1024 + 1)
four = ctypes.c_void_p(256 * 1024 + 4)
f, d = ctypes.c_float, ctypes.c_double
nan, inf = float("nan"), float("inf")


def test_rope_frequencies():
    call = lambda **k: L.sv_rope_frequencies(k.get("rot", 8), d(k.get("base", 1e4)), k.get("scaling", 0), d(k.get("factor", 2.0)),
                                             d(k.get("low", 1.0)), d(k.get("high", 4.0)), k.get("length", 100), k.get("freq", p), None)
    for bad in (dict(rot=0), dict(rot=7), dict(rot=-2), dict(base=1.0), dict(base=nan), dict(base=inf), dict(scaling=4), dict(scaling=-1),
                dict(scaling=1, factor=0.0), dict(scaling=2, factor=nan), dict(scaling=3, factor=inf), dict(scaling=3, low=-1.0),
                dict(scaling=3, low=4.0), dict(scaling=3, high=inf), dict(scaling=3, high=nan), dict(scaling=3, length=0)):
        assert call(**bad) == Bd.SV_ERR_INVALID_ARG, bad
    assert call(rot=1026) == Bd.SV_ERR_TOO_LARGE
    assert call(freq=None) == Bd.SV_ERR_NULL and call(freq=four) == Bd.SV_ERR_ALIGN


def test_rope():
    call = lambda **k: L.sv_rope(k.get("x", p), k.get("xs", 16), k.get("pos", p), k.get("n", 2), k.get("H", 2), k.get("D", 8), k.get("dt", 1),
                                 k.get("freq", p), k.get("rot", 8), k.get("layout", 0), f(k.get("amp", 1.0)), 0, k.get("out", p2),
                                 k.get("os", 16), None)
    for bad in (2, 3, -1):
        assert call(dt=bad) == Bd.SV_ERR_DTYPE
    for bad in (dict(n=-1), dict(H=0), dict(D=0), dict(rot=0), dict(rot=3), dict(rot=10), dict(layout=2), dict(amp=0.0), dict(amp=nan),
                dict(amp=inf), dict(xs=15), dict(os=15), dict(out=p, os=17)):
        assert call(**bad) == Bd.SV_ERR_INVALID_ARG, bad
    for bad in (dict(D=1025, xs=4096, os=4096), dict(H=1025, xs=1 << 20, os=1 << 20), dict(xs=1 << 40), dict(n=(1 << 25) + 1)):
        assert call(**bad) == Bd.SV_ERR_TOO_LARGE, bad
    for bad in ("x", "pos", "freq", "out"):
        assert call(**{bad: None}) == Bd.SV_ERR_NULL, bad
        assert call(**{bad: odd}) == Bd.SV_ERR_ALIGN, bad
    assert call(n=0) == Bd.SV_OK


def rows(k):
    return k.get("offs"), k.get("n_rows", 4), k.get("len", p), k.get("pages", p), k.get("mp", 3), k.get("B", 2), k.get("P", 2)


ROWS_INVALID = (dict(B=-1), dict(P=0), dict(n_rows=-1), dict(mp=0), dict(np=-1), dict(np=0), dict(heads=0), dict(page=0), dict(D=0))
ROWS_LARGE = (dict(page=65537), dict(B=1 << 16, P=1 << 16), dict(B=1 << 13, P=(1 << 12) + 1), dict(offs=p, n_rows=(1 << 25) + 1))


def write(**k):
    return L.sv_cache_write(k.get("k", p), k.get("ks", 16), k.get("v", p), k.get("vs", 16), k.get("q"), k.get("qs", 32), k.get("Hq", 4),
                            k.get("qo"), k.get("qos", 32), *rows(k), k.get("heads", 2), k.get("D", 8), k.get("dt", 1), k.get("freq"),
                            k.get("rot", 8), k.get("layout", 0), f(k.get("amp", 1.0)), k.get("kc", p), k.get("vc", p), k.get("ct", 1),
                            k.get("ksc"), k.get("vsc"), k.get("np", 5), k.get("page", 4), k.get("flags"), None)


def read(**k):
    offs, n_rows, start, pages, mp, B, P_ = rows(k)
    return L.sv_cache_read(k.get("kc", p), k.get("vc", p), k.get("ct", 1), k.get("ksc"), k.get("vsc"), k.get("np", 5), k.get("page", 4), offs,
                           n_rows, start, pages, mp, B, P_, k.get("heads", 2), k.get("D", 8), k.get("dt", 1), k.get("k", p), k.get("ks", 16),
                           k.get("v", p), k.get("vs", 16), k.get("flags"), None)


@pytest.mark.parametrize("call", [write, read])
def test_cache(call):
    for bad in (dict(dt=2, ct=2), dict(dt=3, ct=3), dict(dt=0, ct=1), dict(dt=1, ct=0), dict(ct=3)):
        assert call(**bad) == Bd.SV_ERR_DTYPE, bad
    for bad in ROWS_INVALID + (dict(ks=15), dict(vs=15)):
        assert call(**bad) == Bd.SV_ERR_INVALID_ARG, bad
    for bad in ROWS_LARGE + (dict(D=1025, ks=4096, vs=4096), dict(heads=1025, ks=1 << 20, vs=1 << 20), dict(ks=1 << 40), dict(vs=1 << 40)):
        assert call(**bad) == Bd.SV_ERR_TOO_LARGE, bad
    for bad in ("k", "v", "len", "pages", "kc", "vc"):
        assert call(**{bad: None}) == Bd.SV_ERR_NULL, bad
        assert call(**{bad: odd}) == Bd.SV_ERR_ALIGN, bad
    for bad in ("offs", "flags"):
        assert call(**{bad: odd}) == Bd.SV_ERR_ALIGN, bad
    assert call(ct=2) == Bd.SV_ERR_NULL and call(ct=2, ksc=p) == Bd.SV_ERR_NULL and call(ct=2, ksc=p, vsc=odd) == Bd.SV_ERR_ALIGN
    assert call(B=0) == Bd.SV_OK and call(offs=p, n_rows=0) == Bd.SV_OK


def test_cache_write_with_queries():
    assert write(q=p) == Bd.SV_ERR_NULL and write(qo=p) == Bd.SV_ERR_NULL
    for bad in (dict(Hq=0), dict(qs=31), dict(qos=31), dict(qo=p, qos=40), dict(freq=p, rot=7), dict(freq=p, rot=10), dict(freq=p, layout=5),
                dict(freq=p, amp=-1.0), dict(freq=p, amp=nan)):
        assert write(**{**dict(q=p, qo=p2), **bad}) == Bd.SV_ERR_INVALID_ARG, bad
    assert write(q=p, qo=p2, Hq=1025, qs=1 << 20, qos=1 << 20) == Bd.SV_ERR_TOO_LARGE
    assert write(q=odd, qo=p2) == Bd.SV_ERR_ALIGN and write(q=p, qo=odd) == Bd.SV_ERR_ALIGN and write(freq=four) == Bd.SV_ERR_ALIGN


def attend(**k):
    offs, n_rows, start, pages, mp, B, P_ = rows(k)
    return L.sv_chunk_attention(k.get("q", p), k.get("qs", 32), offs, n_rows, start, k.get("first"), pages, mp, B, P_, k.get("Hq", 4),
                                k.get("heads", 2), k.get("D", 8), k.get("dt", 1), k.get("kc", p), k.get("vc", p), k.get("ct", 1), k.get("ksc"),
                                k.get("vsc"), k.get("np", 5), k.get("page", 4), f(k.get("scale", 1.0)), k.get("window", 0), k.get("out", p2),
                                k.get("os", 32), k.get("lse"), k.get("flags"), k.get("ws"), k.get("wsb", 0), None)


def test_chunk_attention():
    for bad in (dict(dt=2, ct=2), dict(dt=0, ct=1), dict(ct=3)):
        assert attend(**bad) == Bd.SV_ERR_DTYPE, bad
    for bad in ROWS_INVALID + (dict(Hq=1), dict(Hq=5), dict(Hq=0), dict(D=12), dict(D=4), dict(window=-1), dict(scale=nan), dict(scale=inf),
                               dict(qs=31), dict(os=31), dict(out=p)):
        assert attend(**bad) == Bd.SV_ERR_INVALID_ARG, bad
    for bad in ROWS_LARGE + (dict(D=264, qs=4096, os=4096), dict(Hq=2048, qs=1 << 20, os=1 << 20), dict(qs=1 << 40), dict(os=1 << 40),
                             dict(B=1 << 13, P=1 << 14), dict(offs=p, B=1 << 13, P=1 << 13, Hq=2), dict(B=1 << 24, P=1 << 1, Hq=16, qs=128, os=128)):
        assert attend(**bad) == Bd.SV_ERR_TOO_LARGE, bad
    for bad in ("q", "len", "pages", "kc", "vc", "out"):
        assert attend(**{bad: None}) == Bd.SV_ERR_NULL, bad
        assert attend(**{bad: odd}) == Bd.SV_ERR_ALIGN, bad
    for bad in ("offs", "flags", "lse", "first"):
        assert attend(**{bad: odd}) == Bd.SV_ERR_ALIGN, bad
    assert attend(ct=2) == Bd.SV_ERR_NULL and attend(ct=2, ksc=odd, vsc=p) == Bd.SV_ERR_ALIGN
    long = dict(mp=64, page=16)
    need = P.sv_chunk_attention_workspace_bytes(2, 2, 4, 2, 8, 1, 64, 16)
    assert need > 0 and need % 256 == 0
    assert attend(ws=four, wsb=need, **long) == Bd.SV_ERR_WORKSPACE and attend(ws=p, wsb=need - 1, **long) == Bd.SV_ERR_WORKSPACE
    assert attend(B=0) == Bd.SV_OK and attend(offs=p, n_rows=0) == Bd.SV_OK


def test_chunk_attention_scratch():
    w = P.sv_chunk_attention_workspace_bytes
    ok = (2, 2, 4, 2, 64, 1, 64, 16)
    for i, bad in ((0, 0), (1, 0), (2, 5), (2, 2048), (3, 0), (4, 12), (4, 264), (5, 2), (6, 0), (7, 0), (7, 65537)):
        assert w(*ok[:i], bad, *ok[i + 1:]) == 0, (i, bad)
    assert w(1, 1, 4, 4, 64, 1, 1, 16) == 0                # (one page: nothing to divide)
    for shape in ((1, 1, 32, 8, 128, 1, 1024, 16), (64, 9, 32, 8, 128, 1, 1024, 16), (1, 2048, 32, 8, 128, 1, 1024, 16),
                  (300, 1, 8, 8, 256, 0, 4096, 16), (1, 1, 1024, 1, 256, 0, 65536, 65536), (1 << 18, 1, 1024, 1024, 256, 1, 1, 1)):
        assert 0 <= w(*shape) <= (1 << 28), shape          # however large the call: parts are kept to what the last-level cache holds


def test_sample():
    call = lambda **k: L.sv_sample(k.get("z", p), k.get("zs", 8), k.get("rows", 2), k.get("V", 8), k.get("dt", 1), f(k.get("T", 1.0)),
                                   k.get("K", 0), f(k.get("top_p", 1.0)), f(k.get("min_p", 0.0)), k.get("u", p), k.get("token", p),
                                   k.get("lp"), k.get("flags"), k.get("ws"), k.get("wsb", 0), None)
    for bad in (2, -1, 7):
        assert call(dt=bad) == Bd.SV_ERR_DTYPE
    for bad in (dict(rows=-1), dict(V=0), dict(zs=7), dict(T=0.0), dict(T=1e-4), dict(T=nan), dict(top_p=0.0), dict(top_p=nan), dict(min_p=-0.1),
                dict(min_p=1.5), dict(min_p=nan)):
        assert call(**bad) == Bd.SV_ERR_INVALID_ARG, bad
    assert call(V=(1 << 24) + 1, zs=1 << 25) == Bd.SV_ERR_TOO_LARGE and call(zs=1 << 40) == Bd.SV_ERR_TOO_LARGE
    for bad in ("z", "u", "token"):
        assert call(**{bad: None}) == Bd.SV_ERR_NULL, bad
        assert call(**{bad: odd}) == Bd.SV_ERR_ALIGN, bad
    assert call(u=four) == Bd.SV_ERR_ALIGN and call(lp=odd) == Bd.SV_ERR_ALIGN and call(flags=odd) == Bd.SV_ERR_ALIGN
    need = P.sv_sample_workspace_bytes(2, 152064, 1)
    assert need > 0 and need % 256 == 0
    assert call(V=152064, zs=152064, ws=four, wsb=need) == Bd.SV_ERR_WORKSPACE
    assert call(V=152064, zs=152064, ws=p, wsb=need - 1) == Bd.SV_ERR_WORKSPACE
    assert call(rows=0) == Bd.SV_OK
    w = P.sv_sample_workspace_bytes
    assert w(0, 152064, 1) == 0 and w(2, 0, 1) == 0 and w(2, (1 << 24) + 1, 1) == 0 and w(2, 152064, 2) == 0 and w(2, 100, 1) == 0


def test_cache_tensors():
    t = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)
    F8 = torch.float8_e4m3fn
    code = lambda *a, **k: pytest.raises(Bd.SvError, Bd.Cache, *a, **k).value.status
    k, s = t(3, 2, 4, 8), t(3, 2, 4)
    assert code(t(3, 2, 32), t(3, 2, 32)) == Bd.SV_ERR_INVALID_ARG
    assert code(k, t(3, 2, 4, 16)) == Bd.SV_ERR_INVALID_ARG
    assert code(k, k.bfloat16()) == Bd.SV_ERR_DTYPE and code(k.half(), k.half()) == Bd.SV_ERR_DTYPE
    assert code(k, k, s, s) == Bd.SV_ERR_INVALID_ARG
    q = k.to(F8)
    assert code(q, q) == Bd.SV_ERR_NULL and code(q, q, s) == Bd.SV_ERR_NULL
    assert code(q, q, s, t(3, 2, 5)) == Bd.SV_ERR_INVALID_ARG
