"""Host checks of the operators around the decode step: refusals before anything is enqueued, scratch sizes, and
the outputs a binding refuses.  No GPU is needed, no pointer is dereferenced."""
import ctypes

import pytest

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
odd = ctypes.c_void_p(256 * 1024 + 1)
f = ctypes.c_float


def test_token_logprobs():
    call = lambda **k: L.sv_token_logprobs(
        k.get("z", p), k.get("stride", 8), k.get("offs"), k.get("n_rows", 0), k.get("tok", p), k.get("B", 2), k.get("P", 2),
        k.get("V", 8), k.get("dt", 1), f(k.get("T", 1.0)), k.get("top", 0), k.get("lp", p), None, None, k.get("rank"),
        k.get("tt"), k.get("tl"), k.get("flags"), k.get("ws"), k.get("wsb", 0), None)
    assert call(dt=2) == Bd.SV_ERR_DTYPE
    for bad in (dict(B=-1), dict(P=0), dict(V=0), dict(stride=7), dict(top=-1), dict(offs=p, n_rows=-1), dict(T=0.0),
                dict(T=float("nan")), dict(T=1e4)):
        assert call(**bad) == Bd.SV_ERR_INVALID_ARG, bad
    assert call(V=1 << 25, stride=1 << 25) == Bd.SV_ERR_TOO_LARGE
    assert call(top=33, tt=p, tl=p) == Bd.SV_ERR_TOO_LARGE
    assert call(B=1 << 20, P=1 << 20) == Bd.SV_ERR_TOO_LARGE
    for bad in (dict(z=None), dict(tok=None), dict(tok=None, lp=None, rank=p), dict(top=1, tt=p), dict(top=1, tl=p)):
        assert call(**bad) == Bd.SV_ERR_NULL, bad
    for bad in (dict(z=odd), dict(tok=odd), dict(lp=odd), dict(rank=odd), dict(flags=odd), dict(offs=odd)):
        assert call(**bad) == Bd.SV_ERR_ALIGN, bad
    assert call(V=152064, stride=152064, ws=odd, wsb=1 << 30) == Bd.SV_ERR_WORKSPACE
    assert call(V=152064, stride=152064, ws=p, wsb=64) == Bd.SV_ERR_WORKSPACE
    assert call(B=0) == Bd.SV_OK


def test_token_logprobs_grad():
    call = lambda **k: L.sv_token_logprobs_grad(
        k.get("z", p), k.get("stride", 8), k.get("tok", p), k.get("rows", 2), k.get("V", 8), k.get("dt", 1),
        f(k.get("T", 1.0)), k.get("g", p), k.get("h"), None, None, k.get("dz", p), k.get("ds", 8), None, k.get("ws"),
        k.get("wsb", 0), None)
    assert call(dt=-1) == Bd.SV_ERR_DTYPE
    for bad in (dict(rows=-1), dict(V=0), dict(stride=7), dict(ds=7), dict(ds=9), dict(T=-1.0)):
        assert call(**bad) == Bd.SV_ERR_INVALID_ARG, bad
    assert call(V=1 << 25, stride=1 << 25, ds=1 << 25) == Bd.SV_ERR_TOO_LARGE
    for bad in (dict(z=None), dict(dz=None), dict(tok=None), dict(g=None)):
        assert call(**bad) == Bd.SV_ERR_NULL, bad
    for bad in (dict(z=odd), dict(dz=odd), dict(h=odd)):
        assert call(**bad) == Bd.SV_ERR_ALIGN, bad
    assert call(V=152064, stride=152064, ds=152064, ws=p, wsb=8) == Bd.SV_ERR_WORKSPACE
    assert call(rows=0) == Bd.SV_OK


def test_embedding():
    call = lambda **k: L.sv_embedding(k.get("w", p), k.get("ids", p), k.get("n", 2), k.get("V", 8), k.get("D", 4),
                                      k.get("dt", 1), f(1.0), k.get("out", p), k.get("flags"), None)
    assert call(dt=3) == Bd.SV_ERR_DTYPE
    for bad in (dict(n=-1), dict(V=0), dict(D=0)):
        assert call(**bad) == Bd.SV_ERR_INVALID_ARG, bad
    assert call(V=1 << 25) == Bd.SV_ERR_TOO_LARGE and call(D=1 << 21) == Bd.SV_ERR_TOO_LARGE
    for bad in (dict(w=None), dict(ids=None), dict(out=None)):
        assert call(**bad) == Bd.SV_ERR_NULL, bad
    for bad in (dict(w=odd), dict(ids=odd), dict(out=odd), dict(flags=odd)):
        assert call(**bad) == Bd.SV_ERR_ALIGN, bad
    assert call(n=0) == Bd.SV_OK
    need = P.sv_embedding_grad_workspace_bytes(2, 8, 4)
    call = lambda **k: L.sv_embedding_grad(k.get("g", p), k.get("dt", 1), k.get("ids", p), k.get("n", 2), k.get("V", 8),
                                           k.get("D", 4), f(1.0), k.get("w", p), k.get("wt", 0), k.get("acc", 0),
                                           k.get("ws", p), k.get("wsb", need), None)
    assert call(dt=3) == Bd.SV_ERR_DTYPE and call(wt=3) == Bd.SV_ERR_DTYPE
    for bad in (dict(n=-1), dict(V=0), dict(D=0)):
        assert call(**bad) == Bd.SV_ERR_INVALID_ARG, bad
    assert call(n=(1 << 24) + 1) == Bd.SV_ERR_TOO_LARGE
    for bad in (dict(g=None), dict(ids=None), dict(w=None), dict(n=0, w=None)):
        assert call(**bad) == Bd.SV_ERR_NULL, bad
    for bad in (dict(g=odd), dict(ids=odd), dict(w=odd)):
        assert call(**bad) == Bd.SV_ERR_ALIGN, bad
    for bad in (dict(ws=None), dict(ws=odd), dict(wsb=need - 1)):
        assert call(**bad) == Bd.SV_ERR_WORKSPACE, bad
    assert call(n=0, acc=1, w=None, g=None, ids=None, ws=None) == Bd.SV_OK


def test_grad_norm():
    def call(n=2, g=(p, p), numel=(4, 4), dt=(0, 1), out=(p, p), odt=(0, 1), M=1.0, norm=p, ws=p, wsb=1 << 20):
        arr = lambda a: (ctypes.c_void_p * len(a))(*[x.value if x is not None else None for x in a])
        return L.sv_clip_grad_norm(n, arr(g), (ctypes.c_longlong * len(numel))(*numel), (ctypes.c_int * len(dt))(*dt),
                                   f(M), arr(out) if out else None, (ctypes.c_int * len(odt))(*odt), norm, None, ws,
                                   ctypes.c_size_t(wsb), None)
    assert call(dt=(0, 2)) == Bd.SV_ERR_DTYPE and call(odt=(0, 2)) == Bd.SV_ERR_DTYPE
    for bad in (dict(n=-1), dict(numel=(4, -1)), dict(M=0.0), dict(M=-1.0), dict(M=float("nan")), dict(odt=(1, 1))):
        assert call(**bad) == Bd.SV_ERR_INVALID_ARG, bad
    assert call(numel=(4, 1 << 45)) == Bd.SV_ERR_TOO_LARGE
    for bad in (dict(g=(p, None)), dict(out=(p, None)), dict(out=None), dict(norm=None)):
        assert call(**bad) == Bd.SV_ERR_NULL, bad
    for bad in (dict(g=(p, odd)), dict(out=(odd, p)), dict(norm=odd)):
        assert call(**bad) == Bd.SV_ERR_ALIGN, bad
    for bad in (dict(ws=None), dict(ws=odd), dict(wsb=256)):
        assert call(**bad) == Bd.SV_ERR_WORKSPACE, bad


def test_scratch_sizes():
    w = P.sv_token_logprobs_workspace_bytes
    assert w(1, 152064, P.SV_BF16, 20) > 0 and w(1, 152064, P.SV_BF16, 20) % 256 == 0
    assert w(1, 152064, P.SV_BF16, 20) > w(1, 152064, P.SV_BF16, 0)
    assert w(100000, 152064, P.SV_BF16, 20) == 0 and w(1, 1000, P.SV_F32, 5) == 0 and w(0, 152064, P.SV_F32, 0) == 0
    assert w(-1, 100, 0, 0) == 0 and w(1, 0, 0, 0) == 0 and w(1, 100, 5, 0) == 0 and w(1, 100, 0, 33) == 0
    e = P.sv_embedding_grad_workspace_bytes
    for n in (0, 1, 4096, 4097, 65536, 1 << 24):
        assert e(n, 152064, 2048) >= 256 and e(n, 152064, 2048) % 256 == 0
    assert e(5, 0, 1) == 0 and e(5, 1, 0) == 0 and e(-1, 1, 1) == 0
    g = P.sv_grad_norm_workspace_bytes
    assert g(0) > 0 and g(121) > g(120) and g(-1) == 0
