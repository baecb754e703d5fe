"""sv_cache_write and sv_cache_read against the fp64 definitions.

A stored column is off by half a step of its type: 2^-24 or 2^-8 of itself, or in 8 bits 2^-4 of itself plus half the smallest step, 2^-10
of the scale; a scale by half a float32 step.  Reading back rounds once more.  Turning in fp64 adds 1e-8 of a pair."""
import numpy as np
import pytest
import torch

import paper_2509_24328_amd as P
from oracle import model_side_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16, F8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def held(cache):
    """Keys and values of a cache as float64."""
    if cache.k.dtype != F8:
        return cache.k.cpu().double().numpy(), cache.v.cpu().double().numpy()
    k, v = (O.e4m3(t.view(torch.uint8).cpu().numpy()) for t in (cache.k, cache.v))
    return k * cache.k_scale.cpu().double().numpy()[..., None], v * cache.v_scale.cpu().double().numpy()[..., None]


def setup(B, P_, heads, D, page, dtype, kind, max_pages, seed=0):
    g = torch.Generator().manual_seed(seed)
    n_pages = B * max_pages + 3
    cache = P.Cache.empty(n_pages, heads, page, D, kind)
    for t in (cache.k, cache.v):
        t.view(torch.uint8).fill_(0x3C)
    if kind == F8:
        cache.k_scale.fill_(0.5)
        cache.v_scale.fill_(0.5)
    pages = torch.randperm(n_pages, generator=g)[:B * max_pages].view(B, max_pages).to(torch.int32)
    return g, cache, pages


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("page, D, rot, pairs", [(16, 64, 64, False), (7, 80, 40, True), (1, 24, 0, False), (64, 128, 128, False), (20, 9, 2, True),
                                                 (16, 256, 2, False)])
@pytest.mark.parametrize("dtype, kind", [(F32, F32), (BF16, BF16), (F32, F8), (BF16, F8)])
def test_write_and_read(dtype, kind, page, D, rot, pairs, packed):
    B, T, heads, Hq, max_pages = 4, 5, 3, 6, 12
    g, cache, pages = setup(B, T, heads, D, page, dtype, kind, max_pages, seed=page + D)
    counts = [5, 0, 1, 3] if packed else [T] * B
    offs = np.concatenate([[0], np.cumsum(counts)])
    n_rows = int(offs[-1]) + (2 if packed else 0)
    lengths = torch.tensor([0, 3, 7, 2], dtype=torch.int32)
    wide = torch.randn((n_rows, Hq + 2 * heads, D), generator=g).to(dtype).cuda()
    wide[0, Hq] = 0.0                                     # a head of zeros
    wide[0, Hq + heads] *= 1e-30
    q, k, v = wide[:, :Hq], wide[:, Hq:Hq + heads], wide[:, Hq + heads:]
    q_out = torch.full((n_rows, Hq, D), 7.0, dtype=dtype, device="cuda")
    flags = torch.full((n_rows,), 9, dtype=torch.int32, device="cuda")
    freq = torch.from_numpy(O.frequencies(rot)).cuda() if rot else None
    was = held(cache)
    t_off = torch.from_numpy(offs).to(torch.int32).cuda() if packed else None
    shape = (lambda t: t) if packed else (lambda t: t.unflatten(0, (B, T)))
    P.sv_cache_write(cache, shape(k), shape(v), lengths.cuda(), pages.cuda(), t_offsets=t_off, P=T, q=shape(q), q_out=shape(q_out),
                     freq=freq, layout=int(pairs), amplitude=1.0, flags=flags if packed else flags.view(B, T))
    torch.cuda.synchronize()
    now = held(cache)
    x = wide.cpu().double().numpy()
    want_q = np.full((n_rows, Hq, D), 7.0)
    want_flags = np.full(n_rows, 9)
    back = [np.full((n_rows, heads, D), 7.0) for _ in range(2)]
    touched = np.zeros(was[0].shape[:3], bool)
    for r, b, i in O.rows_of(offs.tolist() if packed else None, n_rows, B, T):
        p = int(lengths[b]) + i
        turn = lambda y: O.turned(y[None], [p], O.frequencies(rot), pairs)[0] if rot else y
        want_q[r] = turn(x[r, :Hq])
        at = O.place(pages.numpy(), b, p, page, cache.n_pages)
        want_flags[r] = 0 if at else O.BAD_PAGE
        for j, y in enumerate((turn(x[r, Hq:Hq + heads]), x[r, Hq + heads:])):
            if at is None:
                back[j][r] = np.nan
                continue
            touched[at[0], :, at[1]] = True
            got = now[j][at[0], :, at[1]]
            back[j][r] = got
            if kind == F8:
                s = O.scale_of(y)
                scale = (cache.k_scale, cache.v_scale)[j][at[0], :, at[1]].cpu().double().numpy()
                assert np.allclose(scale, s, rtol=2.0 ** -22, atol=0)
                tol = 2.0 ** -4 * np.abs(y) + 2.0 ** -10 * s[:, None]
            else:
                tol = HALF[dtype] * np.abs(y)
            assert (np.abs(got - y) <= tol * (1 + 1e-6) + 1e-8 * (j == 0) * (rot > 0)).all()
    assert np.array_equal(flags.cpu().numpy(), want_flags)
    assert (np.abs(q_out.cpu().double().numpy() - want_q) <= HALF[dtype] * np.abs(want_q) * (1 + 1e-6) + 1e-8).all()
    for j in range(2):                                    # nothing else was written
        assert np.array_equal(now[j][~touched], was[j][~touched])
    k2, v2 = (torch.full((n_rows, heads, D), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    flags.fill_(9)
    P.sv_cache_read(cache, shape(k2), shape(v2), lengths.cuda(), pages.cuda(), t_offsets=t_off, P=T,
                    flags=flags if packed else flags.view(B, T))
    assert np.array_equal(flags.cpu().numpy(), want_flags)
    for got, ref in ((k2, back[0]), (v2, back[1])):
        got = got.cpu().double().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        ok = ~np.isnan(ref)
        assert (np.abs(got - ref)[ok] <= HALF[dtype] * np.abs(ref[ok]) * (kind == F8)).all()


@pytest.mark.parametrize("kind", [BF16, F8])
def test_positions_in_no_page(kind):
    """Entries outside the cache, a table that ends, a length below 0 or near 2^31: flagged, nothing written, NaN read."""
    B, T, heads, D, page, max_pages = 5, 3, 2, 16, 4, 2
    g, cache, pages = setup(B, T, heads, D, page, BF16, kind, max_pages)
    pages[0, 0], pages[1, 0] = -1, cache.n_pages
    lengths = torch.tensor([2, 2, 6, -1, 0x7FFFFFFE], dtype=torch.int32)
    was = held(cache)
    k, v, k2, v2 = (torch.randn((B, T, heads, D), generator=g).to(BF16).cuda() for _ in range(4))
    flags = torch.full((B, T), 9, dtype=torch.int32, device="cuda")
    P.sv_cache_write(cache, k, v, lengths.cuda(), pages.cuda(), flags=flags)
    want = np.array([[256, 256, 0], [256, 256, 0], [0, 0, 256], [256] * 3, [256] * 3])
    assert np.array_equal(flags.cpu().numpy(), want)
    now = held(cache)
    assert (now[0] != was[0]).any((1, 3)).sum() == 4 and (now[1] != was[1]).any((1, 3)).sum() == 4
    P.sv_cache_read(cache, k2, v2, lengths.cuda(), pages.cuda(), flags=flags)
    assert np.array_equal(flags.cpu().numpy(), want)
    assert np.array_equal(torch.isnan(k2).all(-1).all(-1).cpu().numpy(), want == 256)
    assert not torch.isnan(v2.cpu()[torch.from_numpy(want == 0)]).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_heads_that_are_not_finite_and_extreme_scales(dtype):
    B, T, heads, D, page = 1, 6, 2, 32, 16
    g, cache, pages = setup(B, T, heads, D, page, dtype, F8, 1)
    k = torch.randn((B, T, heads, D), generator=g).to(dtype)
    k[0, 0, 0, 5], k[0, 1, 1, 31], k[0, 2, 0, 0] = float("nan"), float("inf"), float("-inf")
    k[0, 3] = 1e-38 * k[0, 3]                             # the scale is its smallest
    k[0, 4] = 1e37 * k[0, 4]
    k[0, 5, :, 1:] = 0.0
    P.sv_cache_write(cache, k.cuda(), k.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"), pages.cuda())
    got = held(cache)[0][pages[0, 0].item()].transpose(1, 0, 2)[:T]
    ref = k[0].double().numpy()
    bad = ~np.isfinite(ref).all(-1)
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()
    s = O.scale_of(ref)[~bad][:, None]
    assert (np.abs(got - ref)[~bad] <= 2.0 ** -4 * np.abs(ref[~bad]) * (1 + 1e-6) + 2.0 ** -10 * s).all()
    assert np.array_equal(held(cache)[0], held(cache)[1], equal_nan=True)


def test_rows_beyond_32_bits():
    """A cache of more than 2^32 elements, its last page used."""
    heads, page, D = 8, 128, 256
    n_pages = (1 << 32) // (heads * page * D) + 3
    cache = P.Cache.empty(n_pages, heads, page, D, BF16)
    pages = torch.tensor([[n_pages - 1]], dtype=torch.int32, device="cuda")
    k, v = (torch.randn((1, 2, heads, D), device="cuda").to(BF16) for _ in range(2))
    at = torch.tensor([100], dtype=torch.int32, device="cuda")
    P.sv_cache_write(cache, k, v, at, pages)
    assert torch.equal(cache.k[-1, :, 100:102].transpose(0, 1), k[0]) and torch.equal(cache.v[-1, :, 100:102].transpose(0, 1), v[0])
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    P.sv_cache_read(cache, k2, v2, at, pages)
    assert torch.equal(k, k2) and torch.equal(v, v2)


def test_batches_longer_than_a_wavefront():
    """The sequence of a packed row among 150 of them, some without rows; groups of four rows (5000 of them)."""
    g = torch.Generator().manual_seed(5)
    B, heads, D, page = 150, 1, 8, 16
    counts = torch.randint(0, 70, (B,), generator=g)
    counts[::7] = 0
    T = int(counts.max())
    offs = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)])
    n = int(offs[-1])
    assert n > 4096
    max_pages = (T + 40) // page + 1
    cache = P.Cache.empty(B * max_pages, heads, page, D, F32)
    pages = torch.randperm(B * max_pages, generator=g).view(B, max_pages).to(torch.int32)
    lengths = torch.randint(0, 40, (B,), generator=g).to(torch.int32)
    k, v = (torch.randn((n + 3, heads, D), generator=g).cuda() for _ in range(2))
    cu = lambda t: t.to(torch.int32).cuda()
    P.sv_cache_write(cache, k, v, cu(lengths), cu(pages), t_offsets=cu(offs), P=T)
    b = torch.repeat_interleave(torch.arange(B), counts)
    pos = lengths.long()[b] + torch.arange(n) - offs[b]
    pg, sl = pages.long()[b, pos // page].cuda(), (pos % page).cuda()
    assert torch.equal(cache.k[pg, :, sl], k[:n]) and torch.equal(cache.v[pg, :, sl], v[:n])
    k2, v2 = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    P.sv_cache_read(cache, k2, v2, cu(lengths), cu(pages), t_offsets=cu(offs), P=T)
    assert torch.equal(k2[:n], k[:n]) and (k2[n:] == 3).all() and torch.equal(v2[:n], v[:n])
