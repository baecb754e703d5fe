"""sv_chunk_attention against the fp64 definition.

With smax the largest sum of a score's magnitudes (scale sum_d |q_d k_d|), a float32 score over D columns is off by at most
(D + 4) 2^-24 smax, and an exponential of it by 2^-22 of itself more (its argument's roundings in units of log2: 2^-24 (smax + |lse|) each for
product and difference).  Twice that is a weight's error, relative to the sum.  Sums over n keys add n 2^-24 of sum_j w_j |v_j|; for bfloat16
queries, weights are rounded to bfloat16 (2^-8 of each), and at the end the output is rounded once."""
import numpy as np
import pytest
import torch

import paper_2509_24328_amd as P
from oracle import model_side_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16, F8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def quantised(x):
    top = x.abs().amax(-1)
    s = torch.where(top > 0, top / 448.0, torch.ones_like(top))
    return (x / s[..., None]).to(F8), s


def held(cache):
    if cache.k.dtype != F8:
        return cache.k.cpu().double().numpy(), cache.v.cpu().double().numpy()
    k, v = (O.e4m3(t.view(torch.uint8).cpu().numpy()) for t in (cache.k, cache.v))
    return k * cache.k_scale.cpu().double().numpy()[..., None], v * cache.v_scale.cpu().double().numpy()[..., None]


def make(lengths, counts, heads, D, page, kind, seed=0, spare=1, garbage=True):
    """(cache, pages): what no sequence holds is NaN."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-(n + c) // page) for n, c in zip(lengths, counts)]
    max_pages, n_pages = max(max(need), 1) + spare, sum(need) + 2
    order = torch.randperm(n_pages, generator=g).tolist()
    pages = torch.full((len(lengths), max_pages), -1, dtype=torch.int32)
    shape = (n_pages, heads, page, D)
    k, v = torch.randn(shape, generator=g), torch.randn(shape, generator=g)
    here = torch.zeros(n_pages, page, dtype=torch.bool)
    for b, m in enumerate(need):
        for j in range(m):
            pages[b, j] = order.pop()
            here[pages[b, j], :min(page, lengths[b] + counts[b] - j * page)] = True
    gone = ~here[:, None, :, None].expand(shape)
    if kind == F8:
        (k, ks), (v, vs) = quantised(k), quantised(v)
        if garbage:
            k.view(torch.uint8)[gone] = 0x7F
            v.view(torch.uint8)[gone] = 0xFF
            ks[gone[..., 0]] = vs[gone[..., 0]] = float("nan")
        return P.Cache(k.cuda(), v.cuda(), ks.cuda(), vs.cuda()), pages
    if garbage:
        k[gone], v[gone] = float("nan"), float("inf")
    return P.Cache(k.to(kind).cuda(), v.to(kind).cuda()), pages


def run(cache, q, lengths, pages, offs, T, window=0, first=None, scale=None, ws=None, flags=True):
    i32 = lambda v: None if v is None else torch.as_tensor(v, dtype=torch.int32).cuda()
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:-1], 7.0, device="cuda")
    fl = torch.full(q.shape[:-2], 9, dtype=torch.int32, device="cuda")
    P.sv_chunk_attention(cache, q, out, i32(lengths), i32(pages), t_offsets=i32(offs), P=T, scale=scale, window=window, first=i32(first),
                         lse=lse, flags=fl, ws=ws)
    return out, lse, fl


def check(cache, q, got, lengths, pages, offs, T, window=0, first=None, scale=None):
    out, lse, fl = (t.cpu().double().numpy() for t in got)
    Hq, D = q.shape[-2:]
    scale = D ** -0.5 if scale is None else scale
    qd = q.cpu().double().numpy().reshape(-1, Hq, D)
    k, v = held(cache)
    ref, rlse, rfl, wabs, smax = O.attention(qd, k, v, lengths, np.asarray(pages), offs, T, scale, window, first)
    out, lse, fl = out.reshape(ref.shape), lse.reshape(rlse.shape), fl.reshape(-1)
    none = rfl < 0
    assert (out[none] == 7).all() and (lse[none] == 7).all() and (fl[none] == 9).all()
    assert np.array_equal(fl[~none], rfl[~none])
    bad = rfl == O.BAD_PAGE
    assert np.isnan(out[bad]).all() and np.isnan(lse[bad]).all()
    ok = rfl == 0
    n = max(lengths) + T
    dw = 2 * ((D + 4) * 2.0 ** -24 * smax + 2.0 ** -22 * (1 + smax + np.where(np.isfinite(rlse), np.abs(rlse), 0)))
    bf = 2.0 ** -8 if q.dtype == BF16 else 0.0
    tol = (dw[..., None] + n * 2.0 ** -24 + bf) * wabs + (2.0 ** -8 if q.dtype == BF16 else 2.0 ** -24) * np.abs(ref)
    with np.errstate(all="ignore"):
        same = (out == ref) | (np.isnan(out) & np.isnan(ref)) | (np.abs(out - ref) <= tol * (1 + 1e-6))
        same_l = (lse == rlse) | (np.isnan(lse) & np.isnan(rlse)) | (np.abs(lse - rlse) <= dw + n * 2.0 ** -24 + 2.0 ** -23 * np.abs(rlse))
    assert same[ok].all(), (np.argwhere(~same & ok[:, None, None])[:5], np.nanmax(np.abs(out - ref)[ok]))
    assert same_l[ok].all(), np.argwhere(~same_l & ok[:, None])[:5]


def queries(n, Hq, D, dtype, seed=1):
    return torch.randn((n, Hq, D), generator=torch.Generator().manual_seed(seed)).mul_(2).to(dtype).cuda()


TYPES = [(F32, F32), (BF16, BF16), (F32, F8), (BF16, F8)]


@pytest.mark.parametrize("D, page", [(64, 16), (128, 32), (256, 64), (80, 16), (128, 20), (8, 1), (200, 7), (72, 48)])
@pytest.mark.parametrize("dtype, kind", TYPES)
def test_widths_and_pages(dtype, kind, D, page):
    lengths, counts = [0, 1, 33, 130, 64], [3, 1, 3, 2, 3]
    cache, pages = make(lengths, counts, 2, D, page, kind, seed=D)
    offs = np.concatenate([[0], np.cumsum(counts)]).tolist()
    q = queries(offs[-1] + 2, 6, D, dtype)
    check(cache, q, run(cache, q, lengths, pages, offs, 3), lengths, pages, offs, 3)


@pytest.mark.parametrize("T, group", [(1, 1), (1, 16), (5, 3), (9, 7), (17, 1), (40, 2), (140, 1), (19, 8)])
@pytest.mark.parametrize("dtype, kind", TYPES)
def test_rows(dtype, kind, T, group):
    """One row to several row blocks; every layout of rows over wavefronts, dense and packed, with pages of whole tiles and of others."""
    for page in (16, 12):
        lengths, counts = [70, 3, 0], [T, max(1, T // 2), T]
        cache, pages = make(lengths, [T] * 3, 2, 64, page, kind, seed=T)
        q = queries(3 * T, 2 * group, 64, dtype)
        got = run(cache, q.view(3, T, 2 * group, 64), lengths, pages, None, None)
        check(cache, q, got, lengths, pages, None, T)
        offs = np.concatenate([[0], np.cumsum(counts)]).tolist()
        check(cache, q, run(cache, q, lengths, pages, offs, T), lengths, pages, offs, T)


@pytest.mark.parametrize("window, first", [(1, None), (5, None), (40, [0, 90, 3, 500]), (0, [0, 90, 103, 4]), (300, [-7, 1, 2, 203])])
@pytest.mark.parametrize("dtype, kind", TYPES)
def test_masks(dtype, kind, window, first):
    """Windows and left padding, some of which leave rows with nothing; pages that no row sees are not there."""
    lengths, counts = [50, 95, 100, 200], [9, 4, 9, 1]
    for D, page in ((64, 16), (40, 10)):
        cache, pages = make(lengths, counts, 1, D, page, kind)
        for b in range(4):
            lo = max(first[b] if first else 0, lengths[b] - window + 1 if window else 0, 0)
            pages[b, :lo // page] = -5
        offs = np.concatenate([[0], np.cumsum(counts)]).tolist()
        q = queries(offs[-1], 4, D, dtype)
        check(cache, q, run(cache, q, lengths, pages, offs, 9, window, first), lengths, pages, offs, 9, window, first)


@pytest.mark.parametrize("dtype, kind", TYPES)
@pytest.mark.parametrize("D, page", [(64, 16), (128, 16), (256, 16), (48, 5)])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(dtype, kind, D, page):
    """Keys and values of the new tokens themselves and of what a window has left behind: NaN and infinities reach the rows that see them, as
    the definition has it, and no other."""
    T, n = 6, 45
    for at in (n + 1, n + 4, n - 20, 3):
        for bad in ((float("nan"), float("inf"), float("-inf")) if kind != F8 else (float("nan"),)):
            cache, pages = make([n], [T], 1, D, page, kind, seed=at)
            pg, sl = pages[0, at // page].item(), at % page
            if kind == F8:
                cache.v.view(torch.uint8)[pg, 0, sl, 2] = 0x7F
            else:
                cache.v[pg, 0, sl, 2] = bad
            q = queries(T, 2, D, dtype)
            for window in (0, 24):
                check(cache, q, run(cache, q, [n], pages, [0, T], T, window), [n], pages, [0, T], T, window)
            if kind == F8:
                cache.k_scale[pg, 0, sl] = float("nan")
            else:
                cache.k[pg, 0, sl, 1] = bad
            got = run(cache, q, [n], pages, [0, T], T, 0)
            sees = n + np.arange(T) >= at
            assert np.array_equal(np.isfinite(got[0].float().cpu().numpy()).all((1, 2)), ~sees)


@pytest.mark.parametrize("page", [16, 6])
@pytest.mark.parametrize("dtype, kind", TYPES)
def test_pages_that_are_not_there(dtype, kind, page):
    """Rows that see a position in no page are NaN and flagged, the others of the same call are not touched by it."""
    lengths, counts, T = [40, 90, 60, -1, 2000, 90], [3, 3, 3, 2, 1, 9], 9
    cache, pages = make([40, 90, 60, 1, 1, 90], counts, 2, 64, page, kind, spare=0)
    pages[0, 1], pages[1, 90 // page] = cache.n_pages, -1
    pages[5, 2] = -7
    offs = np.concatenate([[0], np.cumsum(counts)]).tolist()
    q = queries(offs[-1], 4, 64, dtype)
    for window in (0, 30):
        check(cache, q, run(cache, q, lengths, pages, offs, T, window), lengths, pages, offs, T, window)
    lengths[2] = pages.shape[1] * page - 1               # the last position there is, then none
    check(cache, q, run(cache, q, lengths, pages, offs, T), lengths, pages, offs, T)


@pytest.mark.parametrize("T, group", [(9, 4), (12, 4), (6, 8), (33, 1), (7, 7)])
@pytest.mark.parametrize("D, page", [(128, 16), (112, 24), (64, 16)])
@pytest.mark.parametrize("kind", [F8, BF16])
def test_rows_between_two_blocks_and_four(kind, D, page, T, group):
    """33 to 49 rows to a head, and fewer in the sequences that have fewer tokens; lengths that are divided and lengths that are not."""
    lengths, counts = [1500, 3, 0, 700, 260], [T, max(1, T // 2), T, 1, T - 1]
    cache, pages = make(lengths, [T] * 5, 2, D, page, kind, seed=T)
    offs = np.concatenate([[0], np.cumsum(counts)]).tolist()
    q = queries(offs[-1], 2 * group, D, BF16)
    check(cache, q, run(cache, q, lengths, pages, offs, T), lengths, pages, offs, T)


@pytest.mark.parametrize("T", [1, 3, 7, 12])
@pytest.mark.parametrize("D, page", [(128, 16), (112, 24), (64, 16), (40, 8)])
@pytest.mark.parametrize("kind", [F8, BF16])
def test_many_sequences(kind, D, page, T):
    """270 heads of sequences that differ in length, some with no new tokens, some behind their pages, some with a window or a first position
    that leaves nothing; more sequences than a wavefront has lanes."""
    B, g = 135, torch.Generator().manual_seed(T)
    lengths = (torch.rand(B, generator=g) ** 6 * 1500).to(torch.int32).tolist()
    counts = torch.randint(0, T + 1, (B,), generator=g).tolist()
    lengths[:4], counts[:4] = [0, 1400, 5, 31], [T, T, 0, 1]
    cache, pages = make(lengths, [T] * B, 2, D, page, kind, seed=T)
    offs = np.concatenate([[0], np.cumsum(counts)]).tolist()
    q = queries(offs[-1], 8, D, BF16)
    got = run(cache, q, lengths, pages, offs, T)
    check(cache, q, got, lengths, pages, offs, T)
    again = run(cache, q, lengths, pages, offs, T)
    assert all(torch.equal(x.nan_to_num(3.0), y.nan_to_num(3.0)) for x, y in zip(got, again))
    lengths[7], lengths[90] = -1, 100000
    pages[1, 3] = -2
    first = [0] * B
    first[1], first[9], first[134] = 900, 5000, lengths[134]
    for window in (0, 50):
        check(cache, q, run(cache, q, lengths, pages, offs, T, window, first), lengths, pages, offs, T, window, first)


@pytest.mark.parametrize("dtype, kind", TYPES)
def test_long_sequences_are_divided(dtype, kind):
    """Lengths from 1 to 4000 in one call, with and without scratch: the parts of a long one are joined."""
    lengths, counts = [4000, 0, 700, 2500, 31], [2, 1, 3, 1, 3]
    cache, pages = make(lengths, counts, 2, 128, 16, kind)
    offs = np.concatenate([[0], np.cumsum(counts)]).tolist()
    q = queries(offs[-1], 8, 128, dtype)
    assert P.sv_chunk_attention_workspace_bytes(5, 3, 8, 2, 128, 0, pages.shape[1], 16) > 0
    got = run(cache, q, lengths, pages, offs, 3)
    check(cache, q, got, lengths, pages, offs, 3)
    L = P.binding.lib
    i32 = lambda v: torch.as_tensor(v, dtype=torch.int32).cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    le, pg, of = i32(lengths), i32(pages), i32(offs)
    c = cache._args
    assert L.sv_chunk_attention(q.data_ptr(), 8 * 128, of.data_ptr(), q.shape[0], le.data_ptr(), None, pg.data_ptr(), pages.shape[1], 5, 3, 8, 2,
                                128, int(dtype == BF16), c[0], c[1], c[2], c[3], c[4], c[5], c[6], 128 ** -0.5, 0, out.data_ptr(), 8 * 128,
                                lse.data_ptr(), None, None, 0, torch.cuda.current_stream().cuda_stream) == 0
    check(cache, q, (out, lse, got[2]), lengths, pages, offs, 3)
    again = run(cache, q, lengths, pages, offs, 3)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, again))


def test_large_scores_and_equal_keys():
    """Scores of several thousand, of either sign, and rows of equal scores."""
    lengths, T = [300], 2
    cache, pages = make(lengths, [T], 1, 64, 16, F32)
    for factor in (400.0, 1e-3, 0.0):
        q = queries(T, 2, 64, F32) * factor
        check(cache, q, run(cache, q, lengths, pages, [0, T], T), lengths, pages, [0, T], T)
    check(cache, q, run(cache, q, lengths, pages, [0, T], T, scale=-3.0), lengths, pages, [0, T], T, scale=-3.0)


def test_strided_rows_and_odd_addresses():
    lengths, T, Hq, D = [40, 20], 3, 4, 64
    cache, pages = make(lengths, [T, T], 2, D, 16, BF16)
    wide = torch.randn((2, T, Hq + 3, D), generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    flat = torch.zeros(wide.numel() + 3, dtype=BF16, device="cuda")
    flat[3:] = wide.view(-1)
    for base in (wide, flat[3:].view(wide.shape)):
        q = base[:, :, 2:2 + Hq]
        out = torch.zeros_like(wide)
        i32 = lambda v: torch.as_tensor(v, dtype=torch.int32).cuda()
        P.sv_chunk_attention(cache, q, out[:, :, 1:1 + Hq], i32(lengths), i32(pages))
        ref = run(cache, q.contiguous(), lengths, pages, None, None)[0]
        assert torch.equal(out[:, :, 1:1 + Hq], ref) and (out[:, :, 0] == 0).all() and (out[:, :, 1 + Hq:] == 0).all()


def test_another_stream_and_graph_replays():
    """Captured with device-side lengths: replays with other lengths, eager calls in between."""
    T, Hq, D, page = 3, 4, 64, 16
    cache, pages = make([600, 300], [T, T], 2, D, page, F8)
    q = queries(2 * T, Hq, D, BF16).view(2, T, Hq, D)
    i32 = lambda v: torch.as_tensor(v, dtype=torch.int32).cuda()
    le, pg = i32([600, 300]), i32(pages)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:-1], device="cuda")
    ws = torch.empty(P.sv_chunk_attention_workspace_bytes(2, T, Hq, 2, D, 1, pages.shape[1], page), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    P.sv_chunk_attention(cache, q, out, le, pg, lse=lse, ws=ws, stream=s)
    s.synchronize()
    first = out.clone()
    assert torch.equal(first, run(cache, q, [600, 300], pages, None, None)[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.sv_chunk_attention(cache, q, out, le, pg, lse=lse, ws=ws)
    for lengths in ([600, 300], [5, 299], [511, 0], [600, 300]):
        le.copy_(i32(lengths))
        out.zero_()
        graph.replay()
        ref = run(cache, q, lengths, pages, None, None)
        torch.cuda.synchronize()
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])


@pytest.mark.parametrize("T", [1, 12, 40])
@pytest.mark.parametrize("kind, n_pages, D, page", [(BF16, 140000, 128, 16), (BF16, 140000, 120, 17), (F8, 280000, 128, 16)])
def test_a_cache_beyond_32_bits(kind, n_pages, D, page, T):
    """Pages more than 2^32 bytes apart: the same numbers as from a small cache with the same pages, to the last bit."""
    lengths, used = [200, 37], [[n_pages - 1 - 3 * j for j in range(16)], [n_pages - 2 - 3 * j for j in range(15)] + [0]]
    used[0][5], used[1][1] = 3, n_pages // 2
    small, pages = make(lengths, [T] * 2, 8, D, page, kind, seed=T)
    pages = pages[:, :16]
    big = P.Cache.empty(n_pages, 8, page, D, kind)
    far = torch.full_like(pages, -1)
    for b in range(2):
        for j in range(pages.shape[1]):
            if pages[b, j] >= 0:
                far[b, j] = used[b][j]
                for to, of in zip(big._tensors, small._tensors):
                    if to is not None:
                        to[used[b][j]].view(torch.uint8).copy_(of[pages[b, j]].view(torch.uint8))
    q = queries(2 * T, 32, D, BF16).view(2, T, 32, D)
    for got, want in zip(run(big, q, lengths, far, None, None), run(small, q, lengths, pages, None, None)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype, kind", TYPES)
def test_shared_pages(dtype, kind):
    """Sequences that share their first pages, and a table that names one page twice."""
    lengths, T = [600, 600, 90], 5
    cache, pages = make(lengths, [T] * 3, 2, 64, 16, kind)
    pages[1, :30] = pages[0, :30]
    pages[2, 3] = pages[2, 1]
    q = queries(3 * T, 8, 64, dtype)
    check(cache, q, run(cache, q.view(3, T, 8, 64), lengths, pages, None, None), lengths, pages, None, T)


def test_two_calls_at_once():
    """Two batches over one cache on two streams, each with scratch of its own."""
    lengths, T = [3000, 20, 1500, 2500], 3
    cache, pages = make(lengths, [T] * 4, 2, 128, 16, BF16)
    q = queries(4 * T, 8, 128, BF16).view(4, T, 8, 128)
    i32 = lambda v: torch.as_tensor(v, dtype=torch.int32).cuda()
    n, table = i32(lengths), pages.cuda()
    calls = [(q, n, table), (q.flip(0).contiguous(), n.flip(0).contiguous(), table.flip(0).contiguous())]
    outs, streams = [torch.empty_like(q) for _ in calls], [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(20):
        for (x, le, pg), out, s in zip(calls, outs, streams):
            P.sv_chunk_attention(cache, x, out, le, pg, stream=s)
    torch.cuda.synchronize()
    want = run(cache, q, lengths, pages, None, None)[0]
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want.flip(0))


def test_nothing_to_do():
    cache, pages = make([3], [1], 1, 64, 16, BF16)
    q = torch.empty((0, 2, 64), dtype=BF16, device="cuda")
    run(cache, q, [], pages[:0], [0], 4)
    q = queries(4, 2, 64, BF16)
    out, lse, fl = run(cache, q, [3], pages, [2, 2], 4)
    assert (out == 7).all() and (lse == 7).all() and (fl == 9).all()
