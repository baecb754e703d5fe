"""Target and draft with an attention layer over a paged cache: their logits, chunk by chunk with tokens taken back, against the whole
sequence in float64, and that the command runs with them."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def held(m, b, n):
    """Keys and values of sequence b's first n positions as its cache has them, [n, heads, width] in float64."""
    c = m.cache
    at = m.pages[b].cpu().long().repeat_interleave(c.page)[:n], torch.arange(n) % c.page
    rows = [t.cpu().double()[at[0], :, at[1]] for t in (c.k, c.v)]
    if c.k_scale is None:
        return rows
    return [r * s.cpu().double()[at[0], :, at[1]][..., None] for r, s in zip(rows, (c.k_scale, c.v_scale))]


def whole(m, tokens, cached=None):
    """(logits after every token of one sequence, keys, values) in float64 and from the formulas; cached: over these keys and values."""
    table, qkv, out, layer = (t.double().cpu() for t in (m.table, m.qkv, m.out, m.layer))
    n, w, half = len(tokens), m.width, m.width // 2
    x = table[tokens.cpu().long()] * m.scale
    q, k, v = (t.unflatten(-1, (-1, w)) for t in (x @ qkv).split([m.heads * w, m.heads * w // 2, m.heads * w // 2], -1))
    t = torch.arange(n, dtype=torch.float64)[:, None] * (10000.0 ** (-2.0 * torch.arange(half, dtype=torch.float64) / w))
    c, s = t.cos()[:, None], t.sin()[:, None]
    turn = lambda y: torch.cat([y[..., :half] * c - y[..., half:] * s, y[..., half:] * c + y[..., :half] * s], -1)
    q, k = turn(q).transpose(0, 1), turn(k)
    own = k, v
    k, v = cached or own
    k, v = (t.transpose(0, 1).repeat_interleave(2, 0) for t in (k, v))
    a = (q @ k.transpose(1, 2)) * w ** -0.5
    a = a.masked_fill(torch.ones(n, n).triu(1).bool(), float("-inf")).softmax(-1)
    o = (a @ v).transpose(0, 1).reshape(n, -1)
    return m.gain * (torch.tanh((x + o @ out) @ layer) @ table.t()), *own


@pytest.mark.parametrize("cache", [torch.float32, F8], ids=str)
def test_chunks_and_tokens_taken_back(cache):
    """Five products one after the other, of sums over at most 64 terms, each off by at most 64 * 2^-24 of its terms' magnitudes, which are some
    eight times the sum: 1.5e-4, and a score's error counts twice in a weight: 1e-3 of the largest logit.  What the cache holds is a key or
    value to 2^-12 of its head's largest column (float32, from 32 terms and a rotation), and in 8 bits to half a step (2^-4 of a column) more."""
    from paper_2509_24328_amd import companion_fit as C
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    V, D, B = 300, 32, 3
    m = C.Reader(V, D, gen, B, 70, cache, scale=1.0)
    history = torch.randint(0, V, (B, 70), generator=gen, device="cuda", dtype=torch.int32)
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    keep = [[5, 1, 3], [1, 1, 1], [2, 9, 4], [6, 6, 1], [9, 2, 9], [1, 1, 1]]
    for step, n in enumerate(keep):
        P = max(n) + 2                                     # the two behind are taken back: other tokens than the sequence's
        at = lengths.long()[:, None] + torch.arange(P, device="cuda")
        tokens = history.gather(1, at)
        taken = torch.tensor(n, device="cuda")
        tokens = torch.where(torch.arange(P, device="cuda") < taken[:, None], tokens, (tokens + 7) % V).to(torch.int32)
        z = m.logits(tokens, lengths).double().cpu()
        for b in range(B):
            end = int(lengths[b]) + n[b]
            kv = held(m, b, end)
            want, *own = whole(m, history[b, :end], kv)
            for have, true in zip(kv, own):
                top = true.abs().amax(-1, keepdim=True)
                assert ((have - true).abs() <= 2.0 ** -12 * top + (0 if cache != F8 else 2.0 ** -4 * true.abs())).all(), (step, b)
            assert (z[b, :n[b]] - want[-n[b]:]).abs().max() <= 1e-3 * want.abs().max(), (step, b)
        lengths += taken.to(torch.int32)


@pytest.mark.parametrize("cache", [torch.float32, F8], ids=str)
def test_the_command_runs(cache):
    from paper_2509_24328_amd import companion_fit as C
    log = C.run(V=256, D=32, B=16, k=4, steps=30, seed=2, attention=cache, max_tokens=48)
    assert len(log) == 30 and all(abs(v) < 1e6 for r in log for v in r.values())
    assert all(0 <= r["accepted"] <= 4 and 0 <= r["similarity"] <= 1 + 1e-6 for r in log)
    assert sum(r["accepted"] for r in log) > 0
    again = C.run(V=256, D=32, B=16, k=4, steps=30, seed=2, attention=cache, max_tokens=48)
    assert [r["target"] for r in again] == [r["target"] for r in log]


def test_a_noisy_copy_has_a_cache_of_its_own():
    from paper_2509_24328_amd import companion_fit as C
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    m = C.Reader(50, 16, gen, 2, 20)
    n = m.noisy(0.0, gen)
    assert isinstance(n, C.Reader) and n.cache.k.data_ptr() != m.cache.k.data_ptr() and n.cache.k.shape == m.cache.k.shape
