"""The timed cases of the operators on the model side of a decode step: what a draft does to draw a token, and
what a target does to look at the drafted ones.

  rope        rotary positions of queries or keys, and of their gradients (the inverse rotation)
  cache       keys and values of a step's new tokens, rotated, into the pages of a cache (and its queries rotated
              beside them), and rows of the cache back into dense tensors
  attend      attention of the new tokens of every sequence over its pages
  sample      a token of every row under temperature, top-k, top-p and min-p, from given random numbers

Fields of a case (those that its form uses):
  form      one of the above
  dtype     storage type of queries, keys, values, outputs or logits, "bf16" or "f32"
  n, H, D   rope: tokens, heads, columns of a head;  rot: leading columns of a head that are rotated
  layout    "half": column j turns with column j + rot / 2, "pairs": column 2 j with column 2 j + 1
  scaling   frequencies for contexts longer than those trained on: "plain", "linear", "ntk" or "parts"
  inverse   rope: the gradient's direction
  B, P      sequences, largest number of new tokens of one
  ragged    sequences have 1 to P new tokens and contexts of a quarter to the whole of ctx
  Hq, Hkv   heads of the queries, heads of the cache
  ctx       tokens of the longest sequence that are in the cache before the new ones
  page      tokens a page
  cache     storage type of the cache: "bf16", "f32" or "f8" (e4m3 with a float32 scale for each token and head)
  window    attend: tokens that a query sees at most (0: all before it, and itself)
  padded    attend: every third sequence begins behind its first new token, which sees nothing then
  back      cache: whole sequences are read back, not the new rows alone
  V         sample: vocabulary;  T, top_k, top_p, min_p: warps
"""
import math

import torch

own = False          # whether run() calls the package or computes the plain form

SCRATCH = 256 << 20  # device scratch that a program keeps for the calls that take some
_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32, "f8": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "f32": 4, "f8": 1}
F8_MAX = 448.0       # largest e4m3 number
SCALING = {"plain": 0, "linear": 1, "ntk": 2, "parts": 3}
LAYOUT = {"half": 0, "pairs": 1}
BASE, FACTOR, LOW, HIGH, TRAINED = 10000.0, 4.0, 1.0, 32.0, 4096


def _rope(name, n, H, D, rot, dtype, layout, scaling, inverse):
    return dict(name=name, form="rope", n=n, H=H, D=D, rot=rot, dtype=dtype, layout=layout, scaling=scaling,
                inverse=inverse)


def _cache(name, B, P, Hq, Hkv, D, rot, ctx, page, dtype, cache, layout, ragged=False, back=False, scaling="plain"):
    return dict(name=name, form="cache", B=B, P=P, Hq=Hq, Hkv=Hkv, D=D, rot=rot, ctx=ctx, page=page, dtype=dtype,
                cache=cache, layout=layout, ragged=ragged, back=back, scaling=scaling)


def _attend(name, B, P, Hq, Hkv, D, ctx, page, dtype, cache, ragged=False, window=0, padded=False):
    return dict(name=name, form="attend", B=B, P=P, Hq=Hq, Hkv=Hkv, D=D, ctx=ctx, page=page, dtype=dtype, cache=cache,
                ragged=ragged, window=window, padded=padded)


def _sample(name, B, V, dtype, T, top_k, top_p, min_p):
    return dict(name=name, form="sample", B=B, V=V, dtype=dtype, T=T, top_k=top_k, top_p=top_p, min_p=min_p)


def listed():
    return [
        # the positions of one sequence's verification, a small model: nothing but latency
        _rope("rope_9_h14_d64_bf16", 9, 14, 64, 64, "bf16", "half", "plain", False),
        # gradient of the queries of a fitting batch, a part of the head rotated, frequencies of a long context
        _rope("rope_grad_16384_h32_d128_bf16", 16384, 32, 128, 64, "bf16", "pairs", "parts", True),
        # one verification step of the headline batch: what it writes, in 8 bits
        _cache("cache_64x9_h32_d128_f8", 64, 9, 32, 8, 128, 128, 8192, 64, "bf16", "f8", "half", ragged=True),
        # a prompt's keys and values in float32, pages of an odd size, and the sequence handed on as dense tensors
        _cache("cache_prompt_4096_d80_f32", 1, 4096, 8, 8, 80, 40, 1000, 20, "f32", "f32", "pairs", back=True, scaling="linear"),
        # one user's draft, one token: latency
        _attend("attend_1x1_ctx1500_bf16", 1, 1, 14, 2, 64, 1500, 16, "bf16", "bf16"),
        # a small float32 model, head width and pages of odd sizes, rows that see nothing, a sliding window
        _attend("attend_5x7_d80_f32", 5, 7, 12, 4, 80, 900, 20, "f32", "f32", ragged=True, window=512, padded=True),
        # the verification of the headline batch over an 8-bit cache, lengths as verification chose them
        _attend("attend_64x9_ctx8192_f8", 64, 9, 32, 8, 128, 8192, 64, "bf16", "f8", ragged=True),
        # plain decoding of a batch over long contexts
        _attend("attend_64x1_ctx16384_bf16", 64, 1, 32, 8, 128, 16384, 128, "bf16", "bf16"),
        # a chunk of a long prompt: the matrix product counts
        _attend("attend_1x2048_ctx6144_bf16", 1, 2048, 32, 8, 128, 6144, 64, "bf16", "bf16"),
        # one user's draft draws from the whole distribution: latency
        _sample("sample_1_v32000_f32", 1, 32000, "f32", 1.0, 0, 1.0, 0.0),
        # a drafting step of the headline batch with the warps of the model series
        _sample("sample_64_v152064_bf16", 64, 152064, "bf16", 0.7, 20, 0.8, 0.0),
        # a large batch, nucleus and floor without a K
        _sample("sample_512_v128256_bf16", 512, 128256, "bf16", 1.0, 0, 0.95, 0.02),
    ]


def draw(rng):
    """One more case: sizes over the ranges that the listed ones span, odd ones among them."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    form = rng.choice(("rope", "cache", "attend", "attend", "sample", "sample"))
    while True:
        dtype = rng.choice(("bf16", "bf16", "f32"))
        D = rng.choice((64, 64, 72, 80, 96, 128, 128, 128, 192, 256))
        rot = rng.choice((D, D, D // 2, 2 * (D // 5)))
        layout, scaling = rng.choice(("half", "pairs")), rng.choice(("plain", "linear", "ntk", "parts"))
        Hkv = rng.choice((1, 2, 4, 8, 8))
        Hq = Hkv * rng.choice((1, 2, 4, 4, 7, 8))
        page = rng.choice((16, 16, 32, 64, 64, 128, 20, 7))
        cache = rng.choice((dtype, "f8"))
        ragged = rng.random() < 0.5
        if form == "rope":
            c = dict(form=form, n=log(1, 16384), H=rng.choice((1, 4, 14, 32)), D=D, rot=rot, dtype=dtype, layout=layout,
                     scaling=scaling, inverse=rng.random() < 0.4)
        elif form == "cache":
            B = log(1, 64)
            c = dict(form=form, B=B, P=log(1, 4096 / B), Hq=Hq, Hkv=Hkv, D=D, rot=rot, ctx=log(1, 8192), page=page,
                     dtype=dtype, cache=cache, layout=layout, ragged=ragged, back=rng.random() < 0.3, scaling=scaling)
        elif form == "attend":
            B = log(1, 64)
            P = rng.choice((1, rng.randrange(2, 18), rng.randrange(2, 18), log(18, 2048)))
            c = dict(form=form, B=B, P=P, Hq=Hq, Hkv=Hkv, D=D, ctx=log(16, 16384), page=page, dtype=dtype, cache=cache,
                     ragged=ragged, window=rng.choice((0, 0, 0, log(16, 4096))), padded=rng.random() < 0.25)
        else:
            V = log(4096, 152064)
            c = dict(form=form, B=log(1, 512), V=V if rng.random() < 0.5 else max(64, V - V % 64), dtype=dtype,
                     T=rng.choice((1.0, 0.7, 1.3)), top_k=rng.choice((0, 0, 1, 20, 50, 1000)),
                     top_p=rng.choice((1.0, 0.8, 0.95)), min_p=rng.choice((0.0, 0.0, 0.02, 0.1)))
        w = work(c)
        if form == "attend":
            # (a plain form holds all scores, and keys and values in 32 bits)
            L = c["ctx"] + c["P"]
            if w["bytes"] > 4.3e9 or w["flops"] > 2.4e11 or 4.0 * c["B"] * L * (c["Hq"] * c["P"] + 2 * c["Hkv"] * D) > 9e9:
                continue
        if form == "cache" and w["bytes"] > 3e8:
            continue
        return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _counts(case):
    """New tokens of every sequence, in some order."""
    return [1 + (5 * b) % case["P"] if case["ragged"] else case["P"] for b in range(case["B"])]


def _contexts(case):
    """Tokens that are in the cache before, of every sequence, in some order."""
    B, ctx = case["B"], case["ctx"]
    return [ctx - (3 * ctx * ((7 * b) % B)) // (4 * B) if case["ragged"] else ctx for b in range(B)]


def _first(case, lengths):
    """First token of every sequence that may be seen."""
    return [n + 1 if case["padded"] and b % 3 == 2 else 0 for b, n in enumerate(lengths)]


def _frequencies(case):
    """Angle per position of every pair of columns, float64."""
    rot = case["rot"]
    j = torch.arange(0, rot, 2, dtype=torch.float64, device="cuda")
    base = BASE
    if case["scaling"] == "ntk" and rot > 2:
        base = BASE * FACTOR ** (rot / (rot - 2.0))
    f = torch.exp(-(j / rot) * math.log(base))
    if case["scaling"] == "linear":
        f = f / FACTOR
    elif case["scaling"] == "parts":
        turns = TRAINED * f / (2.0 * math.pi)
        keep = ((turns - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        f = f / FACTOR * (1.0 - keep) + f * keep
    return f


def _quantised(x):
    """e4m3 numbers and the scale of every row, from float32."""
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.where(top > 0, top / F8_MAX, torch.ones_like(top))
    return (x / scale).to(torch.float8_e4m3fn), scale[..., 0]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(2000 + seed)
    form, dev = case["form"], "cuda"
    dtype = _TYPE[case["dtype"]]
    randn = lambda *s: torch.randn(s, generator=g, device=dev)
    f32 = lambda *s: torch.zeros(s, dtype=torch.float32, device=dev)
    st = dict(case=case)
    if form == "sample":
        B, V = case["B"], case["V"]
        # a model's logits: a broad middle, one entry in a hundred well above it
        z = randn(B, V) * 2.5 + 8.0 * (torch.rand((B, V), generator=g, device=dev) < 0.01)
        st.update(z=z.to(dtype), u=torch.rand(B, generator=g, device=dev, dtype=torch.float64),
                  token=torch.zeros(B, dtype=torch.int32, device=dev), logprob=f32(B))
        return st
    H, D = case.get("H", case.get("Hq")), case["D"]
    if form == "rope":
        n = case["n"]
        # tokens at far positions; the queries are columns of one product with keys and values, as a layer makes them
        wide = randn(n, H + 2, D).to(dtype)
        st.update(x=wide[:, :H], positions=torch.randint(0, 131072, (n,), generator=g, device=dev, dtype=torch.int32),
                  freq=_frequencies(case), out=torch.zeros((n, H, D), dtype=dtype, device=dev))
        return st
    B, P, Hkv, page = case["B"], case["P"], case["Hkv"], case["page"]
    order = torch.randperm(B, generator=g, device=dev).tolist()
    counts, lengths = _counts(case), _contexts(case)
    counts, lengths = [counts[b] for b in order], [lengths[b] for b in order]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    total = sum(counts)
    st["lengths"], st["t_offsets"] = i32(lengths), i32([sum(counts[:b]) for b in range(B + 1)])
    n_rows = total + (-total) % 8                     # (rows behind the last sequence: a captured step's largest size)
    # every sequence's pages lie anywhere; the table has a place for one page more than the longest needs
    need = [-(-(n + c) // page) for n, c in zip(lengths, counts)]
    n_pages, max_pages = sum(need) + 1, max(need) + 1
    shuffled = torch.randperm(n_pages, generator=g, device=dev).tolist()
    table = []
    for m in need:
        table.append(shuffled[:m] + [-1] * (max_pages - m))
        shuffled = shuffled[m:]
    st["pages"] = i32(table)
    kind = _TYPE[case["cache"]]
    shape = (n_pages, Hkv, page, D)
    if form == "cache":
        st["k_cache"], st["v_cache"] = (torch.zeros(shape, dtype=torch.uint8, device=dev).view(kind) if case["cache"] == "f8"
                                        else torch.zeros(shape, dtype=kind, device=dev) for _ in range(2))
        st["k_scale"], st["v_scale"] = (f32(*shape[:3]) if case["cache"] == "f8" else None for _ in range(2))
        wide = randn(n_rows, H + 2 * Hkv, D).to(dtype)
        st.update(q=wide[:, :H], k=wide[:, H:H + Hkv], v=wide[:, H + Hkv:], freq=_frequencies(case),
                  q_out=torch.zeros((n_rows, H, D), dtype=dtype, device=dev))
        # what is read back: the new rows, or whole sequences from their first token on
        many = [n + c for n, c in zip(lengths, counts)] if case["back"] else counts
        st["from"] = torch.zeros_like(st["lengths"]) if case["back"] else st["lengths"]
        st["back_offsets"] = i32([sum(many[:b]) for b in range(B + 1)])
        st["back_P"] = max(many)
        st["k_back"], st["v_back"] = (torch.zeros((sum(many), Hkv, D), dtype=dtype, device=dev) for _ in range(2))
        return st
    k, v = randn(*shape), randn(*shape)
    if case["cache"] == "f8":
        st["k_cache"], st["k_scale"] = _quantised(k)
        st["v_cache"], st["v_scale"] = _quantised(v)
    else:
        st.update(k_cache=k.to(kind), v_cache=v.to(kind), k_scale=None, v_scale=None)
    del k, v
    st["first"] = i32(_first(case, lengths)) if case["padded"] else None
    # (queries some times as long as keys: a trained model's weights of the keys are far from equal)
    st.update(q=(randn(n_rows, H, D) * 2.0).to(dtype), out=torch.zeros((n_rows, H, D), dtype=dtype, device=dev),
              lse=f32(n_rows, H), scale=1.0 / math.sqrt(D), scratch=torch.empty(SCRATCH, dtype=torch.uint8, device=dev))
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _plain_rotated(x, positions, freq, rot, layout, inverse):
    """float32 [n, H, D]; angles and products in 64 bits."""
    angle = positions.double()[:, None, None] * freq
    c, s = torch.cos(angle), torch.sin(angle)
    if inverse:
        s = -s
    t = x[..., :rot].double()
    if layout == "half":
        a, b = t[..., :rot // 2], t[..., rot // 2:]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = t[..., 0::2], t[..., 1::2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([turned.float(), x[..., rot:].float()], -1)


def _plain_rope(st):
    c = st["case"]
    y = _plain_rotated(st["x"], st["positions"], st["freq"], c["rot"], c["layout"], c["inverse"])
    return y.to(st["x"].dtype)


def _places(offsets, start, pages, page, n_rows):
    """(whether a row is a sequence's, position, physical page, place in the page) of every row."""
    row = torch.arange(n_rows, device="cuda")
    b = (row[:, None] >= offsets[1:][None, :]).sum(-1)
    there = b < offsets.numel() - 1
    b = b.clamp(max=offsets.numel() - 2)
    position = start.long()[b] + row - offsets.long()[b]
    return there, position, pages.long()[b, torch.where(there, position, torch.zeros_like(position)) // page], position % page


def _plain_cache(st):
    c = st["case"]
    n_rows = st["q"].shape[0]
    there, position, pg, sl = _places(st["t_offsets"], st["lengths"], st["pages"], c["page"], n_rows)
    turn = lambda x: _plain_rotated(x, position, st["freq"], c["rot"], c["layout"], False)
    q = torch.where(there[:, None, None], turn(st["q"]).to(st["q"].dtype), torch.zeros_like(st["q_out"]))
    pg, sl = pg[there], sl[there]
    k, v = turn(st["k"])[there], st["v"].float()[there]
    if c["cache"] == "f8":
        k, st["k_scale"][pg, :, sl] = _quantised(k)
        v, st["v_scale"][pg, :, sl] = _quantised(v)
        st["k_cache"].view(torch.uint8)[pg, :, sl] = k.view(torch.uint8)
        st["v_cache"].view(torch.uint8)[pg, :, sl] = v.view(torch.uint8)
    else:
        st["k_cache"][pg, :, sl] = k.to(st["k_cache"].dtype)
        st["v_cache"][pg, :, sl] = v.to(st["v_cache"].dtype)
    _, _, pg, sl = _places(st["back_offsets"], st["from"], st["pages"], c["page"], st["k_back"].shape[0])

    def back(cache, scale):
        if scale is None:
            return cache[pg, :, sl].to(st["q"].dtype)
        codes = cache.view(torch.uint8)[pg, :, sl].view(torch.float8_e4m3fn)
        return (codes.float() * scale[pg, :, sl][..., None]).to(st["q"].dtype)

    return {"q": q, "k": back(st["k_cache"], st["k_scale"]), "v": back(st["v_cache"], st["v_scale"])}


def _plain_attend(st):
    c = st["case"]
    B, P, Hq, Hkv, D, page = (c[n] for n in ("B", "P", "Hq", "Hkv", "D", "page"))
    G = Hq // Hkv
    n_rows = st["q"].shape[0]
    offsets, lengths = st["t_offsets"].long(), st["lengths"].long()
    L = c["ctx"] + P
    pages = st["pages"][:, :-(-L // page)].long().clamp(min=0)

    def dense(cache, scale):                          # [B, Hkv, tokens, D]
        x = cache.view(torch.uint8)[pages].view(cache.dtype).float() if scale is not None else cache[pages].float()
        if scale is not None:
            x = x * scale[pages][..., None]
        return x.transpose(1, 2).reshape(B, Hkv, -1, D)[:, :, :L]

    k, v = dense(st["k_cache"], st["k_scale"]), dense(st["v_cache"], st["v_scale"])
    i = torch.arange(P, device="cuda")
    at = (offsets[:-1, None] + i).clamp(max=n_rows - 1)
    q = st["q"][at].float().reshape(B, P, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * P, D)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(st["scale"])
    s = s.view(B, Hkv, G, P, L)
    position = (lengths[:, None] + i)[:, :, None]
    key = torch.arange(L, device="cuda")
    seen = key <= position
    if c["window"]:
        seen = seen & (key > position - c["window"])
    if st["first"] is not None:
        seen = seen & (key >= st["first"][:, None, None])
    s.masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    base = top.clamp(min=-1e30)
    e = s.sub_(base).exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(B, Hkv, G * P, L), v).view(B, Hkv, G, P, D) / total.clamp(min=1e-30)
    o = torch.where(total > 0, o, torch.zeros_like(o))
    lse = (base + torch.log(total))[..., 0]
    here = i < (offsets[1:] - offsets[:-1])[:, None]
    out, out_lse = torch.zeros_like(st["out"]), torch.zeros_like(st["lse"])
    out[at[here]] = o.permute(0, 3, 1, 2, 4).reshape(B, P, Hq, D)[here].to(out.dtype)
    out_lse[at[here]] = lse.permute(0, 3, 1, 2).reshape(B, P, Hq)[here]
    return {"out": out, "lse": out_lse}


def _f32(x):
    """A number as a call in single precision gets it."""
    return torch.tensor(x, dtype=torch.float32).double().item()


def _plain_sample(st):
    c = st["case"]
    B, V = c["B"], c["V"]
    z = st["z"].double()
    y = (z - z.amax(-1, keepdim=True)) / _f32(c["T"])
    w = torch.exp(y)
    if 0 < c["top_k"] < V:
        kth = z.topk(c["top_k"], -1).values[:, -1:]
        w = w * (z >= kth)
    if c["top_p"] < 1.0:
        s = z.sort(-1, descending=True)
        ws = w.gather(-1, s.indices)
        before = ws.cumsum(-1) - ws
        start = torch.ones_like(s.values, dtype=torch.bool)
        start[:, 1:] = s.values[:, 1:] != s.values[:, :-1]
        before = torch.where(start, before, torch.zeros_like(before)).cummax(-1).values   # mass above a group of equal values
        kept = (before < _f32(c["top_p"]) * w.sum(-1, keepdim=True)) & (ws > 0)
        lowest = torch.where(kept, s.values, torch.full_like(s.values, math.inf)).amin(-1, keepdim=True)
        w = w * (z >= lowest)
    if c["min_p"] > 0.0:
        w = w * (w >= _f32(c["min_p"]))
    run_sum = w.cumsum(-1)
    total = run_sum[:, -1:]
    number = torch.arange(V, device="cuda")
    last = torch.where(w > 0, number, torch.zeros_like(number)).amax(-1)
    token = torch.minimum((run_sum <= st["u"][:, None] * total).sum(-1), last)
    logprob = y.gather(-1, token[:, None])[:, 0] - torch.log(total[:, 0])
    return {"token": token.to(torch.int32), "logprob": logprob.float()}


# ---------------------------------------------------------------------------
# the package's calls
# ---------------------------------------------------------------------------
def _own_rope(st):
    import paper_2509_24328_amd as sv
    c = st["case"]
    sv.sv_rope(st["x"], st["positions"], st["freq"], st["out"], layout=LAYOUT[c["layout"]], inverse=c["inverse"])
    return st["out"]


def _handle(st):
    import paper_2509_24328_amd as sv
    if "handle" not in st:
        st["handle"] = sv.Cache(st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"])
    return st["handle"]


def _own_cache(st):
    import paper_2509_24328_amd as sv
    c, cache = st["case"], _handle(st)
    sv.sv_cache_write(cache, st["k"], st["v"], st["lengths"], st["pages"], t_offsets=st["t_offsets"], P=c["P"], q=st["q"],
                      q_out=st["q_out"], freq=st["freq"], layout=LAYOUT[c["layout"]])
    sv.sv_cache_read(cache, st["k_back"], st["v_back"], st["from"], st["pages"], t_offsets=st["back_offsets"],
                     P=st["back_P"])
    return {"q": st["q_out"], "k": st["k_back"], "v": st["v_back"]}


def _own_attend(st):
    import paper_2509_24328_amd as sv
    c = st["case"]
    sv.sv_chunk_attention(_handle(st), st["q"], st["out"], st["lengths"], st["pages"], t_offsets=st["t_offsets"], P=c["P"],
                          scale=st["scale"], window=c["window"], first=st["first"], lse=st["lse"], ws=st["scratch"])
    return {"out": st["out"], "lse": st["lse"]}


def _own_sample(st):
    import paper_2509_24328_amd as sv
    c = st["case"]
    sv.sv_sample(st["z"], st["u"], st["token"], st["logprob"], temperature=c["T"], top_k=c["top_k"], top_p=c["top_p"],
                 min_p=c["min_p"])
    return {"token": st["token"], "logprob": st["logprob"]}


_PLAIN = {"rope": _plain_rope, "cache": _plain_cache, "attend": _plain_attend, "sample": _plain_sample}
_OWN = {"rope": _own_rope, "cache": _own_cache, "attend": _own_attend, "sample": _own_sample}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["form"]](state)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_turned(x, positions, case, freq):
    """Rotation as a product of complex numbers."""
    rot, half = case["rot"], case["rot"] // 2
    x = x.double()
    t = x[..., :rot]
    pairs = torch.stack([t[..., :half], t[..., half:]], -1) if case["layout"] == "half" else t.reshape(*t.shape[:-1], half, 2)
    angle = positions.double()[:, None] * freq * (-1.0 if case.get("inverse") else 1.0)
    turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), angle)[:, None])
    turned = torch.cat([turned[..., 0], turned[..., 1]], -1) if case["layout"] == "half" else turned.reshape(t.shape)
    return torch.cat([turned, x[..., rot:]], -1)


def _exact_stored(x, case):
    """What the cache holds of rows, in 64 bits."""
    x = x.float()
    if case["cache"] != "f8":
        return x.to(_TYPE[case["cache"]]).double()
    top = x.abs().amax(-1, keepdim=True)
    scale = (top.double() / F8_MAX).float().double()
    scale = torch.where(top > 0, scale, torch.ones_like(scale))
    r = x.double() / scale
    # e4m3: three bits behind the leading one, steps of 2^-9 below 2^-6
    step = torch.exp2(torch.floor(torch.log2(r.abs().clamp(min=2.0 ** -6))) - 3.0)
    return (torch.round(r / step) * step).clamp(-F8_MAX, F8_MAX) * scale


def exact(case, seed):
    st = prepare(case, seed)
    form = case["form"]
    if form == "rope":
        return _exact_turned(st["x"], st["positions"], case, st["freq"])
    if form == "sample":
        out = {"token": None, "logprob": torch.empty(case["B"], dtype=torch.float64, device="cuda")}
        token = torch.empty(case["B"], dtype=torch.int32, device="cuda")
        for r in range(case["B"]):
            x = st["z"][r].double()
            order = x.sort(descending=True).indices
            p = torch.softmax(x / _f32(case["T"]), 0)
            if 0 < case["top_k"] < case["V"]:
                p = torch.where(x >= x[order[case["top_k"] - 1]], p, torch.zeros_like(p))
                p = p / p.sum()
            if case["top_p"] < 1.0:
                reach = torch.searchsorted(p[order].cumsum(0), torch.tensor(_f32(case["top_p"]), device="cuda", dtype=torch.float64))
                p = torch.where(x >= x[order[reach.clamp(max=case["V"] - 1)]], p, torch.zeros_like(p))
            p = torch.where(p >= _f32(case["min_p"]) * p[order[0]], p, torch.zeros_like(p))
            p = p / p.sum()
            t = torch.searchsorted(p.cumsum(0), st["u"][r], right=True).clamp(max=case["V"] - 1)
            token[r] = t
            out["logprob"][r] = torch.log(p[t])
        out["token"] = token
        return out
    counts = (st["t_offsets"][1:] - st["t_offsets"][:-1]).tolist()
    lengths, page, Hkv, D = st["lengths"].tolist(), case["page"], case["Hkv"], case["D"]
    if form == "cache":
        q = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        k, v = (torch.zeros(st["k_back"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
        row = at = 0
        for n, c in zip(lengths, counts):
            position = torch.arange(n, n + c, device="cuda")
            q[row:row + c] = _exact_turned(st["q"][row:row + c], position, case, st["freq"])
            at += n if case["back"] else 0               # (what was in the cache before is zeros)
            k[at:at + c] = _exact_stored(_exact_turned(st["k"][row:row + c], position, case, st["freq"]), case)
            v[at:at + c] = _exact_stored(st["v"][row:row + c].double(), case)
            row, at = row + c, at + c
        return {"q": q, "k": k, "v": v}
    G = case["Hq"] // Hkv
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device="cuda")
    first = st["first"].tolist() if st["first"] is not None else [0] * case["B"]
    row = 0
    for b, (n, c) in enumerate(zip(lengths, counts)):
        L = n + c
        held = st["pages"][b, :-(-L // page)].long()
        position = torch.arange(n, L, device="cuda")[:, None]
        key = torch.arange(L, device="cuda")
        hidden = (key > position) | (key < first[b])
        if case["window"]:
            hidden |= key <= position - case["window"]
        for h in range(Hkv):
            def rows(cache, scale):
                x = (cache.view(torch.uint8)[held, h].view(cache.dtype) if scale is not None else cache[held, h]).double()
                x = x * scale[held, h].double()[..., None] if scale is not None else x
                return x.reshape(-1, D)[:L]
            k, v = rows(st["k_cache"], st["k_scale"]), rows(st["v_cache"], st["v_scale"])
            for j in range(h * G, (h + 1) * G):
                s = (st["q"][row:row + c, j].double() @ k.t().contiguous()) * st["scale"]
                s = s.masked_fill(hidden, -math.inf)
                norm = torch.logsumexp(s, -1)
                p = torch.exp(s - norm.clamp(min=-1e300)[:, None])
                out[row:row + c, j] = p @ v
                lse[row:row + c, j] = norm
        row += c
    return {"out": out, "lse": lse}


def work(case):
    """Every needed input read once, every output written once."""
    form, e = case["form"], _BYTES[case["dtype"]]
    if form == "sample":
        B, V = case["B"], case["V"]
        # per entry: the exponent, an exponential, a sum, a comparison
        return {"bytes": float(B) * V * e + 16.0 * B, "flops": 5.0 * B * V}
    if form == "rope":
        n, H, D = case["n"], case["H"], case["D"]
        return {"bytes": 2.0 * n * H * D * e + 4.0 * n + 4.0 * case["rot"], "flops": 3.0 * n * H * case["rot"]}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    held = D * _BYTES[case["cache"]] + (4 if case["cache"] == "f8" else 0)      # a row of the cache
    counts, lengths = _counts(case), _contexts(case)
    total = sum(counts)
    if form == "cache":
        back = total + (sum(lengths) if case["back"] else 0)
        return {"bytes": float(total) * ((2 * Hq + 2 * Hkv) * D * e + 2 * Hkv * held) + float(back) * 2 * Hkv * (held + D * e),
                "flops": 3.0 * total * (Hq + Hkv) * case["rot"]}
    first = _first(case, lengths)
    pairs = keys = 0
    for n, c, f in zip(lengths, counts, first):
        lowest = n + c
        for p in range(n, n + c):
            lo = max(f, p - case["window"] + 1 if case["window"] else 0)
            if lo <= p:
                pairs, lowest = pairs + p - lo + 1, min(lowest, lo)
        keys += n + c - lowest
    return {"bytes": 2.0 * keys * Hkv * held + 2.0 * total * Hq * D * e + 4.0 * total * Hq, "flops": 4.0 * pairs * Hq * D}
