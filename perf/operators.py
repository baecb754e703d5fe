"""The timed cases of the operators at the two ends of a draft or companion model that have the
vocabulary's size, and of the step between them.

  score       log-probabilities of given tokens, with the row's normaliser, entropy, the token's rank
              and the most probable alternatives (the emitted tokens of a verification step; a prompt)
  score_grad  the same log-probabilities and entropies, with the gradient of a weighted sum of them
              (fitting a draft or a companion to a target's answers)
  embed       embedding rows of tokens, scaled
  embed_grad  gradient of the embedding table from the gradients of its looked-up rows
  clip        2-norm over the gradients of all parameters, and the gradients scaled to a largest norm

Fields of a case (those that its form uses):
  form      one of the above
  B, P, V   sequences, positions per sequence, vocabulary; score_grad: B rows
  dtype     storage type of logits, table or gradients, "bf16" or "f32"
  emitted   score: only the leading 1 to P positions of a sequence hold a token, as verification leaves them
  packed    score: those positions' logit rows lie one after the other, addressed by offsets
  pad       score, score_grad: columns of a row beyond the vocabulary (a model's output padded to a multiple)
  masked    score, score_grad: every fourth row has all but a few tokens at -inf (constrained decoding)
  T, top    temperature; number of alternatives
  entropy   score_grad: the sum has an entropy term
  n, D      embed, embed_grad: tokens, columns of the table
  out       embed_grad, clip: storage type of the result
  layers, d clip: layers and width of the model whose gradients they are
  clips     clip: whether the norm is above the largest one allowed
"""
import math

import torch

own = False          # whether run() calls the package or computes the plain form

SCRATCH = 128 << 20  # device scratch that a program keeps for the calls that take some
PAD = -1             # "no token here"
_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


def _score(name, B, P, V, dtype, top, T=1.0, emitted=False, packed=False, pad=0, masked=False):
    return dict(name=name, form="score", B=B, P=P, V=V, dtype=dtype, top=top, T=T, emitted=emitted, packed=packed,
                pad=pad, masked=masked)


def _score_grad(name, B, V, dtype, entropy, T=1.0, pad=0, masked=False):
    return dict(name=name, form="score_grad", B=B, V=V, dtype=dtype, entropy=entropy, T=T, pad=pad, masked=masked)


def _embed(name, n, V, D, dtype):
    return dict(name=name, form="embed", n=n, V=V, D=D, dtype=dtype)


def _embed_grad(name, n, V, D, dtype, out):
    return dict(name=name, form="embed_grad", n=n, V=V, D=D, dtype=dtype, out=out)


def _clip(name, layers, d, V, dtype, out, clips):
    return dict(name=name, form="clip", layers=layers, d=d, V=V, dtype=dtype, out=out, clips=clips)


def listed():
    return [
        # one user's next token with five alternatives beside it: nothing but latency
        _score("score_1x1_v32000_f32", 1, 1, 32000, "f32", 5),
        # what a step of the headline batch has emitted, with the most alternatives an answer shows
        _score("score_64x9_v152064_bf16", 64, 9, 152064, "bf16", 20, emitted=True),
        # selected prefixes only, packed; a vocabulary extended by one token, rows padded; constrained decoding
        _score("score_packed_24x6_v32001_bf16", 24, 6, 32001, "bf16", 5, T=0.75, emitted=True, packed=True, pad=63,
               masked=True),
        # a prompt's log-probabilities, each with the most probable token
        _score("score_prompt_4096_v128256_bf16", 1, 4096, 128256, "bf16", 1),
        # a batch of a draft's fitting step, with an entropy term: the largest
        _score_grad("score_grad_2048_v152064_bf16", 2048, 152064, "bf16", True),
        # a small batch of float32 logits, rows on odd elements
        _score_grad("score_grad_96_v32001_f32", 96, 32001, "f32", False),
        # the positions of one decode step
        _embed("embed_9_v152064_d2048_bf16", 9, 152064, 2048, "bf16"),
        # a batch of prompts
        _embed("embed_16384_v128256_d4096_bf16", 16384, 128256, 4096, "bf16"),
        # a small fitting batch: most rows of the gradient are zeros
        _embed_grad("embed_grad_512_v32001_d896_f32", 512, 32001, 896, "f32", "f32"),
        # a large one, whose frequent tokens occur thousands of times
        _embed_grad("embed_grad_65536_v32000_d2048_bf16", 65536, 32000, 2048, "bf16", "bf16"),
        # a small draft: few tensors, float32
        _clip("clip_2x256_v32000_f32", 2, 256, 32000, "f32", "f32", True),
        # a draft of 1.3 billion parameters in 170 tensors
        _clip("clip_24x2048_v128256_bf16", 24, 2048, 128256, "bf16", "bf16", True),
    ]


def draw(rng):
    """One more case: sizes over the ranges that the listed ones span, odd ones among them."""
    def log(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return v + 1 if v == 3072 else v

    def vocabulary():
        V = log(4096, 152064)
        return V if rng.random() < 0.5 else max(64, V - V % 64)

    form = rng.choice(("score", "score", "score_grad", "embed", "embed_grad", "clip"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    while True:
        V = vocabulary()
        if form == "score":
            emitted = rng.random() < 0.6
            c = dict(form=form, B=log(1, 64) if emitted else 1, P=rng.randrange(2, 18) if emitted else log(1, 4096),
                     V=V, dtype=dtype, top=rng.choice((0, 1, 5, 20, 32)), T=rng.choice((1.0, 1.0, 0.75)),
                     emitted=emitted, packed=emitted and rng.random() < 0.5, pad=rng.choice((0, 0, rng.randrange(1, 64))),
                     masked=rng.random() < 0.25)
        elif form == "score_grad":
            c = dict(form=form, B=log(1, 2048), V=V, dtype=dtype, entropy=rng.random() < 0.5,
                     T=rng.choice((1.0, 1.0, 0.75)), pad=rng.choice((0, 0, rng.randrange(1, 64))),
                     masked=rng.random() < 0.25)
        elif form == "embed":
            c = dict(form=form, n=log(1, 16384), V=V, D=log(64, 4096), dtype=dtype)
        elif form == "embed_grad":
            c = dict(form=form, n=log(1, 65536), V=V, D=log(64, 2048), dtype=dtype, out=rng.choice((dtype, "f32")))
        else:
            c = dict(form=form, layers=rng.randrange(1, 25), d=8 * log(16, 256), V=V, dtype=dtype,
                     out=rng.choice((dtype, dtype, "f32")), clips=rng.random() < 0.8)
            c["d"] += 8 if c["d"] == 3072 else 0
        if work(c)["bytes"] <= (5.5e9 if form == "clip" else 1.3e9):
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _rows(case):
    """Positions of a score case that hold a token."""
    B, P = case["B"], case["P"]
    return sum(1 + (5 * b) % P for b in range(B)) if case["emitted"] else B * P


def _logits(rows, case, g):
    """A model's logits: a broad middle, one entry in a hundred well above it."""
    V, dev = case["V"], "cuda"
    z = torch.randn((rows, V), generator=g, device=dev) * 2.5
    z += 8.0 * (torch.rand((rows, V), generator=g, device=dev) < 0.01)
    if case["masked"]:
        allowed = torch.rand((rows, V), generator=g, device=dev) < 12.0 / V
        allowed[:, torch.randint(0, V, (1,), generator=g, device=dev)] = True
        allowed[torch.arange(rows, device=dev) % 4 != 0] = True
        z.masked_fill_(~allowed, float("-inf"))
    wide = torch.zeros((rows, V + case["pad"]), dtype=_TYPE[case["dtype"]], device=dev)
    wide[:, :V] = z
    # a token of the distribution itself
    u = torch.rand((rows, V), generator=g, device=dev).clamp_(1e-20, 1 - 1e-7)
    return wide, (z - torch.log(-torch.log(u))).argmax(-1).to(torch.int32)


def _tokens(n, V, g):
    """Tokens of a text: the frequency falls with the token's number; one in fifty is padding."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    t = (torch.exp(u * math.log(V + 1)) - 1).long().clamp_(0, V - 1).to(torch.int32)
    t[torch.rand(n, generator=g, device="cuda") < 0.02] = PAD
    return t


def _shapes(case):
    """Parameters of a model: tied embedding, per layer two norms and four products, a last norm."""
    d, f, kv = case["d"], 8 * (case["d"] * 11 // 32), max(8, case["d"] // 4)
    layer = [(d,), (d + 2 * kv, d), (d, d), (d,), (2 * f, d), (d, f)]
    return [(case["V"], d)] + layer * case["layers"] + [(d,)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 + seed)
    form, dev = case["form"], "cuda"
    st = dict(case=case, scratch=torch.empty(SCRATCH, dtype=torch.uint8, device=dev))
    f32 = lambda *s: torch.empty(s, dtype=torch.float32, device=dev)
    i32 = lambda *s: torch.empty(s, dtype=torch.int32, device=dev)
    if form == "score":
        B, P, V, top = case["B"], case["P"], case["V"], case["top"]
        count = torch.full((B,), P, device=dev)
        if case["emitted"]:
            count = (1 + (5 * torch.arange(B, device=dev)) % P)[torch.randperm(B, generator=g, device=dev)]
        here = torch.arange(P, device=dev)[None, :] < count[:, None]
        packed = case["packed"]
        wide, tok = _logits(_rows(case) if packed else B * P, case, g)
        st["tokens"] = torch.full((B, P), PAD, dtype=torch.int32, device=dev)
        st["tokens"][here] = tok if packed else tok.view(B, P)[here]
        st["offsets"] = torch.cat([count.new_zeros(1), count.cumsum(0)]).to(torch.int32) if packed else None
        st["z"] = (wide if packed else wide.view(B, P, -1))[..., :V]
        st.update(logprob=f32(B, P), lse=f32(B, P), entropy=f32(B, P), rank=i32(B, P))
        if top:
            st.update(top_token=i32(B, P, top), top_logprob=f32(B, P, top))
    elif form == "score_grad":
        B, V = case["B"], case["V"]
        wide, st["tokens"] = _logits(B, case, g)
        # positions that carry no loss: a tenth of them; weights: advantages of sampled answers
        st["tokens"][torch.arange(B, device=dev) % 10 == 9] = PAD
        st["z"] = wide[:, :V]
        st["g_logprob"] = torch.randn(B, generator=g, device=dev) / B
        st["g_entropy"] = torch.full((B,), 0.01 / B, device=dev) if case["entropy"] else None
        st.update(logprob=f32(B), entropy=f32(B) if case["entropy"] else None,
                  dz=torch.empty((B, V), dtype=_TYPE[case["dtype"]], device=dev))
    elif form in ("embed", "embed_grad"):
        n, V, D, dtype = case["n"], case["V"], case["D"], _TYPE[case["dtype"]]
        st["ids"] = _tokens(n, V, g)
        st["scale"] = math.sqrt(D)
        if form == "embed":
            st["table"] = (torch.randn((V, D), generator=g, device=dev) * 0.02).to(dtype)
            st["out"] = torch.empty((n, D), dtype=dtype, device=dev)
        else:
            st["grad_out"] = (torch.randn((n, D), generator=g, device=dev) * 1e-3).to(dtype)
            st["grad_table"] = torch.empty((V, D), dtype=_TYPE[case["out"]], device=dev)
    else:
        shapes = _shapes(case)
        size = [math.prod(s) for s in shapes]
        # norms' gradients are float32, as their parameters are
        kind = [torch.float32 if len(s) == 1 else _TYPE[case["dtype"]] for s in shapes]
        st["grads"] = [(torch.randn(s, generator=g, device=dev) * 1e-3).to(t) for s, t in zip(shapes, kind)]
        # clipped gradients go into one bucket, which the optimizer (or a reduction over ranks) reads
        st["bucket"] = torch.empty(sum(size), dtype=_TYPE[case["out"]], device=dev)
        st["clipped"] = [b.view(s) for b, s in zip(st["bucket"].split(size), shapes)]
        st["norm"] = f32(1)
        st["max_norm"] = 1e-3 * math.sqrt(sum(size)) * (0.37 if case["clips"] else 2.0)
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _plain_score(st):
    case = st["case"]
    B, P, V, T, top = case["B"], case["P"], case["V"], case["T"], case["top"]
    token = st["tokens"].long()
    here = token >= 0
    if case["packed"]:
        row = (st["offsets"][:-1, None] + torch.arange(P, device="cuda")).clamp(max=st["z"].shape[0] - 1)
        z = st["z"][row].float()
    else:
        z = st["z"].float()
    at = token.clamp(min=0)[..., None]
    x = z / T
    d = x - x.max(-1, keepdim=True).values
    e = torch.exp(d)
    s = e.sum(-1)
    lse = x.max(-1).values + torch.log(s)
    entropy = torch.log(s) - (e * d.clamp(min=-1e30)).sum(-1) / s
    logprob = d.gather(-1, at)[..., 0] - torch.log(s)
    z_at = z.gather(-1, at)
    number = torch.arange(V, device="cuda")
    rank = 1 + ((z > z_at) | ((z == z_at) & (number < at))).sum(-1)
    zero = torch.zeros_like(lse)
    out = {"logprob": torch.where(here, logprob, zero), "lse": torch.where(here, lse, zero),
           "entropy": torch.where(here, entropy, zero), "rank": (rank * here).to(torch.int32)}
    if top:
        bits = (z + 0.0).view(torch.int32)
        order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + (V - 1 - number)
        token = V - 1 - (order.topk(top, -1).values & 0xFFFFFFFF)
        value = d.gather(-1, token) - torch.log(s)[..., None]
        there = here[..., None] & (value > -math.inf)
        out["top_token"] = torch.where(there, token, torch.full_like(token, PAD)).to(torch.int32)
        out["top_logprob"] = torch.where(there, value, torch.full_like(value, -math.inf))
    return out


def _plain_score_grad(st):
    T, z = st["case"]["T"], st["z"]
    token = st["tokens"].long()
    here = token >= 0
    at = token.clamp(min=0)[:, None]
    x = z.float() / T
    d = x - x.max(-1, keepdim=True).values
    e = torch.exp(d)
    s = e.sum(-1, keepdim=True)
    p = e / s
    logp = d.clamp(min=-1e30) - torch.log(s)
    g = (st["g_logprob"] * here)[:, None]
    dx = -g * p
    dx.scatter_add_(1, at, g)
    logprob = d.gather(-1, at)[:, 0] - torch.log(s)[:, 0]
    out = {"logprob": torch.where(here, logprob, torch.zeros_like(logprob))}
    if st["g_entropy"] is not None:
        entropy = -(p * logp).sum(-1)
        dx -= (st["g_entropy"] * here)[:, None] * p * (logp + entropy[:, None])
        out["entropy"] = torch.where(here, entropy, torch.zeros_like(entropy))
    out["dz"] = (dx / T).to(z.dtype)
    return out


def _plain_embed(st):
    ids = st["ids"].long()
    rows = st["table"][ids.clamp(min=0)].float() * st["scale"]
    return (rows * (ids >= 0)[:, None]).to(st["table"].dtype)


def _plain_embed_grad(st):
    ids, g = st["ids"].long(), st["grad_out"]
    total = torch.zeros(st["grad_table"].shape, dtype=torch.float32, device="cuda")
    total.index_add_(0, ids.clamp(min=0), g.float() * (ids >= 0)[:, None])
    return (total * st["scale"]).to(st["grad_table"].dtype)


def _plain_clip(st):
    norm = torch.stack([g.float().square().sum() for g in st["grads"]]).sum().sqrt()
    factor = (st["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    bucket = torch.cat([(g.float() * factor).to(st["bucket"].dtype).view(-1) for g in st["grads"]])
    return {"norm": norm.view(1), "bucket": bucket}


# ---------------------------------------------------------------------------
# the package's calls
# ---------------------------------------------------------------------------
def _own_score(st):
    import paper_2509_24328_amd as sv
    case = st["case"]
    top_token, top_logprob = (st["top_token"], st["top_logprob"]) if case["top"] else (None, None)
    sv.sv_token_logprobs(st["z"], st["tokens"], st["logprob"], st["lse"], st["entropy"], st["rank"], top_token,
                         top_logprob, temperature=case["T"], t_offsets=st["offsets"])
    names = ["logprob", "lse", "entropy", "rank"] + (["top_token", "top_logprob"] if case["top"] else [])
    return {n: st[n] for n in names}


def _own_score_grad(st):
    import paper_2509_24328_amd as sv
    sv.sv_token_logprobs_grad(st["z"], st["tokens"], st["g_logprob"], st["dz"], g_entropy=st["g_entropy"],
                              logprob=st["logprob"], entropy=st["entropy"], temperature=st["case"]["T"])
    return {n: st[n] for n in ("logprob", "entropy", "dz") if st[n] is not None}


def _own_embed(st):
    import paper_2509_24328_amd as sv
    sv.sv_embedding(st["table"], st["ids"], st["out"], scale=st["scale"])
    return st["out"]


def _own_embed_grad(st):
    import paper_2509_24328_amd as sv
    sv.sv_embedding_grad(st["grad_out"], st["ids"], st["grad_table"], scale=st["scale"], ws=st["scratch"])
    return st["grad_table"]


def _own_clip(st):
    import paper_2509_24328_amd as sv
    sv.sv_clip_grad_norm(st["grads"], st["max_norm"], st["norm"], out=st["clipped"], ws=st["scratch"])
    return {"norm": st["norm"], "bucket": st["bucket"]}


_PLAIN = {"score": _plain_score, "score_grad": _plain_score_grad, "embed": _plain_embed,
          "embed_grad": _plain_embed_grad, "clip": _plain_clip}
_OWN = {"score": _own_score, "score_grad": _own_score_grad, "embed": _own_embed, "embed_grad": _own_embed_grad,
        "clip": _own_clip}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["form"]](state)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    form = case["form"]
    if form == "score":
        B, P, V, top = case["B"], case["P"], case["V"], case["top"]
        n = B * P
        token = st["tokens"].reshape(n).long()
        on = (token >= 0).nonzero()[:, 0]                          # positions with a token, in order
        rows = st["z"].reshape(-1, V) if case["packed"] else st["z"].reshape(n, V)[on]
        f64 = lambda fill, *s: torch.full((n, *s), fill, dtype=torch.float64, device="cuda")
        i32 = lambda fill, *s: torch.full((n, *s), fill, dtype=torch.int32, device="cuda")
        out = {"logprob": f64(0.0), "lse": f64(0.0), "entropy": f64(0.0), "rank": i32(0)}
        if top:
            out.update(top_token=i32(PAD, top), top_logprob=f64(-math.inf, top))
        for lo in range(0, on.numel(), 512):
            i = on[lo:lo + 512]
            x = rows[lo:lo + 512].double() / case["T"]
            lse = torch.logsumexp(x, -1)
            logp = x - lse[:, None]
            order = x.sort(dim=-1, descending=True, stable=True).indices
            out["logprob"][i] = logp.gather(1, token[i, None])[:, 0]
            out["lse"][i] = lse
            out["entropy"][i] = torch.special.entr(logp.exp()).sum(-1)
            out["rank"][i] = (1 + (order == token[i, None]).long().argmax(-1)).to(torch.int32)
            if top:
                best = order[:, :top]
                value = logp.gather(1, best)
                out["top_logprob"][i] = value
                out["top_token"][i] = best.masked_fill(value == -math.inf, PAD).to(torch.int32)
        return {k: v.reshape(B, P, *v.shape[1:]) for k, v in out.items()}
    if form == "score_grad":
        B, T = case["B"], case["T"]
        out = {"logprob": torch.zeros(B, dtype=torch.float64, device="cuda")}
        if case["entropy"]:
            out["entropy"] = torch.zeros_like(out["logprob"])
        out["dz"] = torch.zeros((B, case["V"]), dtype=torch.float64, device="cuda")
        on = (st["tokens"] >= 0).nonzero()[:, 0]
        for lo in range(0, on.numel(), 256):
            i = on[lo:lo + 256]
            t = st["tokens"][i, None].long()
            x = st["z"][i].double() / T
            lp = x - torch.logsumexp(x, -1, keepdim=True)
            p = lp.exp()
            g = st["g_logprob"][i].double()[:, None]
            dx = (torch.zeros_like(p).scatter_(1, t, 1.0) - p) * g
            if case["entropy"]:
                h = torch.special.entr(p).sum(-1)
                dx += (torch.special.entr(p) - p * h[:, None]) * st["g_entropy"][i].double()[:, None]
                out["entropy"][i] = h
            out["logprob"][i] = lp.gather(1, t)[:, 0]
            out["dz"][i] = dx / T
        return out
    if form == "embed":
        out = torch.zeros((case["n"], case["D"]), dtype=torch.float64, device="cuda")
        on = st["ids"] >= 0
        out[on] = st["table"][st["ids"][on].long()].double() * math.sqrt(case["D"])
        return out
    if form == "embed_grad":
        # rows summed in the order of their tokens, as differences of one running sum per block of columns
        ids = st["ids"].long()
        order = ids.argsort(stable=True)
        last = torch.searchsorted(ids[order].contiguous(), torch.arange(-1, case["V"], device="cuda"), right=True)
        out = torch.empty((case["V"], case["D"]), dtype=torch.float64, device="cuda")
        for lo in range(0, case["D"], 512):
            run_sum = st["grad_out"][order, lo:lo + 512].double().cumsum(0)
            run_sum = torch.cat([torch.zeros_like(run_sum[:1]), run_sum])
            out[:, lo:lo + 512] = run_sum[last[1:]] - run_sum[last[:-1]]
        return out * math.sqrt(case["D"])
    squares = sum(float(g.double().pow(2).sum()) for g in st["grads"])
    norm = math.sqrt(squares)
    factor = min(1.0, st["max_norm"] / (norm + 1e-6))
    bucket = torch.cat([g.double().reshape(-1) * factor for g in st["grads"]])
    return {"norm": torch.tensor([norm], dtype=torch.float64), "bucket": bucket}


def work(case):
    """Every needed input read once, every output written once."""
    form = case["form"]
    if form == "score":
        rows, V = _rows(case), case["V"]
        # per entry: the exponent (subtraction, product), exponential, two sums, comparison
        return {"bytes": float(rows) * V * _BYTES[case["dtype"]] + case["B"] * case["P"] * (20.0 + 8.0 * case["top"]),
                "flops": 7.0 * rows * V}
    if form == "score_grad":
        B, V = case["B"], case["V"]
        read = B - B // 10                        # (rows without a token are written, not read)
        return {"bytes": float(B + read) * V * _BYTES[case["dtype"]] + 20.0 * B,
                "flops": float(read) * V * (12.0 if case["entropy"] else 8.0)}
    if form == "embed":
        return {"bytes": 2.0 * case["n"] * case["D"] * _BYTES[case["dtype"]] + 4.0 * case["n"],
                "flops": float(case["n"]) * case["D"]}
    if form == "embed_grad":
        n, V, D = case["n"], case["V"], case["D"]
        return {"bytes": float(n) * D * _BYTES[case["dtype"]] + float(V) * D * _BYTES[case["out"]] + 4.0 * n,
                "flops": float(n + V) * D}
    count = sum(math.prod(s) for s in _shapes(case))
    return {"bytes": float(count) * (_BYTES[case["dtype"]] + _BYTES[case["out"]]), "flops": 3.0 * count}
