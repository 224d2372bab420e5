"""The operators of layers with a sliding window and of drafted tokens, as timed cases.

Four operators, each through the package's public functions:

``rotary``  rotary positions of queries and keys;
``append``  new tokens into the cache of a layer with a sliding window, whose
            slots behind the first few tokens are a ring, keys and queries
            rotated on the way;
``window``  attention over such a cache: every query sees the last tokens up
            to itself and a few first ones; prompts, drafts, single tokens;
``verify``  drafted tokens against the target's probabilities, and the token
            that follows the accepted ones.

Shapes are those of the repository's workloads (28 query / 4 KV heads of 128
channels, contexts up to 131072 tokens, batches up to 64) and their
neighbours. ``run`` computes them in plain torch operations, or with the
package's functions where ``own`` is set.
"""
import math

import torch

own = False

D = 128          # head dimension
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ALL = 1 << 30    # a window that every key is in


# ------------------------------------------------------------------- cases

def listed():
    return [
        # the prompts of a serving batch, as a projection leaves them (token-major), rotated in one go
        {"name": "rotary_8k_b8", "op": "rotary", "batch": 8, "tokens": 8192, "hq": 28, "hkv": 4, "pairs": 64,
         "interleaved": False, "dtype": "bf16", "layout": "bthd", "positions": "first", "start": 0, "scaling": 1.0},
        # packed sequences far into a long context, part of the head, neighbouring channels as pairs
        {"name": "rotary_1001_b3", "op": "rotary", "batch": 3, "tokens": 1001, "hq": 16, "hkv": 16, "pairs": 24,
         "interleaved": True, "dtype": "fp32", "layout": "bhtd", "positions": "each", "start": 1000000,
         "scaling": 8.0},
        # a decoding step with four drafts: q and k rotated, k and v into a ring that has wrapped
        {"name": "append_drafts_b16", "op": "append", "batch": 16, "tokens": 5, "hq": 28, "hkv": 4, "pairs": 64,
         "interleaved": False, "window": 1024, "sinks": 4, "rows": 1056, "held": 5000, "ragged": False,
         "layout": "bthd"},
        # prompts of different lengths, longer than the ring they leave their last tokens in
        {"name": "append_4097_b8", "op": "append", "batch": 8, "tokens": 4097, "hq": 28, "hkv": 4, "pairs": 32,
         "interleaved": True, "window": 2048, "sinks": 16, "rows": 2100, "held": 0, "ragged": True,
         "layout": "bhtd"},
        # one token of one request: latency is all that counts
        {"name": "window_step_b1", "op": "window", "batch": 1, "tokens": 1, "hq": 28, "hkv": 4, "window": 1024,
         "sinks": 4, "rows": 1056, "held": 5000, "ragged": False, "layout": "bhtd"},
        # one token of a full serving batch: keys and values in reach are read
        {"name": "window_step_b64", "op": "window", "batch": 64, "tokens": 1, "hq": 28, "hkv": 4, "window": 4096,
         "sinks": 4, "rows": 8192, "held": 8191, "ragged": True, "layout": "bhtd"},
        # five drafted tokens each over a ring, odd sizes
        {"name": "window_drafts_b16", "op": "window", "batch": 16, "tokens": 5, "hq": 16, "hkv": 2, "window": 1000,
         "sinks": 3, "rows": 1011, "held": 3333, "ragged": False, "layout": "bthd"},
        # prompts of very different lengths in one batch (one empty, one of a single token), as many KV as query heads
        {"name": "window_4097_ragged", "op": "window", "batch": 16, "tokens": 4097, "hq": 16, "hkv": 16,
         "window": 512, "sinks": 4, "rows": 4097, "held": 0, "ragged": True, "layout": "bthd"},
        # one very long prompt
        {"name": "window_64k_b1", "op": "window", "batch": 1, "tokens": 65536, "hq": 28, "hkv": 4, "window": 4096,
         "sinks": 4, "rows": 65536, "held": 0, "ragged": False, "layout": "bhtd"},
        # one request, four drafts of a small model at the temperature that it sampled with
        {"name": "verify_b1_d4", "op": "verify", "batch": 1, "drafts": 4, "vocab": 32000, "dtype": "fp32",
         "temperature": 0.8, "model": True, "ragged": False},
        # greedy serving with drafts that came from the text itself, odd sizes, some sequences with fewer drafts
        {"name": "verify_b7_d3", "op": "verify", "batch": 7, "drafts": 3, "vocab": 65537, "dtype": "fp16",
         "temperature": 0.0, "model": False, "ragged": True},
        # a large batch, five drafts, a large vocabulary
        {"name": "verify_b32_d5", "op": "verify", "batch": 32, "drafts": 5, "vocab": 150001, "dtype": "bf16",
         "temperature": 1.0, "model": True, "ragged": False},
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    what = rng.choice(["rotary", "append", "step", "prompt", "prompt", "verify"])
    hq, hkv = rng.choice([(28, 4), (28, 4), (16, 16), (8, 8), (12, 4), (16, 2), (7, 1)])
    layout = rng.choice(["bhtd", "bthd"])
    if what == "rotary":
        tokens = _log_uniform(rng, 1, 65536)
        most = 8 * 8192 * 32 // (tokens * (hq + hkv))
        return {"op": "rotary", "batch": _log_uniform(rng, 1, max(1, min(64, most))), "tokens": tokens if most else 32768,
                "hq": hq, "hkv": hkv, "pairs": rng.choice([64, 64, 32, 20, 1, 63]), "interleaved": rng.random() < 0.5,
                "dtype": rng.choice(["bf16", "bf16", "fp16"]), "layout": layout,
                "positions": rng.choice(["first", "each"]), "start": rng.choice([0, 1000, 1000000]),
                "scaling": rng.choice([1.0, 4.0, 32.0])}
    window = _log_uniform(rng, 1, 8192)
    sinks = rng.choice([0, 1, 4, 4, 16, 100])
    if what == "append":
        tokens = rng.randint(1, 8) if rng.random() < 0.5 else _log_uniform(rng, 9, 8192)
        most = 8 * 8192 * 32 // (tokens * (hq + 2 * hkv))
        return {"op": "append", "batch": _log_uniform(rng, 1, max(1, min(64, most))), "tokens": tokens, "hq": hq,
                "hkv": hkv, "pairs": rng.choice([64, 32, 17]), "interleaved": rng.random() < 0.5, "window": window,
                "sinks": sinks, "rows": sinks + window + tokens - 1 + rng.randint(0, 64) if tokens <= 8
                else sinks + window + rng.randint(7, 64), "held": rng.choice([0, 10, 7777]),
                "ragged": rng.random() < 0.4, "layout": layout}
    if what == "step":
        # drafts or single tokens over a ring, or over rows that hold every token
        tokens = rng.randint(1, 8)
        ring = rng.random() < 0.6
        held = _log_uniform(rng, 1, 16384)
        # at most the rows of the largest listed case
        most = max(1, min(64, (1 << 21) // (hkv * ((window if ring else held) + sinks + 8))))
        return {"op": "window", "batch": _log_uniform(rng, 1, most), "tokens": tokens, "hq": hq, "hkv": hkv,
                "window": window if ring or rng.random() < 0.7 else ALL, "sinks": sinks,
                "rows": sinks + window + tokens - 1 + rng.randint(0, 64) if ring else held + tokens + rng.randint(0, 9),
                "held": held, "ragged": rng.random() < 0.5, "layout": layout}
    if what == "prompt":
        # at most the products of the largest listed case
        tokens = _log_uniform(rng, 9, 65536)
        if tokens < 16384 and rng.random() < 0.3:
            window = ALL
        most = 65536 * 4096 * 28 // (tokens * min(window, tokens) * hq)
        rows = 8 * 8192 * 32 // (tokens * (hq + hkv))
        if most == 0:
            window = 1024
        held = rng.choice([0, 0, 500])
        return {"op": "window", "batch": _log_uniform(rng, 1, max(1, min(64, most, rows))), "tokens": tokens,
                "hq": hq, "hkv": hkv, "window": window, "sinks": sinks, "rows": held + tokens + rng.randint(0, 3),
                "held": held, "ragged": rng.random() < 0.4, "layout": layout}
    return {"op": "verify", "batch": _log_uniform(rng, 1, 32), "drafts": rng.randint(1, 5),
            "vocab": _log_uniform(rng, 1000, 150001), "dtype": rng.choice(["fp32", "bf16", "fp16"] if rng.random() < 0.3
                                                                          else ["bf16", "fp16"]),
            "temperature": rng.choice([0.0, 0.6, 1.0, 1.0, 1.5]), "model": rng.random() < 0.6,
            "ragged": rng.random() < 0.3}


# ------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _counts(case, most):
    """Of each sequence: all of them, or spread down to one and none."""
    B = case["batch"]
    if not case["ragged"]:
        return [most] * B
    n = [max(1, most - (most * b) // B) for b in range(B)]
    if B > 1:
        n[1] = 0
    if B > 2:
        n[2] = 1
    return n


def _held(case):
    """Tokens that each sequence of a step holds before it."""
    B, held = case["batch"], case["held"]
    return [held - (held * b) // (2 * B) if case["ragged"] else held for b in range(B)]


def _new(case):
    """New tokens of each sequence: ragged prompts end early, steps are whole."""
    return _counts(case, case["tokens"]) if case["held"] == 0 else [case["tokens"]] * case["batch"]


def _freqs(pairs, scaling):
    """Radians per token of each pair; scaled: slow pairs by 1 / scaling, fast
    ones not at all, those between in proportion to their turns over 8192 tokens."""
    out = []
    for i in range(pairs):
        f = 10000.0 ** (-i / pairs)
        keep = min(1.0, max(0.0, (8192 * f / (2 * math.pi) - 1.0) / 3.0))
        out.append(f * (keep + (1.0 - keep) / scaling))
    return out


def _rows(g, B, H, T, layout, dtype=torch.bfloat16):
    if layout == "bthd":    # as a projection leaves them: [B, T, H, D] seen as [B, H, T, D]
        return torch.randn((B, T, H, D), generator=g, device=DEV, dtype=torch.float32).to(dtype).transpose(1, 2)
    return torch.randn((B, H, T, D), generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _prepare_rotary(case, g):
    B, T = case["batch"], case["tokens"]
    dtype = DTYPES[case["dtype"]]
    s = {"q": _rows(g, B, case["hq"], T, case["layout"], dtype), "k": _rows(g, B, case["hkv"], T, case["layout"], dtype),
         "interleaved": case["interleaved"], "scale": 1.0 + 0.1 * math.log(case["scaling"])}
    s["freqs"] = _freqs(case["pairs"], case["scaling"])
    first = case["start"] + torch.randint(0, 1000, (B, 1), generator=g, device=DEV)
    if case["positions"] == "each":     # sequences packed one behind another start anew now and then
        first = first + torch.arange(T, device=DEV) % max(1, T - T // 3)
    s["positions"] = first.to(torch.int32)
    return s


def _prepare_cache(case, g):
    B, hkv, rows = case["batch"], case["hkv"], case["rows"]
    return {"cache_k": _rows(g, B, hkv, rows, "bhtd"), "cache_v": _rows(g, B, hkv, rows, "bhtd"),
            "window": case["window"], "sinks": case["sinks"], "n_rows": rows}


def _prepare_append(case, g):
    B, T = case["batch"], case["tokens"]
    s = _prepare_cache(case, g)
    s.update({"q": _rows(g, B, case["hq"], T, case["layout"]), "k": _rows(g, B, case["hkv"], T, case["layout"]),
              "v": _rows(g, B, case["hkv"], T, case["layout"]), "freqs": _freqs(case["pairs"], 1.0),
              "interleaved": case["interleaved"], "scale": 1.0, "ragged": case["ragged"] and case["held"] == 0,
              "held": _ints(_held(case)), "new": _ints(_new(case))})
    return s


def _prepare_window(case, g):
    # keys are in the cache already, the new tokens' among them; a ring holds what it holds behind the last
    s = _prepare_cache(case, g)
    s["q"] = _rows(g, case["batch"], case["hq"], case["tokens"], case["layout"])
    new = _new(case)
    s["host"] = [(h + n, n) for h, n in zip(_held(case), new)]
    s["lengths"], s["new"] = _ints([x[0] for x in s["host"]]), _ints(new)
    s["ragged"] = case["ragged"] and case["held"] == 0
    return s


def _prepare_verify(case, g):
    B, T, V = case["batch"], case["drafts"], case["vocab"]
    dtype, tau = DTYPES[case["dtype"]], case["temperature"]
    x = torch.randn((B, T + 1, V), generator=g, device=DEV) * 2.5
    ban = torch.rand((B, T + 1, V), generator=g, device=DEV) < 0.01    # as a sampler's filters leave them
    target = x.masked_fill(ban, -math.inf).to(dtype)
    draft = None
    if case["model"]:
        # a drafter that mostly agrees
        draft = (x[:, :T] + 0.5 * torch.randn((B, T, V), generator=g, device=DEV)).masked_fill_(ban[:, :T], -math.inf) \
            .to(dtype)
    del x, ban
    noise = torch.empty((B, T, V), device=DEV).exponential_(generator=g)
    source = (target[:, :T] if draft is None else draft).float()
    tokens = (source / max(tau, 0.1) - noise.log()).argmax(dim=-1)
    s = {"target": target, "draft": draft, "tokens": tokens.to(torch.int32), "temperature": tau,
         "n": _ints(_counts(case, T)) if case["ragged"] else None, "u": None, "noise": None}
    if tau > 0:
        s["u"] = torch.rand((B, T), generator=g, device=DEV)
        s["noise"] = torch.empty((B, V), device=DEV).exponential_(generator=g).clamp_(min=1e-30)
    return s


def prepare(case, seed):
    g = _generator(seed)
    s = {"rotary": _prepare_rotary, "append": _prepare_append, "window": _prepare_window,
         "verify": _prepare_verify}[case["op"]](case, g)
    s["op"] = case["op"]
    if own:
        # what such a program keeps: the rotation's table and the cache's description
        import paper_2609_32831_gb300 as uc
        if "freqs" in s:
            s["rotary"] = uc.Rotary(s["freqs"], interleaved=s["interleaved"], scale=s["scale"])
        if "cache_k" in s:
            s["cache"] = uc.WindowCache(s["cache_k"], s["cache_v"], s["window"], s["sinks"])
    return s


# -------------------------------------------------------------- one pass

def _turn(x, positions, freqs, interleaved, scale):
    """x [B, H, T, D] turned by positions [B, T] times freqs; far angles need 64 bits."""
    n = len(freqs)
    angle = positions.double()[:, None, :, None] * torch.tensor(freqs, dtype=torch.float64, device=DEV)
    cos, sin = torch.cos(angle).float() * scale, torch.sin(angle).float() * scale
    y = x.float()
    if interleaved:
        a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = y[..., :n], y[..., n:2 * n]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((turned, y[..., 2 * n:]), dim=-1).to(x.dtype)


def _plain_rotary(s):
    T = s["q"].shape[2]
    p = s["positions"]
    if p.shape[1] == 1:
        p = p + torch.arange(T, device=DEV)
    return {"q": _turn(s["q"], p, s["freqs"], s["interleaved"], s["scale"]),
            "k": _turn(s["k"], p, s["freqs"], s["interleaved"], s["scale"])}


def _slots(s, p):
    """The cache's row of each position."""
    return torch.where(p < s["sinks"], p, s["sinks"] + (p - s["sinks"]) % (s["n_rows"] - s["sinks"]))


def _plain_append(s):
    B, hkv, T, _ = s["k"].shape
    t = torch.arange(T, device=DEV)
    p = s["held"].long()[:, None] + t
    q = _turn(s["q"], p, s["freqs"], s["interleaved"], s["scale"])
    k = _turn(s["k"], p, s["freqs"], s["interleaved"], s["scale"])
    # of a ring's slot the last token that falls into it stays
    total = s["held"] + s["new"]
    write = (t < s["new"][:, None]) & ((p < s["sinks"]) | (p >= total[:, None] - (s["n_rows"] - s["sinks"])))
    b, i = torch.nonzero(write, as_tuple=True)
    at = _slots(s, p)[b, i]
    s["cache_k"][b, :, at] = k[b, :, i]
    s["cache_v"][b, :, at] = s["v"][b, :, i]
    # queries behind a sequence's last token are turned as well: their rows are nobody's
    return {"q": q, "k": s["cache_k"], "v": s["cache_v"], "total": total}


def _attend(q, k, v, seen):
    """q [.., g t, D], k, v [.., n, D], seen: which keys a query sees. Rows that see none: 0 and -inf."""
    x = (q @ k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    x = x.masked_fill_(~seen, -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    base = torch.where(top == -math.inf, 0.0, top)
    e = x.sub_(base).exp_()
    total = e.sum(dim=-1, keepdim=True)
    o = (e @ v) / torch.where(total == 0, 1.0, total)
    return o, (torch.log(total) + base)[..., 0]


def _plain_window(s):
    q, W, S = s["q"], s["window"], s["sinks"]
    B, hq, T, _ = q.shape
    hkv = s["cache_k"].shape[1]
    grp = hq // hkv
    if T <= 8:
        # every slot of the cache, masked by the token that it holds
        R = s["n_rows"] - S
        n = s["lengths"].long()[:, None]
        slot = torch.arange(s["n_rows"], device=DEV)
        held = torch.where(slot < S, slot, slot + (n - 1 - slot).div(R, rounding_mode="floor") * R)     # [B, rows]
        p = n - s["new"][:, None] + torch.arange(T, device=DEV)                                         # [B, T]
        seen = (held[:, None] <= p[..., None]) & ((p[..., None] - held[:, None] < W) | (held[:, None] < S))
        # (a ring's slot that no token has reached yet would stand for one before the ring's first)
        seen &= ((slot < S) | (held >= S))[:, None] & (p >= 0)[..., None] & (p < n)[..., None]
        seen = seen[:, None, None].expand(B, 1, grp, T, -1).reshape(B, 1, grp * T, -1)
        o, lse = _attend(q.reshape(B, hkv, grp * T, D).float(), s["cache_k"].float(), s["cache_v"].float(), seen)
        return {"out": o.reshape(B, hq, T, D).to(q.dtype), "lse": lse.reshape(B, hq, T)}
    out = torch.zeros_like(q)
    lse = torch.full((B, hq, T), -math.inf, device=DEV)
    step = 512
    for b, (n, new) in enumerate(s["host"]):
        for t0 in range(0, new, step):
            t1 = min(new, t0 + step)
            p = n - new + torch.arange(t0, t1, device=DEV)
            lo = max(0, n - new + t0 - W + 1)
            keys = torch.cat((torch.arange(min(S, lo), device=DEV), torch.arange(lo, n - new + t1, device=DEV)))
            at = _slots(s, keys)
            seen = (keys <= p[:, None]) & ((p[:, None] - keys < W) | (keys < S))
            qb = q[b, :, t0:t1].reshape(hkv, grp * (t1 - t0), D).float()
            o, l = _attend(qb, s["cache_k"][b][:, at].float(), s["cache_v"][b][:, at].float(), seen.repeat(grp, 1))
            out[b, :, t0:t1] = o.view(hq, t1 - t0, D).to(q.dtype)
            lse[b, :, t0:t1] = l.view(hq, t1 - t0)
    return {"out": out, "lse": lse}


def _log_probs(x, tau):
    x = x.double() / tau
    top = x.amax(dim=-1, keepdim=True)
    return x - (top + torch.log(torch.exp(x - top).sum(dim=-1, keepdim=True)))


def _plain_verify(s):
    B, T1, V = s["target"].shape
    T, tau = T1 - 1, s["temperature"]
    tokens = s["tokens"].long()
    n = torch.full((B,), T, device=DEV) if s["n"] is None else s["n"].long()
    ids = torch.arange(V, device=DEV)
    lp = _log_probs(s["target"], tau if tau > 0 else 1.0)
    here = lp[:, :T].gather(2, tokens[..., None])[..., 0]
    if tau == 0:
        best = torch.where(lp == lp.amax(dim=-1, keepdim=True), ids, V).amin(dim=-1)                    # [B, T + 1]
        good = tokens == best[:, :T]
    else:
        lq = None if s["draft"] is None else _log_probs(s["draft"], tau)
        drawn = torch.ones_like(here) if lq is None else lq.gather(2, tokens[..., None])[..., 0].exp()
        good = s["u"].double() * drawn < here.exp()
    good &= torch.arange(T, device=DEV) < n[:, None]
    a = torch.cumprod(good.long(), dim=1).sum(dim=1)
    row = torch.arange(B, device=DEV)
    if tau == 0:
        last = best[row, a]
    else:
        w = lp[row, a].exp()
        at = a.clamp(max=T - 1)
        if lq is None:
            taken = (ids == tokens[row, at][:, None]).double()
        else:
            taken = lq[row, at].exp()
        w = torch.where((a < n)[:, None], (w - taken).clamp_(min=0.0), w)
        w = w / s["noise"].double()
        last = torch.where(w == w.amax(dim=-1, keepdim=True), ids, V).amin(dim=-1)
    t = torch.arange(T1, device=DEV)
    out = torch.cat((tokens, torch.zeros((B, 1), dtype=torch.long, device=DEV)), dim=1)
    out = torch.where(t < a[:, None], out, torch.where(t == a[:, None], last[:, None], -1))
    logp = torch.where(t <= a[:, None], lp.gather(2, out.clamp(min=0)[..., None])[..., 0], 0.0)
    return {"accepted": a.to(torch.int32), "tokens": out.to(torch.int32), "logprob": logp.float()}


def run(s):
    if not own:
        return {"rotary": _plain_rotary, "append": _plain_append, "window": _plain_window,
                "verify": _plain_verify}[s["op"]](s)
    import paper_2609_32831_gb300 as uc
    if s["op"] == "rotary":
        q, k = uc.rotary(s["rotary"], s["positions"], s["q"], s["k"])
        return {"q": q, "k": k}
    if s["op"] == "append":
        total, q = uc.window_append(s["cache"], s["k"], s["v"], s["held"], n_new=s["new"] if s["ragged"] else None,
                                    rotary=s["rotary"], q=s["q"])
        return {"q": q, "k": s["cache_k"], "v": s["cache_v"], "total": total}
    if s["op"] == "window":
        out, lse = uc.window_attend(s["q"], s["cache"], s["lengths"], n_query=s["new"] if s["ragged"] else None)
        return {"out": out, "lse": lse}
    accepted, tokens, logprob = uc.verify_draft(s["target"], s["tokens"], u=s["u"], noise=s["noise"],
                                                draft_logits=s["draft"], n_draft=s["n"], temperature=s["temperature"])
    return {"accepted": accepted, "tokens": tokens, "logprob": logprob}


# ------------------------------------------------------------ the least work

def _reach(case):
    """(pairs of query and key that see each other, keys in reach) summed over the sequences."""
    W, S = case["window"], case["sinks"]
    pairs = keys = 0
    for held, new in zip(_held(case), _new(case)):
        n = held + new
        if new == 0:
            continue
        lo = max(0, held - W + 1)               # the first query's oldest key
        keys += n - lo + min(S, lo)
        a, b = held + 1, n                      # keys up to the first, the last query
        full = min(b, max(a - 1, W))            # queries up to here see everything before them
        pairs += (full * (full + 1) - (a - 1) * a) // 2 + (b - full) * W
        # sinks that the window has left behind
        gone = [max(0, p - W + 1) for p in (held, n - 1)]
        if gone[1] > 0:
            first = max(held, W - 1)
            left = n - 1 - first                # queries from `first` on have 0, 1, 2 .. keys behind their window
            base = first - W + 1
            ramp = max(0, min(left + 1, S - base))
            pairs += sum(base + i for i in (0, ramp - 1)) * ramp // 2 if ramp else 0
            pairs += (left + 1 - ramp) * S
    return pairs, keys


def work(case):
    if case["op"] == "rotary":
        rows = case["batch"] * case["tokens"] * (case["hq"] + case["hkv"])
        return {"bytes": rows * D * (8 if case["dtype"] == "fp32" else 4), "flops": 6.0 * case["pairs"] * rows}
    if case["op"] == "append":
        B, T, R = case["batch"], case["tokens"], case["rows"] - case["sinks"]
        kept = sum(n if n <= R else R + min(case["sinks"], n - R) for n in _new(case))
        return {"bytes": (2 * B * T * case["hq"] + 4 * kept * case["hkv"]) * D * 2,
                "flops": 6.0 * case["pairs"] * (B * T * case["hq"] + kept * case["hkv"])}
    if case["op"] == "window":
        pairs, keys = _reach(case)
        q = sum(_new(case)) * case["hq"] * D * 2
        out = case["batch"] * case["tokens"] * case["hq"] * (D * 2 + 4)
        return {"bytes": q + out + keys * case["hkv"] * D * 4, "flops": 4.0 * D * pairs * case["hq"]}
    size = 4 if case["dtype"] == "fp32" else 2
    drafts = sum(_counts(case, case["drafts"])) if case["ragged"] else case["batch"] * case["drafts"]
    rows = drafts + case["batch"] + (drafts if case["model"] and case["temperature"] > 0 else 0)
    noise = case["batch"] * case["vocab"] * 4 if case["temperature"] > 0 else 0
    return {"bytes": rows * case["vocab"] * size + noise, "flops": 4.0 * rows * case["vocab"]}


# -------------------------------------------------------------- 64 bits

def _exact_turn(x, positions, freqs, interleaved, scale):
    n = len(freqs)
    z = x.double()
    z = torch.complex(*(z[..., 0:2 * n:2], z[..., 1:2 * n:2]) if interleaved else (z[..., :n], z[..., n:2 * n]))
    f = torch.tensor(freqs, dtype=torch.float64, device=DEV)
    angle = positions.double()[..., None] * f
    z = z * torch.polar(torch.full_like(angle, scale), angle)[:, None]
    out = x.double().clone()
    if interleaved:
        out[..., 0:2 * n:2], out[..., 1:2 * n:2] = z.real, z.imag
    else:
        out[..., :n], out[..., n:2 * n] = z.real, z.imag
    return out


def _exact_rotary(case, s):
    p = s["positions"].long()
    if p.shape[1] == 1:
        p = torch.stack([p[:, 0] + t for t in range(case["tokens"])], dim=1)
    return {x: _exact_turn(s[x], p, s["freqs"], s["interleaved"], s["scale"]) for x in ("q", "k")}


def _exact_append(case, s):
    S, R = case["sinks"], case["rows"] - case["sinks"]
    held, new = _held(case), _new(case)
    p = torch.stack([torch.arange(case["tokens"], device=DEV) + h for h in held])
    q, k = (_exact_turn(s[x], p, s["freqs"], s["interleaved"], s["scale"]) for x in ("q", "k"))
    out = {"q": q, "k": s["cache_k"].double(), "v": s["cache_v"].double(), "total": None}
    for b in range(case["batch"]):
        # token after token would leave: the first S, and the last R of the rest
        n = held[b] + new[b]
        keep = [x for x in range(held[b], n) if x < S or x >= n - R]
        if keep:
            at = torch.tensor([x if x < S else S + (x - S) % R for x in keep], device=DEV)
            t = torch.tensor([x - held[b] for x in keep], device=DEV)
            out["k"][b, :, at] = k[b][:, t]
            out["v"][b, :, at] = s["v"][b][:, t].double()
    return out


def _exact_window(case, s):
    W, S, R = case["window"], case["sinks"], case["rows"] - case["sinks"]
    B, hq, T, hkv = case["batch"], case["hq"], case["tokens"], case["hkv"]
    out = torch.zeros((B, hq, T, D), dtype=torch.float64, device=DEV)
    lse = torch.full((B, hq, T), -math.inf, dtype=torch.float64, device=DEV)
    for b, (n, new) in enumerate(s["host"]):
        for t0 in range(0, new, 256):
            p = torch.arange(n - new + t0, n - new + min(new, t0 + 256), device=DEV)
            first = max(0, int(p[0]) - W + 1)
            keys = sorted(set(range(min(S, int(p[-1]) + 1))) | set(range(first, int(p[-1]) + 1)))
            keys = torch.tensor(keys, device=DEV)
            rows = keys.clone()
            rows[keys >= S] = S + torch.remainder(keys[keys >= S] - S, R)
            gap = p[:, None] - keys[None]
            hide = (gap < 0) | ((gap >= W) & (keys[None] >= S))
            for j in range(hkv):
                k, v = s["cache_k"][b, j, rows].double(), s["cache_v"][b, j, rows].double()
                at = slice(j * (hq // hkv), (j + 1) * (hq // hkv))
                x = torch.einsum("htd,nd->htn", s["q"][b, at, t0:t0 + len(p)].double(), k) / math.sqrt(D)
                x = torch.where(hide, -math.inf, x)
                lse[b, at, t0:t0 + len(p)] = torch.logsumexp(x, dim=-1)
                out[b, at, t0:t0 + len(p)] = torch.softmax(x, dim=-1) @ v
    return {"out": out, "lse": lse}


def _exact_verify(case, s):
    B, T1, _ = s["target"].shape
    tau = case["temperature"] or 1.0
    got = _plain_verify(s)      # which tokens come out has no fraction: their log probabilities do
    logp = torch.zeros((B, T1), dtype=torch.float64, device=DEV)
    for b in range(B):
        for t in range(int(got["accepted"][b]) + 1):
            logp[b, t] = torch.log_softmax(s["target"][b, t].double() / tau, dim=-1)[int(got["tokens"][b, t])]
    return {"accepted": None, "tokens": None, "logprob": logp}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "append": _exact_append, "window": _exact_window,
            "verify": _exact_verify}[case["op"]](case, s)
