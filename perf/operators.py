"""The operators of generation with several continuations, as timed cases.

Three operators, each through the package's public functions:

``linear``   linear attention with a decay for each KV head, over a state of
             constant size: prompts (many tokens) and single tokens;
``beam``     the best continuations over a request's beams and vocabulary;
``reorder``  caches and states follow the beams that were chosen.

Shapes are those of the repository's workloads (28 query / 4 KV heads of 128
channels, contexts up to 131072 tokens, batches up to 64) and their
neighbours. ``run`` computes them in plain torch operations in 32 bits, or
with the package's functions where ``own`` is set.
"""
import math

import torch

own = False

D = 128          # head dimension
CHUNK = 128      # tokens per chunk of the plain form's chunked sums
GROUP = 32       # tokens per quantization group of a packed segment
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------- cases

def listed():
    return [
        # one token of one request through a layer: latency is all that counts
        {"name": "step_b1", "op": "linear", "batch": 1, "hq": 28, "hkv": 4, "tokens": 1, "state": True,
         "ragged": False, "layout": "bhtd"},
        # one token of a full serving batch: the states are read and written
        {"name": "step_b64", "op": "linear", "batch": 64, "hq": 28, "hkv": 4, "tokens": 1, "state": True,
         "ragged": False, "layout": "bhtd"},
        # five drafted tokens at once, as many KV as query heads, token-major rows
        {"name": "draft5_b8", "op": "linear", "batch": 8, "hq": 16, "hkv": 16, "tokens": 5, "state": True,
         "ragged": False, "layout": "bthd"},
        # one request's short prompt, from an empty state
        {"name": "prompt_1000_b1", "op": "linear", "batch": 1, "hq": 28, "hkv": 4, "tokens": 1000, "state": False,
         "ragged": False, "layout": "bthd"},
        # prompts of very different lengths in one batch (one empty, one of a
        # single token) on top of earlier turns
        {"name": "prompt_4097_ragged", "op": "linear", "batch": 16, "hq": 16, "hkv": 16, "tokens": 4097,
         "state": True, "ragged": True, "layout": "bthd"},
        # the understanding workload's prompts, batch 8
        {"name": "prompt_8k_b8", "op": "linear", "batch": 8, "hq": 28, "hkv": 4, "tokens": 8192, "state": False,
         "ragged": False, "layout": "bhtd"},
        # one very long context: few (sequence, head) pairs, split over tokens
        {"name": "prompt_128k_b1", "op": "linear", "batch": 1, "hq": 28, "hkv": 4, "tokens": 131072, "state": False,
         "ragged": False, "layout": "bhtd"},
        # the first step of one request: only beam 0 is alive
        {"name": "beam_b1_k4", "op": "beam", "batch": 1, "beams": 4, "vocab": 32000, "n": 4, "dtype": "fp32",
         "first": True, "finished": False},
        # a serving batch with finished beams and banned tokens, odd sizes
        {"name": "beam_b7_k5", "op": "beam", "batch": 7, "beams": 5, "vocab": 65537, "n": 10, "dtype": "fp16",
         "first": False, "finished": True},
        # a large batch, eight beams, a large vocabulary
        {"name": "beam_b32_k8", "op": "beam", "batch": 32, "beams": 8, "vocab": 150001, "n": 8, "dtype": "bf16",
         "first": False, "finished": False},
        # one request, a few generated tokens in bf16 rows and two states
        {"name": "reorder_b1_k4", "op": "reorder", "batch": 1, "beams": 4, "hkv": 4, "kept": 21, "kind": "evict",
         "bits": 16, "layers": 2, "states": 2},
        # sixteen requests, 1000 generated tokens at int4 and a state per layer
        {"name": "reorder_b16_k4", "op": "reorder", "batch": 16, "beams": 4, "hkv": 4, "kept": 1000, "kind": "quant",
         "bits": 4, "layers": 6, "states": 6},
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    what = rng.choice(["step", "prompt", "prompt", "beam", "reorder"])
    hq, hkv = rng.choice([(28, 4), (28, 4), (16, 16), (8, 8), (12, 4), (16, 2), (7, 1)])
    if what == "step":
        return {"op": "linear", "batch": _log_uniform(rng, 1, 64), "hq": hq, "hkv": hkv, "tokens": rng.randint(1, 8),
                "state": rng.random() < 0.8, "ragged": rng.random() < 0.3, "layout": rng.choice(["bhtd", "bthd"])}
    if what == "prompt":
        # at most the tokens x heads of the largest listed case
        tokens = _log_uniform(rng, 9, 131072)
        most = 131072 * 64 // (tokens * 2 * (hq + hkv))
        return {"op": "linear", "batch": _log_uniform(rng, 1, max(1, min(64, most))), "hq": hq, "hkv": hkv,
                "tokens": tokens if most else tokens // 2, "state": rng.random() < 0.5, "ragged": rng.random() < 0.4,
                "layout": rng.choice(["bhtd", "bthd"])}
    if what == "beam":
        k = rng.randint(1, 8)
        return {"op": "beam", "batch": _log_uniform(rng, 1, 32), "beams": k, "vocab": _log_uniform(rng, 1000, 150001),
                "n": rng.randint(1, 2 * k), "dtype": rng.choice(["fp32", "bf16", "fp16"]),
                "first": rng.random() < 0.2, "finished": rng.random() < 0.4}
    kind, bits = rng.choice([("evict", 16), ("quant", 4), ("quant", 2), ("evict_quant", 2)])
    k = rng.randint(1, 8)
    return {"op": "reorder", "batch": _log_uniform(rng, 1, 64 // k), "beams": k, "hkv": rng.choice([1, 2, 4, 8]),
            "kept": _log_uniform(rng, 1, 2000), "kind": kind, "bits": bits, "layers": rng.randint(1, 6),
            "states": rng.randint(0, 6)}


# ------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _lengths(case):
    """Tokens of each sequence: all of them, or spread down to one and none."""
    B, T = case["batch"], case["tokens"]
    if not case["ragged"]:
        return [T] * B
    n = [max(1, T - (T * b) // B) for b in range(B)]
    if B > 1:
        n[1] = 0
    if B > 2:
        n[2] = 1
    return n


def _log_decay(hkv):
    """Memories from about 10 to about 4000 tokens, spread over the heads."""
    return [math.log1p(-2.0 ** -(3.0 + 9.0 * (j + 0.5) / hkv)) for j in range(hkv)]


def _rows(g, B, H, T, layout):
    if layout == "bthd":    # as a projection leaves them: [B, T, H, D] seen as [B, H, T, D]
        return torch.randn((B, T, H, D), generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16).transpose(1, 2)
    return torch.randn((B, H, T, D), generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _prepare_linear(case, g):
    B, hq, hkv, T = case["batch"], case["hq"], case["hkv"], case["tokens"]
    s = {"q": _rows(g, B, hq, T, case["layout"]), "k": _rows(g, B, hkv, T, case["layout"]),
         "v": _rows(g, B, hkv, T, case["layout"]), "log_decay": _log_decay(hkv), "lengths": _lengths(case),
         "ragged": case["ragged"]}
    # a state as earlier tokens left it: sums of about 1 / (1 - gamma^2) products
    s["state"] = None
    if case["state"]:
        size = torch.tensor([1.0 / math.sqrt(-math.expm1(2 * d)) for d in s["log_decay"]], device=DEV)
        s["state"] = torch.randn((B, hkv, D, D), generator=g, device=DEV) * size[:, None, None]
    s["out_state"] = torch.empty((B, hkv, D, D), device=DEV)
    s["decay"] = torch.tensor(s["log_decay"], device=DEV)
    s["n"] = torch.tensor(s["lengths"], device=DEV)
    return s


def _prepare_beam(case, g):
    B, K, V = case["batch"], case["beams"], case["vocab"]
    logits = torch.randn((B, K, V), generator=g, device=DEV) * 2.5
    # banned tokens, as a sampler's filters leave them
    ban = torch.rand((B, K, V), generator=g, device=DEV) < 0.01
    logits = logits.masked_fill_(ban, -math.inf).to(DTYPES[case["dtype"]])
    scores = torch.sort(-2.0 * torch.randn((B, K), generator=g, device=DEV).abs(), dim=1, descending=True).values
    if case["first"]:
        scores = torch.full_like(scores, -math.inf)
        scores[:, 0] = 0.0
    finished = None
    if case["finished"]:
        finished = torch.rand((B, K), generator=g, device=DEV) < 0.3
    return {"logits": logits, "scores": scores, "finished": finished, "n": min(case["n"], K * V), "eos": 2}


def _segment_arrays(case, g):
    """Arrays of one segment as the package lays them out, per sequence and KV
    head, with what lies behind the kept tokens zero: {name: (tensor [S, Hkv,
    units, bytes of a unit as elements], live units [S])}."""
    S, hkv, bits = case["batch"] * case["beams"], case["hkv"], case["bits"]
    cap = (case["kept"] + 63) // 64 * 64
    # counts differ between requests, not between the beams of one
    n = torch.tensor([max(1, case["kept"] - (case["kept"] * (i // case["beams"])) // (4 * case["batch"]))
                      for i in range(S)], device=DEV)
    def rows(units, width, dtype):
        if dtype == torch.bfloat16:
            return torch.randn((S, hkv, units, width), generator=g, device=DEV).to(dtype)
        top = 256 if dtype == torch.uint8 else 100000
        return torch.randint(0, top, (S, hkv, units, width), generator=g, device=DEV, dtype=torch.int32).to(dtype)
    if case["kind"] == "evict":
        live = {"k": n, "v": n, "kept_idx": n}
        arrays = {"k": rows(cap, D, torch.bfloat16), "v": rows(cap, D, torch.bfloat16)}
    else:
        groups = n // GROUP
        live = {"k": n % GROUP, "v": n % GROUP, "kept_idx": n, "k_codes": groups, "v_codes": groups,
                "k_params": groups, "v_params": groups}
        arrays = {"k": rows(GROUP, D, torch.bfloat16), "v": rows(GROUP, D, torch.bfloat16)}
        for name, width in (("k_codes", GROUP * D * bits // 8), ("v_codes", GROUP * D * bits // 8),
                            ("k_params", 4 * D), ("v_params", 16 * GROUP)):
            arrays[name] = rows(cap // GROUP, width, torch.uint8)
    arrays["kept_idx"] = rows(cap, 1, torch.int32)
    for name, x in arrays.items():
        x.mul_(torch.arange(x.shape[2], device=DEV)[None, None, :, None] < live[name][:, None, None, None])
    return {"n": n, "live": live, "arrays": arrays, "cap": cap}


def _prepare_reorder(case, g):
    B, K = case["batch"], case["beams"]
    s = {"layers": [_segment_arrays(case, g) for _ in range(case["layers"])],
         "states": [torch.randn((B * K, case["hkv"], D, D), generator=g, device=DEV) for _ in range(case["states"])],
         "parent": torch.randint(0, K, (B, K), generator=g, device=DEV, dtype=torch.int32), "batch": B, "beams": K}
    s["new_states"] = [torch.empty_like(x) for x in s["states"]]
    if own:
        # the segments such a program keeps: two per layer, used in turn
        import paper_2609_32831_gb300 as uc
        s["pairs"] = []
        for layer in s["layers"]:
            src, dst = (uc.Segment(case["kind"], case["bits"], B * K, case["hkv"], 100000, layer["cap"], DEV)
                        for _ in range(2))
            src.set_keep(layer["n"].tolist())
            src.tensor("n_kept").copy_(layer["n"])
            for name, x in layer["arrays"].items():
                src.tensor(name).copy_(x.reshape(-1))
            s["pairs"].append((src, dst))
        s["pairs"] += list(zip(s["states"], s["new_states"]))
    return s


def prepare(case, seed):
    g = _generator(seed)
    s = {"linear": _prepare_linear, "beam": _prepare_beam, "reorder": _prepare_reorder}[case["op"]](case, g)
    s["op"] = case["op"]
    return s


# -------------------------------------------------------------- one pass

def _plain_linear(s):
    q, k, v, n = s["q"].float(), s["k"].float(), s["v"].float(), s["n"]
    B, hq, T, _ = q.shape
    hkv = k.shape[1]
    grp = hq // hkv
    C = min(CHUNK, T)
    nc = -(-T // C)
    there = (torch.arange(nc * C, device=DEV) < n[:, None])[:, None, :, None]           # [B, 1, t, 1]
    def padded(x):
        return torch.where(there, torch.nn.functional.pad(x, (0, 0, 0, nc * C - T)), 0.0)
    q = padded(q).view(B, hkv, grp, nc, C, D).transpose(2, 3).reshape(B, hkv, nc, grp * C, D)
    k, v = padded(k).view(B, hkv, nc, C, D), padded(v).view(B, hkv, nc, C, D)
    d = s["decay"]
    i = torch.arange(C, device=DEV)
    gap = (i[:, None] - i[None, :]).clamp(min=0)
    tri = torch.where(i[:, None] >= i[None, :], torch.exp(d[:, None, None] * gap), 0.0)  # [hkv, i, j]
    a = (q @ k.transpose(-1, -2)).view(B, hkv, nc, grp, C, C) * tri[:, None, None]
    o = a.view(B, hkv, nc, grp * C, C) @ v
    # the state each chunk starts from: earlier chunks' sums, decayed
    kv = (k * torch.exp(d[:, None] * (C - 1 - i))[:, None, :, None]).transpose(-1, -2) @ v
    c = torch.arange(nc, device=DEV)
    back = c[:, None] - 1 - c[None, :]
    carry = torch.where(back >= 0, torch.exp(d[:, None, None] * C * back.clamp(min=0)), 0.0)
    start = (carry @ kv.view(B, hkv, nc, D * D)).view(B, hkv, nc, D, D)
    if s["state"] is not None:
        start = start + torch.exp(d[:, None] * C * c)[None, :, :, None, None] * s["state"][:, :, None]
    o = o + (q @ start).view(B, hkv, nc, grp, C, D).mul_(torch.exp(d[:, None] * (i + 1))[:, None, None, :, None]) \
        .view(B, hkv, nc, grp * C, D)
    o = o.view(B, hkv, nc, grp, C, D).transpose(2, 3).reshape(B, hq, nc * C, D)[:, :, :T] * (1.0 / math.sqrt(D))
    o = torch.where(there[:, :, :T], o, 0.0).to(torch.bfloat16)
    # the state behind each sequence's own last token
    left = (n[:, None] - 1 - torch.arange(nc * C, device=DEV)).clamp(min=0)              # [B, t]
    w = torch.exp(d[None, :, None] * left[:, None, :])[..., None]
    state = (k.view(B, hkv, nc * C, D) * w).transpose(-1, -2) @ v.view(B, hkv, nc * C, D)
    if s["state"] is not None:
        state = state + torch.exp(d[None, :] * n[:, None])[..., None, None] * s["state"]
    return {"out": o, "state": state}


def _plain_beam(s):
    x = s["logits"].float() + 0.0
    B, K, V = x.shape
    if s["finished"] is not None:
        # a finished beam goes on with the end token alone, at no cost
        only = torch.where(torch.arange(V, device=DEV) == s["eos"], 0.0, -math.inf)
        x = torch.where(s["finished"][..., None], only, x)
    top = x.amax(dim=-1, keepdim=True)
    base = torch.where(torch.isinf(top), 0.0, top)
    total = torch.log(torch.exp(x - base).sum(dim=-1, keepdim=True))
    n = s["n"]
    row, token = (t[..., :n] for t in torch.sort(x, dim=-1, descending=True, stable=True))
    gain = torch.where(torch.isinf(row), -math.inf, (row - base) - total)
    cand = (s["scores"][..., None] + gain).reshape(B, -1)
    best, at = (t[:, :n] for t in torch.sort(cand, dim=-1, descending=True, stable=True))
    per = token.shape[-1]
    token, parent = token.reshape(B, -1).gather(1, at), at // per
    out = {"scores": best, "parent": parent.to(torch.int32), "token": token.to(torch.int32),
           "finished": token == s["eos"]}
    if s["finished"] is not None:
        out["finished"] = out["finished"] | s["finished"].gather(1, parent)
    return out


def _plain_reorder(s):
    src = (torch.arange(s["batch"], device=DEV)[:, None] * s["beams"] + s["parent"]).reshape(-1)
    out = {}
    for i, layer in enumerate(s["layers"]):
        out["n%d" % i] = layer["n"][src].to(torch.int32)
        for name, x in layer["arrays"].items():
            out["%s%d" % (name, i)] = x[src].reshape(-1)
    for i, x in enumerate(s["states"]):
        out["state%d" % i] = x[src]
    return out


def run(s):
    if not own:
        return {"linear": _plain_linear, "beam": _plain_beam, "reorder": _plain_reorder}[s["op"]](s)
    import paper_2609_32831_gb300 as uc
    if s["op"] == "linear":
        out, state = uc.linear_attend(s["q"], s["k"], s["v"], s["log_decay"], state=s["state"],
                                      out_state=s["out_state"], lengths=s["lengths"] if s["ragged"] else None)
        return {"out": out, "state": state}
    if s["op"] == "beam":
        scores, parent, token, finished = uc.beam_select(s["logits"], s["scores"], s["n"], finished=s["finished"],
                                                         eos=s["eos"])
        return {"scores": scores, "parent": parent, "token": token, "finished": finished}
    uc.reorder(s["pairs"], s["parent"])
    out = {}
    for i, layer in enumerate(s["layers"]):
        dst = s["pairs"][i][1]
        out["n%d" % i] = dst.tensor("n_kept")
        for name in layer["arrays"]:
            out["%s%d" % (name, i)] = dst.tensor(name)
    for i, x in enumerate(s["new_states"]):
        out["state%d" % i] = x
    return out


# ------------------------------------------------------------ the least work

def work(case):
    if case["op"] == "linear":
        B, hq, hkv, T = case["batch"], case["hq"], case["hkv"], case["tokens"]
        t = sum(_lengths(case))
        state = B * hkv * D * D * 4
        return {"bytes": t * (hq + 2 * hkv) * D * 2 + B * T * hq * D * 2 + state * (2 if case["state"] else 1),
                "flops": 2.0 * D * D * (hq + hkv) * t}
    if case["op"] == "beam":
        rows = case["batch"] * case["beams"]
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": rows * case["vocab"] * size + rows * 4 + case["batch"] * case["n"] * 13,
                "flops": 4.0 * rows * case["vocab"]}
    B, K, hkv = case["batch"], case["beams"], case["hkv"]
    per_seq = case["states"] * hkv * D * D * 4
    live = 0
    for b in range(B):
        n = max(1, case["kept"] - (case["kept"] * b) // (4 * B))
        if case["kind"] == "evict":
            one = n * (4 * D + 4)
        else:
            one = n // GROUP * (2 * GROUP * D * case["bits"] // 8 + 4 * D + 16 * GROUP) + n % GROUP * 4 * D + 4 * n
        live += K * (case["layers"] * (hkv * one + 4) + per_seq)
    # every beam is written; a parent is read once, however many follow it
    # (independent choices leave 1 - (1 - 1/K)^K of the beams as parents)
    return {"bytes": live * (1.0 + 1.0 - (1.0 - 1.0 / K) ** K), "flops": 0.0}


# -------------------------------------------------------------- 64 bits

def _exact_linear(case, s):
    B, hq, hkv, T = case["batch"], case["hq"], case["hkv"], case["tokens"]
    gamma = torch.exp(torch.tensor(s["log_decay"], dtype=torch.float64, device=DEV)).repeat(B)[:, None, None]
    state = torch.zeros((B * hkv, D, D), dtype=torch.float64, device=DEV)
    if s["state"] is not None:
        state += s["state"].double().view(B * hkv, D, D)
    out = torch.zeros((T, B * hkv, hq // hkv, D), dtype=torch.float64, device=DEV)
    alive = torch.tensor(s["lengths"], device=DEV).repeat_interleave(hkv)
    end = torch.zeros_like(state)
    end[alive == 0] = state[alive == 0]
    ends = set(s["lengths"])
    at = {name: s[name].permute(2, 0, 1, 3).contiguous().view(T, B * hkv, -1, D) for name in ("q", "k", "v")}
    for t in range(max(s["lengths"])):
        # S_t = gamma S_{t-1} + k_t v_t^T, o_t = q_t S_t / sqrt(D)
        state.mul_(gamma).baddbmm_(at["k"][t].double().transpose(1, 2), at["v"][t].double())
        torch.bmm(at["q"][t].double(), state, out=out[t])
        if t + 1 in ends:
            end[alive == t + 1] = state[alive == t + 1]
    out = out.view(T, B, hkv, hq // hkv, D).permute(1, 2, 3, 0, 4).reshape(B, hq, T, D) / math.sqrt(D)
    for b, m in enumerate(s["lengths"]):
        out[b, :, m:] = 0.0
    return {"out": out, "state": end.view(B, hkv, D, D)}


def _exact_beam(case, s):
    x = s["logits"].double()
    for b in range(x.shape[0] if s["finished"] is not None else 0):
        for j in range(x.shape[1]):
            if bool(s["finished"][b, j]):
                x[b, j] = -math.inf
                x[b, j, s["eos"]] = 0.0
    total = s["scores"].double()[..., None] + torch.log_softmax(x, dim=-1)
    best = torch.topk(total.reshape(x.shape[0], -1), s["n"], dim=-1).values
    return {"scores": best, "parent": None, "token": None, "finished": None}


def _exact_reorder(case, s):
    out = {}
    for i, x in enumerate(s["states"]):
        y = torch.empty_like(x, dtype=torch.float64)
        for b in range(case["batch"]):
            for j in range(case["beams"]):
                y[b * case["beams"] + j] = x[b * case["beams"] + int(s["parent"][b, j])]
        out["state%d" % i] = y
    for i, layer in enumerate(s["layers"]):
        out["n%d" % i] = None
        for name, x in layer["arrays"].items():
            out["%s%d" % (name, i)] = None
            if x.dtype == torch.bfloat16:
                rows = [x[b * case["beams"] + int(s["parent"][b, j])] for b in range(case["batch"])
                        for j in range(case["beams"])]
                out["%s%d" % (name, i)] = torch.stack(rows).double().reshape(-1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "beam": _exact_beam, "reorder": _exact_reorder}[case["op"]](case, s)
