"""What a prompt passes between the products of a decoder layer, and what it is scored by, as cases that can be measured.

A case is a dict of plain values; its `kind` says which operator one pass runs:

  chunk      attention of packed chunks of new tokens over a paged cache (`chunk_attention`): sequence b has n_b new tokens behind those
             that its pages hold already, each of which sees the tokens up to itself (the last `window` of them where there is a window)
  residual   behind a block (`residual_norm`): the norm of its output, its gate, the residual's sum, and the next block's norm, in one pass
  gated      inside a block (`gated_norm`): activation of the gate, product, norm ahead of the block's last product
  logprobs   of logits (`token_logprobs`): log probability of a given token, entropy, and the most probable tokens

`own` is set by whoever measures: False runs the plain forms below, True the calls of the binding.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def _chunk(name, news, olds, Hq, Hk, D, src, dst, page, window=0):
    """news, olds: new tokens of the sequences and the tokens ahead of them, as texts (a case holds plain values)."""
    return {"name": name, "kind": "chunk", "news": " ".join(map(str, news)), "olds": " ".join(map(str, olds)), "Hq": Hq, "Hk": Hk, "D": D, "src": src,
            "dst": dst, "page": page, "window": window}


def _residual(name, N, K, src, res, dst, norm=True, gate="none", activation="none", scale=1.0, following=True):
    return {"name": name, "kind": "residual", "N": N, "K": K, "src": src, "res": res, "dst": dst, "norm": norm, "gate": gate, "activation": activation,
            "scale": scale, "following": following}


def _gated(name, N, K, src, dst, activation="silu", norm=True):
    return {"name": name, "kind": "gated", "N": N, "K": K, "src": src, "dst": dst, "activation": activation, "norm": norm}


def _logprobs(name, N, V, src, top, temperature=1.0, masked=False):
    return {"name": name, "kind": "logprobs", "N": N, "V": V, "src": src, "top": top, "temperature": temperature, "masked": masked}


def listed():
    # Head layouts and features: 20 / 5 heads of 128 and 2560 / 6912 features of the 2.4B-style layer, 32 / 8 of 128 and 4096 of the 8B shapes, 32 of 100 and
    # 8640 of the 3B shapes.
    return [
        # one new token of one sequence: latency of a call
        _chunk("chunk_one", [1], [500], 20, 5, 128, "bf16", "f32", 16),
        # a decoding step of 64 sequences of unequal lengths
        _chunk("chunk_decode", [1] * 64, [4095 - (i * 2557) % 2048 for i in range(64)], 32, 8, 128, "bf16", "bf16", 64),
        # what a server has in one step: two chunks of prompts, a short prompt from its start, drafts, single tokens; a model of windows, heads of 100 features
        _chunk("chunk_mixed", [509, 333, 67, 5, 4] + [1] * 11, [1500, 800, 0, 700, 1291] + [1990 - 173 * i for i in range(11)], 32, 32, 100, "f16", "f16", 32, 1024),
        # a prompt in one piece
        _chunk("chunk_prompt", [4096], [0], 20, 5, 128, "bf16", "bf16", 64),
        # a chunk of a long prompt
        _chunk("chunk_behind", [1024], [16384], 32, 8, 128, "bf16", "bf16", 64),
        # one decoded token behind a block
        _residual("residual_one", 1, 2560, "f32", "f32", "f32", norm=False),
        # a long prompt: norms on both sides of the block, a gate for every feature, the residual stream in 16 bits
        _residual("residual_prompt", 4096, 4096, "bf16", "bf16", "bf16", gate="features", scale=0.5),
        # a short prompt, 16-bit projections, no norm
        _gated("gated_odd", 77, 8640, "f16", "f16", norm=False),
        # the stacked gate|up projection of a prompt as the product gives it, to the next product
        _gated("gated_prompt", 1024, 6912, "f32", "f32", activation="relu2"),
        # one sampled token with its alternatives
        _logprobs("logprobs_one", 1, 128000, "f32", 20, temperature=0.7),
        # a decoding step: an odd vocabulary, a part of which is not allowed
        _logprobs("logprobs_odd", 33, 50001, "bf16", 5, masked=True),
        # a prompt that is scored
        _logprobs("logprobs_prompt", 2048, 32000, "f32", 1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["chunk", "chunk", "chunk", "residual", "gated", "logprobs"])
    src = rng.choice(["f32", "bf16", "f16"])
    if kind == "chunk":
        Hq, Hk, D = rng.choice([(20, 5, 128), (32, 8, 128), (32, 32, 100), (16, 2, 64), (8, 1, 256), (12, 4, 96)])
        src = rng.choice(["bf16", "f16"])
        B = _log_int(rng, 1, 64)
        what = rng.choice(["decode", "prompt", "mixed"])
        most = {"decode": 1, "prompt": 4096 // B, "mixed": 1024 // B + 1}[what]
        news, olds = [], []
        for i in range(B):
            n = _log_int(rng, 1, most) if what != "mixed" or i % 3 == 0 else rng.randint(1, 5)
            old = rng.choice([0, _log_int(rng, 1, 16384)]) if n > 1 else _log_int(rng, 1, 16384)
            # the largest listed ones' products and keys are the most that there are, and what the plain form holds of scores is bounded
            old = min(old, 8 * 16384 * 128 * 8 // (B * D * Hk), 1024 * 16384 * 32 * 128 // (B * n * Hq * D))
            news.append(n)
            olds.append(old)
        longest, deepest = max(news), max(n + o for n, o in zip(news, olds))
        room = 1024 * 17408 * 32 // (B * longest * Hq)
        if deepest > room:
            olds = [min(o, max(0, room - n)) for n, o in zip(news, olds)]
        return _chunk("", news, olds, Hq, Hk, D, src, rng.choice([src, src, "f32"]), rng.choice([8, 16, 32, 64, 128]), rng.choice([0, 0, 0, _log_int(rng, 16, 4096)]))
    if kind == "logprobs":
        V = _log_int(rng, 500, 256000)
        N = min(_log_int(rng, 1, 2048), 2048 * 32000 // V)
        return _logprobs("", N, V, src, rng.choice([0, 1, 5, 20, 64]), rng.choice([1.0, 1.0, 0.7, 1.3]), rng.random() < 0.3)
    K = rng.choice([2048, 2560, 3200, 4096, 6912, 8192, 8640, 14336, _log_int(rng, 33, 14336)])
    N = min(_log_int(rng, 1, 4096), 4096 * 4096 // K)
    if kind == "gated":
        return _gated("", N, K, src, rng.choice([src, "f32", "bf16"]), rng.choice(["silu", "relu2", "gelu", "sigmoid"]), rng.random() < 0.6)
    gate = rng.choice(["none", "none", "features", "tokens"])
    return _residual("", N, K, src, rng.choice([src, "f32"]), rng.choice([src, "f32"]), rng.random() < 0.5, gate,
                     rng.choice(["none", "sigmoid"]) if gate != "none" else "none", rng.choice([1.0, 0.5, 0.25]), rng.random() < 0.8)


def _numbers(text):
    return [int(x) for x in text.split()]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape, dtype=torch.float32: torch.randn(shape, generator=gen, device="cuda").to(dtype)  # noqa: E731
    state = dict(case)
    src = TYPES[case["src"]]
    if case["kind"] == "chunk":
        news, olds, Hq, Hk, D, page = _numbers(case["news"]), _numbers(case["olds"]), case["Hq"], case["Hk"], case["D"], case["page"]
        lens = [n + o for n, o in zip(news, olds)]
        B, width = len(news), -(-max(lens) // page)
        state["q"] = normal(sum(news), Hq, D, dtype=src)
        state["k_cache"], state["v_cache"] = (torch.randn((B * width, Hk, page, D), generator=gen, device="cuda", dtype=src) for _ in "kv")
        state["page_table"] = torch.randperm(B * width, generator=gen, device="cuda").to(torch.int32).reshape(B, width)
        state["query_starts"] = torch.tensor([sum(news[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda")
        state["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        state["max_len"], state["max_queries"] = max(lens), max(news)
        return state
    N = case["N"]
    if case["kind"] == "logprobs":
        V = case["V"]
        # a few likely tokens over a flat tail
        logits = normal(N, V) * 2.0
        logits.scatter_(1, torch.randint(0, V, (N, 8), generator=gen, device="cuda"), normal(N, 8) * 2.0 + 12.0)
        if case["masked"]:
            logits[:, torch.randperm(V, generator=gen, device="cuda")[:V // 3]] = -math.inf
        state["logits"] = logits.to(src)
        state["tokens"] = torch.randint(0, V, (N,), generator=gen, device="cuda")
        return state
    K = case["K"]
    weight = lambda: 1.0 + 0.1 * normal(K)  # noqa: E731
    state["weight"] = weight() if case["norm"] else None
    if case["kind"] == "gated":
        state["gate"], state["x"] = normal(N, 2 * K, dtype=src).split(K, dim=1)         # views of the stacked projection's rows
        return state
    state["y"] = normal(N, K, dtype=src)
    state["residual"] = (3.0 * normal(N, K)).to(TYPES[case["res"]])
    state["gate"] = {"none": lambda: None, "features": weight, "tokens": lambda: normal(N, K, dtype=src)}[case["gate"]]()
    state["next_weight"] = weight() if case["following"] else None
    return state


# ---- plain forms: 32 bits throughout, one rounding at the end
def _plain_chunk(state):
    Hq, Hk, D, n = state["Hq"], state["Hk"], state["D"], state["max_queries"]
    G, starts, lens = Hq // Hk, state["query_starts"].long(), state["lens"].long()
    B = lens.numel()
    news = starts[1:] - starts[:-1]
    j = torch.arange(n, device="cuda")
    real = j < news[:, None]                                                                            # [B][n]
    at = torch.where(real, starts[:-1, None] + j, 0)
    q = state["q"][at].float().reshape(B, n, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, n * G, D) * (1.0 / math.sqrt(D))
    k, v = (c[state["page_table"].long()].transpose(1, 2).reshape(B, Hk, -1, D)[:, :, :state["max_len"]].float() for c in (state["k_cache"], state["v_cache"]))
    position = (lens - news)[:, None] + j
    t = torch.arange(state["max_len"], device="cuda")
    seen = (t <= position[:, :, None]) & real[:, :, None]
    if state["window"]:
        seen &= t > position[:, :, None] - state["window"]
    # keys behind a sequence's end are not its own
    v = torch.where((t < lens[:, None])[:, None, :, None], v, 0.0)
    s = torch.where(seen[:, None, :, None, :], (q @ k.transpose(2, 3)).reshape(B, Hk, n, G, -1), -math.inf)
    e = torch.exp(s - s.amax(-1, keepdim=True))
    o = (e.reshape(B, Hk, n * G, -1) @ v).reshape(B, Hk, n, G, D) / e.sum(-1, keepdim=True)
    return [o.permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)[real].to(TYPES[state["dst"]])]                # rows of the sequences one behind the other


def _activated(x, name):
    if name == "none":
        return x
    if name == "relu2":
        return x.clamp(min=0.0).square()
    if name == "gelu":      # by the error function
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    s = 1.0 / (1.0 + torch.exp(-x))
    return s if name == "sigmoid" else x * s


def _normed(x, weight):
    return x if weight is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight


def _plain_residual(state):
    t = _normed(state["y"].float(), state["weight"]) * state["scale"]
    if state["gate"] is not None:
        t = t * _activated(state["gate"].float(), state["activation"])
    h = state["residual"].float() + t
    return [h.to(TYPES[state["res"]])] + ([_normed(h, state["next_weight"]).to(TYPES[state["dst"]])] if state["following"] else [])


def _plain_logprobs(state):
    x = state["logits"].float()
    z = x / state["temperature"]
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    below = z - top                                 # nothing cancels in what is summed
    entropy = (torch.log(total) - torch.where(e > 0.0, e * below, 0.0).sum(-1, keepdim=True) / total)[:, 0]
    out = [(below.gather(1, state["tokens"][:, None]) - torch.log(total))[:, 0], entropy]
    if state["top"]:
        ids = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :state["top"]]
        out += [ids, below.gather(1, ids) - torch.log(total)]
    return out


def run(state):
    kind = state["kind"]
    if not own:
        if kind == "gated":
            return [_normed(_activated(state["gate"].float(), state["activation"]) * state["x"].float(), state["weight"]).to(TYPES[state["dst"]])]
        return {"chunk": _plain_chunk, "residual": _plain_residual, "logprobs": _plain_logprobs}[kind](state)
    from paper_2512_06443_amd import binding as B
    if kind == "chunk":
        return [B.chunk_attention(state["q"], state["k_cache"], state["v_cache"], state["page_table"], state["query_starts"], state["lens"],
                                  max_len=state["max_len"], max_queries=state["max_queries"], window=state["window"], dtype=TYPES[state["dst"]])[0]]
    if kind == "gated":
        return [B.gated_norm(state["x"], state["gate"], activation=state["activation"], weight=state["weight"], eps=EPS, dtype=TYPES[state["dst"]])]
    if kind == "residual":
        h, x = B.residual_norm(state["y"], state["residual"], weight=state["weight"], gate=state["gate"], activation=state["activation"],
                               scale=state["scale"], next_weight=state["next_weight"], eps=EPS, dtype=TYPES[state["dst"]])
        return [h] if x is None else [h, x]
    logprob, entropy, ids, logprobs = B.token_logprobs(state["logits"], state["tokens"], top=state["top"], temperature=state["temperature"])
    return [logprob, entropy] + ([ids, logprobs] if state["top"] else [])


def work(case):
    """Bytes and operations of one pass.  Attention: every sequence's keys and values that any of its new tokens sees, queries and outputs; two
    products of D multiply-adds per query head and seen token.  The others: inputs and outputs."""
    src = SIZE[case["src"]]
    if case["kind"] == "chunk":
        news, olds, Hq, Hk, D, window = _numbers(case["news"]), _numbers(case["olds"]), case["Hq"], case["Hk"], case["D"], case["window"]
        keys = pairs = 0
        for n, o in zip(news, olds):
            first = max(0, o + 1 - window) if window else 0
            keys += n + o - first
            whole = n * o + n * (n + 1) // 2
            # a query at position p is without p + 1 - window of them
            missing = sum(range(max(0, o + 1 - window), n + o + 1 - window)) if window and n + o > window else 0
            pairs += whole - missing
        tables = 4 * (sum(-(-(n + o) // case["page"]) for n, o in zip(news, olds)) + 2 * len(news) + 1)
        return {"bytes": 2 * keys * Hk * D * src + sum(news) * Hq * D * (src + SIZE[case["dst"]]) + tables, "flops": 4 * pairs * Hq * D}
    N = case["N"]
    if case["kind"] == "logprobs":
        V, top = case["V"], case["top"]
        return {"bytes": N * (V * src + 8 + 8 + top * 12), "flops": 5 * N * V}
    K, dst = case["K"], SIZE[case["dst"]]
    if case["kind"] == "gated":
        return {"bytes": N * K * (2 * src + dst) + 4 * K * case["norm"], "flops": 8 * N * K}
    rows = src + 2 * SIZE[case["res"]] + (dst if case["following"] else 0) + (src if case["gate"] == "tokens" else 0)
    return {"bytes": N * K * rows + 4 * K * (case["norm"] + case["following"] + (case["gate"] == "features")), "flops": 10 * N * K}


# ---- the definitions in 64 bits
def _exact_chunk(state):
    Hq, Hk, D, page = state["Hq"], state["Hk"], state["D"], state["page"]
    news, olds = _numbers(state["news"]), _numbers(state["olds"])
    out = torch.zeros((sum(news), Hq, D), dtype=torch.float64, device="cuda")
    row = 0
    for b, (n, old) in enumerate(zip(news, olds)):
        m = n + old
        pages = state["page_table"][b, :-(-m // page)].long()
        distance = torch.arange(old, m, device="cuda")[:, None] - torch.arange(m, device="cuda")[None, :]
        hidden = distance < 0
        if state["window"]:
            hidden |= distance >= state["window"]
        for h in range(Hk):
            k, v = (c[pages, h].reshape(-1, D)[:m].double() for c in (state["k_cache"], state["v_cache"]))
            for g in range(h * Hq // Hk, (h + 1) * Hq // Hk):
                s = (state["q"][row:row + n, g].double() @ k.t()) / math.sqrt(D)
                out[row:row + n, g] = torch.softmax(s.masked_fill(hidden, -math.inf), dim=-1) @ v
        row += n
    return [out]


def _exact_gate(x, name):
    x = x.double()
    functions = {"none": lambda: x, "relu2": lambda: torch.relu(x) ** 2, "sigmoid": lambda: torch.sigmoid(x), "silu": lambda: x * torch.sigmoid(x),
                 "gelu": lambda: x * torch.special.ndtr(x)}
    return functions[name]()


def _exact_norm(x, weight):
    return x if weight is None else x * weight.double() / torch.sqrt((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS)


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "chunk":
        return _exact_chunk(state)
    if case["kind"] == "gated":
        return [_exact_norm(_exact_gate(state["gate"], case["activation"]) * state["x"].double(), state["weight"])]
    if case["kind"] == "residual":
        t = _exact_norm(state["y"].double(), state["weight"])
        if state["gate"] is not None:
            t = t * _exact_gate(state["gate"], case["activation"])
        h = state["residual"].double() + case["scale"] * t
        return [h] + ([_exact_norm(h, state["next_weight"])] if case["following"] else [])
    logprob, entropy, probable = [], [], []
    for rows, tokens in zip(state["logits"].split(256), state["tokens"].split(256)):
        every = torch.log_softmax(rows.double() / case["temperature"], dim=-1)
        logprob.append(every.gather(1, tokens[:, None])[:, 0])
        entropy.append(torch.special.entr(torch.exp(every)).sum(-1))
        probable.append(torch.topk(every, case["top"], dim=-1).values)
    out = [torch.cat(logprob), torch.cat(entropy)]
    return out + ([None, torch.cat(probable)] if case["top"] else [])
