"""Attention over a paged cache whose sequences share a prefix, and what stands before it, as cases that can be measured.

Three operators lie between the stacked q|k|v projection of a decoder layer and its output projection.  A case is a dict of
plain values; its `kind` says which operator one pass runs:

  norm_rope   RMS norm of every query and key head, then the rotation by the token's position, in one pass
              (`norm_rope`): fp32 views of the stacked projection (or fp16 / bf16 tensors) to the type that is stored
  append      keys (normed and rotated on the way) and values to the slots of a paged cache, the queries alongside where the
              program hands them over (`append_kv`); tokens without a slot (padding) are left out
  attention   a batch whose sequences share a prefix: every query sees the whole prefix and its own sequence's tokens up to
              itself (`shared_prefix_attention`); `n` queries per sequence (1: decoding, more: drafts that are verified)

`own` is set by whoever measures: False runs the plain forms below, True the calls of the binding.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
BASE = 500000.0             # of the rotation's frequencies
POSITIONS = 40960           # rows of the tables of cosines and sines that a program keeps


def _norm_rope(name, N, Hq, Hk, D, R, src, dst, norm=True, interleaved=False):
    return {"name": name, "kind": "norm_rope", "N": N, "Hq": Hq, "Hk": Hk, "D": D, "R": R, "src": src, "dst": dst, "norm": norm,
            "interleaved": interleaved}


def _append(name, N, Hq, Hk, D, R, src, dst, page, norm=True, interleaved=False, skip=0, token_major=False):
    return {"name": name, "kind": "append", "N": N, "Hq": Hq, "Hk": Hk, "D": D, "R": R, "src": src, "dst": dst, "page": page,
            "norm": norm, "interleaved": interleaved, "skip": skip, "token_major": token_major}


def _attention(name, B, n, Hq, Hk, D, P, S, src, dst, page, ragged=False, token_major=False):
    return {"name": name, "kind": "attention", "B": B, "n": n, "Hq": Hq, "Hk": Hk, "D": D, "P": P, "S": S, "src": src, "dst": dst,
            "page": page, "ragged": ragged, "token_major": token_major}


def listed():
    # Head layouts: 20 / 5 heads of 128 are the 2560 | 640 | 640 rows of the 2.4B-style layer, 32 / 8 of 128 fit the 8B shapes,
    # 32 of 100 the 3200 features of the 3B shapes.
    return [
        # one decoded token of one sequence: latency of a call
        _norm_rope("norm_rope_one", 1, 20, 5, 128, 128, "f32", "bf16"),
        # odd sizes: a short prompt, heads of 100 features, pairs of neighbouring features
        _norm_rope("norm_rope_odd", 77, 32, 32, 100, 100, "f32", "f16", interleaved=True),
        # a long prompt in one piece
        _norm_rope("norm_rope_prompt", 4096, 32, 8, 128, 128, "f32", "bf16"),
        # a decoding step of 64 sequences, queries in the same call
        _append("append_decode", 64, 20, 5, 128, 128, "f32", "bf16", 16),
        # several prompts padded to one length: every tenth token has no slot; no norms, a rotation of 52 of 100 features, 16-bit inputs
        _append("append_padded", 333, 0, 32, 100, 52, "f16", "f16", 16, norm=False, skip=10, token_major=True),
        # a long prompt
        _append("append_prompt", 4096, 0, 8, 128, 128, "f32", "bf16", 64),
        # one sequence after a short system prompt: the smallest call
        _attention("attention_one", 1, 1, 20, 5, 128, 512, 40, "bf16", "f32", 16),
        # sixteen short answers on one document
        _attention("attention_16", 16, 1, 20, 5, 128, 2048, 256, "bf16", "f32", 16),
        # drafts of up to five tokens that are verified at once, heads of 100 features without sharing, odd lengths
        _attention("attention_drafts", 24, 5, 32, 32, 100, 1500, 300, "f16", "f16", 32, ragged=True, token_major=True),
        # few sequences whose own part is the longer one
        _attention("attention_own_long", 8, 1, 32, 8, 128, 1000, 16384, "bf16", "bf16", 64),
        # many samples of one long context
        _attention("attention_64_long", 64, 1, 32, 8, 128, 32768, 512, "bf16", "bf16", 64),
        # a large batch under one prompt, output as the next projection takes it
        _attention("attention_256", 256, 1, 32, 8, 128, 8192, 128, "bf16", "f32", 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm_rope", "append", "attention", "attention"])
    Hq, Hk, D = rng.choice([(20, 5, 128), (32, 8, 128), (32, 32, 100), (16, 2, 64), (8, 1, 256), (12, 4, 96)])
    dst = rng.choice(["bf16", "f16"])
    if kind == "attention":
        B, n, page = _log_int(rng, 1, 256), rng.choice([1, 1, 1, 2, 5, 8]), rng.choice([8, 16, 32, 64, 128])
        P = rng.choice([0, _log_int(rng, 1, 32768), _log_int(rng, 128, 32768)])
        S = _log_int(rng, n, 16384)
        # no case above the work of the largest listed ones: products of the prefix, bytes of the sequences' own tokens
        P = min(P, 256 * 8192 * 32 * 128 // (B * n * Hq * D))
        S = max(n, min(S, 8 * 16384 * 8 * 128 // (B * Hk * D)))
        return _attention("", B, n, Hq, Hk, D, P, S, dst, rng.choice([dst, "f32"]), page, ragged=n > 1 and rng.random() < 0.5,
                          token_major=rng.random() < 0.3)
    N = min(_log_int(rng, 1, 4096), 4096 * 40 * 128 // ((Hq + Hk) * D))
    R = rng.choice([D, D, D // 8 * 4])
    src, norm, interleaved = rng.choice(["f32", "f32", dst]), rng.random() < 0.7, rng.random() < 0.3
    if kind == "norm_rope":
        return _norm_rope("", N, Hq, Hk, D, R, src, rng.choice([dst, dst, "f32"]), norm, interleaved)
    return _append("", N, rng.choice([0, Hq]), Hk, D, R, src, dst, rng.choice([8, 16, 32, 64, 128]), norm, interleaved,
                   rng.choice([0, 0, 7]), rng.random() < 0.3)


def _lengths(case):
    """Own tokens and queries of each sequence of an attention case: between half and all of S, and between one and n."""
    B, S, n = case["B"], case["S"], case["n"]
    lens = [S - (i * 7919) % (S // 2 + 1) for i in range(B)]
    queries = [n - (i * 31) % n if case["ragged"] else n for i in range(B)]
    return [max(m, q) for m, q in zip(lens, queries)], queries


def _rotation(R):
    """The tables that a program keeps: cosines and sines of position times base^(-2i/R), fp32."""
    angle = torch.arange(POSITIONS, device="cuda", dtype=torch.float64)[:, None] * BASE ** (
        -torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / R)
    return angle.cos().float(), angle.sin().float()


def _cache(gen, pages, Hk, page, D, dtype, token_major):
    """[pages][heads][page][D], or the same indices over memory whose tokens lie ahead of the heads."""
    shape = (pages, page, Hk, D) if token_major else (pages, Hk, page, D)
    c = torch.randn(shape, generator=gen, device="cuda", dtype=dtype)
    return c.transpose(1, 2) if token_major else c


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    Hq, Hk, D, dst = case["Hq"], case["Hk"], case["D"], TYPES[case["dst"]]
    src = TYPES[case["src"]]
    state = dict(case)
    if case["kind"] == "attention":
        B, n, P, page = case["B"], case["n"], case["P"], case["page"]
        lens, queries = _lengths(case)
        prefix_pages, own_pages = -(-P // page), -(-max(lens) // page)
        pages = prefix_pages + B * own_pages
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        state["q"] = torch.randn((B, n, Hq, D), generator=gen, device="cuda").to(src)
        state["k_cache"] = _cache(gen, pages, Hk, page, D, src, case["token_major"])
        state["v_cache"] = _cache(gen, pages, Hk, page, D, src, case["token_major"])
        state["prefix_pages"] = order[:prefix_pages].clone()
        state["page_table"] = order[prefix_pages:].reshape(B, own_pages).clone()
        state["own_lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        state["query_lens"] = torch.tensor(queries, dtype=torch.int32, device="cuda") if case["ragged"] else None
        state["max_own"] = max(lens)
        return state
    N, R = case["N"], case["R"]
    # the stacked projection's output; queries, keys and values are views of its rows
    qkv = torch.randn((N, (Hq + 2 * Hk) * D), generator=gen, device="cuda").to(src)
    q, k, v = qkv.split([Hq * D, Hk * D, Hk * D], dim=1)
    state["q"], state["k"], state["v"] = (q.unflatten(1, (Hq, D)) if Hq else None), k.unflatten(1, (Hk, D)), v.unflatten(1, (Hk, D))
    state["cos"], state["sin"] = _rotation(R)
    state["positions"] = torch.randint(0, POSITIONS, (N,), generator=gen, device="cuda")
    weight = lambda: 1.0 + 0.1 * torch.randn(D, generator=gen, device="cuda") if case["norm"] else None  # noqa: E731
    state["q_weight"], state["k_weight"] = weight() if Hq else None, weight()
    if case["kind"] == "append":
        page = case["page"]
        pages = -(-N * 5 // 4 // page) + 1
        state["k_cache"] = _cache(gen, pages, Hk, page, D, dst, case["token_major"])
        state["v_cache"] = _cache(gen, pages, Hk, page, D, dst, case["token_major"])
        slots = torch.randperm(pages * page, generator=gen, device="cuda")[:N].contiguous()
        if case["skip"]:
            slots[::case["skip"]] = -1
        state["slots"], state["kept"] = slots, (slots >= 0).nonzero()[:, 0]
    return state


# ---- plain forms: 32 bits throughout, one rounding at the end
def _normed_rotated(x, weight, state, rows=slice(None)):
    """[N][H][D] -> the same in fp32: x / sqrt(mean(x^2) + eps) * weight, then the first R features rotated in pairs."""
    x = x[rows].float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight
    R = state["R"]
    p = state["positions"][rows]
    c, s = state["cos"][p][:, None, :], state["sin"][p][:, None, :]
    out = x.clone()
    if state["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        out[..., 0:R:2], out[..., 1:R:2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        out[..., :R // 2], out[..., R // 2:R] = a * c - b * s, b * c + a * s
    return out


def _plain_append(state):
    dst, page = TYPES[state["dst"]], state["page"]
    rows = state["kept"]
    slots = state["slots"][rows]
    at, off = slots // page, slots % page
    state["k_cache"][at, :, off] = _normed_rotated(state["k"], state["k_weight"], state, rows).to(dst)
    state["v_cache"][at, :, off] = state["v"][rows].float().to(dst)
    q = _normed_rotated(state["q"], state["q_weight"], state).to(dst) if state["Hq"] else None
    return [state["k_cache"], state["v_cache"]] + ([q] if state["Hq"] else [])


def _plain_attention(state):
    B, n, Hq, Hk, D, P = (state[x] for x in ("B", "n", "Hq", "Hk", "D", "P"))
    G = Hq // Hk
    # rows of a kv head: (query, head of its group)
    q = state["q"].float().reshape(B, n, Hk, G, D).permute(2, 0, 1, 3, 4) * (1.0 / math.sqrt(D))
    k, v = (c[state["prefix_pages"].long()].transpose(0, 1).reshape(Hk, -1, D)[:, :P].float() for c in (state["k_cache"], state["v_cache"]))
    shared = q.reshape(Hk, B * n * G, D) @ k.transpose(1, 2)                                             # [Hk][B n G][P]
    kb, vb = (c[state["page_table"].long()].transpose(1, 2).reshape(B, Hk, -1, D).float() for c in (state["k_cache"], state["v_cache"]))
    S = kb.shape[2]
    each = q.transpose(0, 1).reshape(B, Hk, n * G, D) @ kb.transpose(2, 3)                               # [B][Hk][n G][S]
    lens = state["own_lens"].long()
    queries = state["query_lens"].long() if state["query_lens"] is not None else torch.full_like(lens, n)
    j = torch.arange(n, device=lens.device)
    last = (lens - queries)[:, None] + j                                                                 # own position of query j
    real = j < queries[:, None]
    seen = torch.arange(S, device=lens.device) <= last[:, :, None]                                       # [B][n][S]
    seen = seen[:, None, :, None, :].expand(B, Hk, n, G, S).reshape(B, Hk, n * G, S)
    each = torch.where(seen, each, -math.inf)
    shared = shared.reshape(Hk, B, n * G, P).transpose(0, 1)
    both = torch.cat([shared, each], dim=-1)
    top = both.amax(-1, keepdim=True)
    e = torch.exp(both - top)
    o = (e[..., :P].transpose(0, 1).reshape(Hk, B * n * G, P) @ v).reshape(Hk, B, n * G, D).transpose(0, 1) + e[..., P:] @ vb
    o = (o / e.sum(-1, keepdim=True)).reshape(B, Hk, n, G, D).transpose(1, 2).reshape(B, n, Hq, D)
    return [torch.where(real[:, :, None, None], o, 0.0).to(TYPES[state["dst"]])]


def run(state):
    kind = state["kind"]
    if not own:
        if kind == "norm_rope":
            return [_normed_rotated(state[x], state[x + "_weight"], state).to(TYPES[state["dst"]]) for x in ("q", "k")]
        return _plain_append(state) if kind == "append" else _plain_attention(state)
    from paper_2512_06443_amd import binding as B
    if kind == "norm_rope":
        return list(B.norm_rope(state["q"], state["k"], state["positions"], state["cos"], state["sin"], state["q_weight"],
                                state["k_weight"], eps=EPS, interleaved=state["interleaved"], dtype=TYPES[state["dst"]]))
    if kind == "append":
        q = B.append_kv(state["k"], state["v"], state["slots"], state["k_cache"], state["v_cache"], state["positions"], state["cos"],
                        state["sin"], k_weight=state["k_weight"], eps=EPS, interleaved=state["interleaved"], q=state["q"],
                        q_weight=state["q_weight"])
        return [state["k_cache"], state["v_cache"]] + ([q] if state["Hq"] else [])
    out, _ = B.shared_prefix_attention(state["q"], state["k_cache"], state["v_cache"], state["prefix_pages"], state["P"],
                                       state["page_table"], state["own_lens"], query_lens=state["query_lens"],
                                       max_own_len=state["max_own"], dtype=TYPES[state["dst"]])
    return [out]


def work(case):
    """Bytes and operations of one pass.  Attention: the prefix once for the whole batch, each sequence's own tokens, queries and outputs;
    two products of D multiply-adds per query head and visible token.  The others: inputs and outputs of every head, the rotation's
    rows and the indices of every token."""
    size = {"f32": 4, "bf16": 2, "f16": 2}
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    if case["kind"] == "attention":
        lens, queries = _lengths(case)
        B, n, P, page = case["B"], case["n"], case["P"], case["page"]
        tables = 4 * (-(-P // page) + sum(-(-m // page) for m in lens) + B)
        seen = sum(q * (P + m) - q * (q - 1) // 2 for m, q in zip(lens, queries))
        return {"bytes": 2 * (P + sum(lens)) * Hk * D * size[case["src"]] + B * n * Hq * D * size[case["dst"]]
                + sum(queries) * Hq * D * size[case["src"]] + tables, "flops": 4 * seen * Hq * D}
    N, R = case["N"], case["R"]
    if case["kind"] == "norm_rope":
        heads = Hq + Hk
        return {"bytes": N * (heads * D * (size[case["src"]] + size[case["dst"]]) + 8 + 4 * R), "flops": 8 * N * heads * D}
    kept = N - (-(-N // case["skip"]) if case["skip"] else 0)
    moved = (kept * 2 * Hk + N * Hq) * D * (size[case["src"]] + size[case["dst"]])
    return {"bytes": moved + N * (16 + 4 * R), "flops": 8 * (kept * Hk + N * Hq) * D}


# ---- the definitions in 64 bits
def _exact_heads(x, weight, state):
    N, H, D = x.shape
    R = state["R"]
    x = x.double()
    if weight is not None:
        x = x * weight.double() / torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS)
    p = state["positions"]
    z = torch.complex(state["cos"].double()[p], state["sin"].double()[p])[:, None, :]
    if state["interleaved"]:
        turned = torch.view_as_real(torch.view_as_complex(x[..., :R].reshape(N, H, R // 2, 2).contiguous()) * z).reshape(N, H, R)
    else:
        w = torch.complex(x[..., :R // 2], x[..., R // 2:R]) * z
        turned = torch.cat([w.real, w.imag], dim=-1)
    return torch.cat([turned, x[..., R:]], dim=-1)


def _exact_attention(state):
    B, n, Hq, Hk, D, P, page = (state[x] for x in ("B", "n", "Hq", "Hk", "D", "P", "page"))
    lens = state["own_lens"].tolist()
    queries = state["query_lens"].tolist() if state["query_lens"] is not None else [n] * B
    out = torch.zeros((B, n, Hq, D), dtype=torch.float64, device="cuda")
    tokens = lambda cache, pages, m: torch.cat(  # noqa: E731   [Hk][m][D] of the first m tokens of these pages
        [cache[pages.long()].double().permute(1, 0, 2, 3).flatten(1, 2)[:, :m], torch.zeros((Hk, 0, D), dtype=torch.float64, device="cuda")], dim=1)
    pk, pv = tokens(state["k_cache"], state["prefix_pages"], P), tokens(state["v_cache"], state["prefix_pages"], P)
    for b in range(B):
        k = torch.cat([pk, tokens(state["k_cache"], state["page_table"][b], lens[b])], dim=1)
        v = torch.cat([pv, tokens(state["v_cache"], state["page_table"][b], lens[b])], dim=1)
        for j in range(queries[b]):
            m = P + lens[b] - queries[b] + j + 1
            q = state["q"][b, j].double().reshape(Hk, Hq // Hk, D)
            weights = torch.softmax(q @ k[:, :m].transpose(1, 2) / math.sqrt(D), dim=-1)
            out[b, j] = (weights @ v[:, :m]).reshape(Hq, D)
    return [out]


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "attention":
        return _exact_attention(state)
    if case["kind"] == "norm_rope":
        return [_exact_heads(state[x], state[x + "_weight"], state) for x in ("q", "k")]
    k, v = _exact_heads(state["k"], state["k_weight"], state), state["v"].double()
    caches = [state["k_cache"].double(), state["v_cache"].double()]
    for cache, x in zip(caches, (k, v)):
        tokens = cache.permute(0, 2, 1, 3).flatten(0, 1).clone()        # [slot][heads][D]
        tokens[state["slots"][state["kept"]]] = x[state["kept"]]
        cache.copy_(tokens.unflatten(0, (cache.shape[0], cache.shape[2])).permute(0, 2, 1, 3))
    return caches + ([_exact_heads(state["q"], state["q_weight"], state)] if case["Hq"] else [])
