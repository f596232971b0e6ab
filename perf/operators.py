"""What the operators around the paged key-value cache cost: rotary positions, writing the cache, reading pages back,
and attention over the whole cache.

Four operators, each with its plain form in elementary torch operations:

  rope     rotary positions of queries and keys (half or interleaved pairs, part of the head, scaled for long contexts)
  append   new keys and values written into the pages of a cache (rounded, or quantised to e4m3 with one power-of-two
           scale per token and head), with the rotation of queries and keys in the same pass; the pages are then read back
  read     chosen pages of a cache, per request and KV head, brought into attention layout
  attn     attention of one or a few new tokens over every token of a paged cache

A page holds `page` tokens of one KV head. 16-bit caches: K [page][dim], V [page][dim]. e4m3 caches: the codes of K, the
codes of V, one exponent byte per token for K, the same for V; a value is code * 2^(byte - 127), and the byte is the
smallest with which the row's largest magnitude is at most 448.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
FAR = 1 << 20                      # the longest context, in tokens


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decode step of a batch of 8: queries and keys of one layer, slices of one projection's output
        dict(name="rope_step_b8", op="rope", tokens=8, heads=32, kv_heads=8, dim=128, rot=128, layout="half", type="bf16",
             scaling="none", far=32768, backward=False),
        # a prompt of 32K tokens with frequencies stretched by parts for a long context
        dict(name="rope_prompt_32k", op="rope", tokens=32768, heads=32, kv_heads=8, dim=128, rot=128, layout="half",
             type="bf16", scaling="parts", far=131072, backward=False),
        # the gradient of a ragged training batch, interleaved pairs on half of the head
        dict(name="rope_grad_odd", op="rope", tokens=5003, heads=32, kv_heads=8, dim=128, rot=64, layout="interleaved",
             type="fp16", scaling="ntk", far=FAR, backward=True),
        # one decode step of a batch of 8: queries and keys turned, the new entries quantised into their pages
        dict(name="append_step_b8", op="append", requests=8, tokens=1, start=32767, heads=32, kv_heads=8, dim=128, page=16,
             cache="e4m3", type="bf16", rope=True, pad=0),
        # eight prompts of 4096 tokens written into a quantised cache
        dict(name="append_prompt_8x4k", op="append", requests=8, tokens=4096, start=0, heads=32, kv_heads=8, dim=128,
             page=16, cache="e4m3", type="bf16", rope=True, pad=0),
        # ragged chunks of prompts that go on in the middle of a page, padded to a fixed number of tokens; 16-bit pages
        dict(name="append_chunks_odd", op="append", requests=5, tokens=613, start=1003, heads=32, kv_heads=8, dim=128,
             page=16, cache="same", type="bf16", rope=False, pad=37),
        # the selected pages of a batch of 8 at 32K context, budget 2048, from a quantised cache on the device
        dict(name="read_b8_32k", op="read", requests=8, kv_heads=8, dim=128, page=16, pages=2048, picked=128, cache="e4m3",
             type="bf16", host=False),
        # the same kind of set from a quantised cache in page-locked host memory
        dict(name="read_host_b8", op="read", requests=8, kv_heads=8, dim=128, page=16, pages=512, picked=64, cache="e4m3",
             type="bf16", host=True),
        # one short request, latency alone
        dict(name="attn_b1_4k", op="attn", requests=1, ctx=4096, ragged=False, tokens=1, heads=32, kv_heads=8, dim=128,
             page=16, cache="same", type="bf16", window=0),
        # a batch of 8 at 32K context, 16-bit pages, output token and speculated token together
        dict(name="attn_b8_32k", op="attn", requests=8, ctx=32768, ragged=False, tokens=2, heads=32, kv_heads=8, dim=128,
             page=16, cache="same", type="bf16", window=0),
        # a ragged batch of short and long requests, quantised pages
        dict(name="attn_ragged_b48", op="attn", requests=48, ctx=32768, ragged=True, tokens=1, heads=32, kv_heads=8,
             dim=128, page=16, cache="e4m3", type="bf16", window=0),
        # one request of a million tokens, quantised pages
        dict(name="attn_b1_1m", op="attn", requests=1, ctx=FAR, ragged=False, tokens=1, heads=32, kv_heads=8, dim=128,
             page=16, cache="e4m3", type="bf16", window=0),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "read", "attn", "attn"])
    dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    kind = rng.choice(["bf16", "bf16", "fp16"])
    cache = rng.choice(["same", "e4m3"])
    page = rng.choice([16, 16, 32, 64])
    if op == "rope":
        return dict(op=op, tokens=_log(rng, 1, 32768), heads=kv_heads * rng.choice([1, 2, 4]), kv_heads=kv_heads, dim=dim,
                    rot=rng.choice([dim, dim // 2, dim // 4]), layout=rng.choice(["half", "interleaved"]), type=kind,
                    scaling=rng.choice(["none", "linear", "ntk", "parts"]), far=_log(rng, 64, FAR),
                    backward=rng.random() < 0.3)
    if op == "append":
        requests = _log(rng, 1, 64)
        return dict(op=op, requests=requests, tokens=_log(rng, 1, 32768 // requests), start=_log(rng, 1, 4096) - 1,
                    heads=kv_heads * rng.choice([1, 2, 4]), kv_heads=kv_heads, dim=dim, page=page, cache=cache, type=kind,
                    rope=rng.random() < 0.6, pad=rng.choice([0, 0, rng.randint(1, 50)]))
    if op == "read":
        requests, pages = _log(rng, 1, 16), _log(rng, 8, 512)
        return dict(op=op, requests=requests, kv_heads=kv_heads, dim=dim, page=page, pages=pages,
                    picked=_log(rng, 1, min(pages, 128)), cache=cache, type=kind, host=rng.random() < 0.2)
    requests = _log(rng, 1, 64)
    return dict(op=op, requests=requests, ctx=_log(rng, 1, 262144 // requests), ragged=rng.random() < 0.6,
                tokens=rng.choice([1, 1, 2, 3]), heads=kv_heads * rng.choice([1, 2, 4, 5, 8]), kv_heads=kv_heads, dim=dim,
                page=page, cache=cache, type=kind, window=rng.choice([0, 0, 0, _log(rng, 16, 4096)]))


# ------------------------------------------------------------------------------------------------ sizes
def _page_bytes(c):
    e = 1 if c["cache"] == "e4m3" else 2
    return 2 * c["page"] * c["dim"] * e + (2 * c["page"] if e == 1 else 0)


def _new_tokens(c):
    """Tokens that each request of an append brings: all alike, or ragged where the call is padded."""
    if not c["pad"]:
        return [c["tokens"]] * c["requests"]
    r = random.Random(c["tokens"] * 131 + c["requests"])
    return [r.randint(1, c["tokens"]) for _ in range(c["requests"])]


def _lens(c):
    """Context length of every request of an attention case: all alike, or from empty to the longest."""
    if not c["ragged"]:
        return [c["ctx"]] * c["requests"]
    r = random.Random(c["ctx"] * 131 + c["requests"])
    lens = [_log(r, 1, c["ctx"] + 1) - 1 for _ in range(c["requests"])]
    lens[0] = c["ctx"]
    return lens


def _seen(c):
    """Tokens that any query token of a request sees, summed over the requests, and the pairs of query token and seen token."""
    read = pairs = 0
    for n in _lens(c):
        span = [(max(0, p + 1 - c["window"]) if c["window"] else 0, p + 1) for p in range(n - c["tokens"], n)]
        span = [s for s in span if s[1] > 0]
        pairs += sum(e - s for s, e in span)
        read += span[-1][1] - span[0][0] if span else 0
    return read, pairs


def work(c):
    d = c["dim"]
    if c["op"] == "rope":
        rows = c["tokens"] * (c["heads"] + c["kv_heads"])
        return {"bytes": 2 * rows * d * 2 + 4 * c["tokens"], "flops": 6 * rows * c["rot"] // 2}
    if c["op"] == "append":
        n, pages = sum(_new_tokens(c)), _append_pages(c) * c["requests"]
        per_token = _page_bytes(c) // c["page"]
        b = n * c["kv_heads"] * (2 * d * 2 + per_token) + (2 * n * c["heads"] * d * 2 if c["rope"] else 0) + 8 * n
        back = c["requests"] * c["kv_heads"] * pages // c["requests"] * (_page_bytes(c) + 2 * c["page"] * d * 2)
        return {"bytes": b + back, "flops": 0}
    if c["op"] == "read":
        n = c["requests"] * c["kv_heads"] * c["picked"]
        return {"bytes": n * (_page_bytes(c) + 2 * c["page"] * d * 2 + 4), "flops": 0}
    read, pairs = _seen(c)
    q = c["requests"] * c["tokens"] * c["heads"]
    return {"bytes": read * c["kv_heads"] * (_page_bytes(c) // c["page"]) + q * (2 * d * 2 + 4) + 4 * c["requests"],
            "flops": 4 * pairs * c["heads"] * d}


def _append_pages(c):
    """Pages of a request's table in an append case, and of the part that is read back."""
    first = c["start"] // c["page"]
    return (c["start"] + c["tokens"] - 1) // c["page"] + 1 - first


# ------------------------------------------------------------------------------------------------ inputs
def _turns(c, far):
    """Turns per position of every rotated pair, and the amplitude: what a model's configuration says."""
    rot = c.get("rot", c["dim"])
    i = np.arange(rot // 2, dtype=np.float64)
    base = 500000.0
    kind = c.get("scaling", "none")
    if kind == "ntk":
        base *= 8.0 ** (rot / (rot - 2))
    freq = base ** (-2.0 * i / rot)
    amplitude = 1.0
    if kind == "linear":
        freq = freq / 8.0
    if kind == "parts":                              # whole turns within the first 8192 positions: below 1 stretched, above 4 kept
        kept = np.clip((8192 * freq / (2 * np.pi) - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        freq = (1.0 - kept) * freq / 8.0 + kept * freq
        amplitude = 0.1 * math.log(8.0) + 1.0
    return freq / (2 * np.pi), amplitude


def _rope_handle(c, layout):
    from paper_2607_26475_b200 import binding as dd
    kind = c.get("scaling", "none")
    return dd.Rope(head_dim=c["dim"], rot_dim=c.get("rot", c["dim"]), base=500000.0,
                   layout=dd.DD_ROPE_HALF if layout == "half" else dd.DD_ROPE_INTERLEAVED,
                   scaling={"none": dd.DD_ROPE_NONE, "linear": dd.DD_ROPE_LINEAR, "ntk": dd.DD_ROPE_NTK,
                            "parts": dd.DD_ROPE_BY_PARTS}[kind],
                   factor=8.0, original_len=8192, low_turns=1.0, high_turns=4.0,
                   amplitude=0.1 * math.log(8.0) + 1.0 if kind == "parts" else 1.0)


def _two_to(e):
    """2^e exactly, for whole e from -127 to 127."""
    return torch.exp2(e.double()).float()


def _quantise(v):
    """Codes and exponent bytes of rows v [..., dim] (32 bits)."""
    amax = v.abs().amax(-1)
    m, x = torch.frexp(amax)                         # amax = m * 2^x, m in [1/2, 1); 448 = 0.875 * 2^9
    e = torch.where(amax > 0, (x - 8 - (m <= 0.875).to(x.dtype)).clamp(min=-127), torch.full_like(x, -127))
    return (v * _two_to(-e).unsqueeze(-1)).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _views(pages, c):
    """K and V parts of pages [..., bytes]: (values or codes [..., 2, page, dim], exponent bytes [..., 2, page] or None)."""
    if c["cache"] == "e4m3":
        n = 2 * c["page"] * c["dim"]
        return (pages[..., :n].unflatten(-1, (2, c["page"], c["dim"])), pages[..., n:].unflatten(-1, (2, c["page"])))
    return pages.view(TYPES[c["type"]]).unflatten(-1, (2, c["page"], c["dim"])), None


def _values(pages, c):
    """What pages [..., bytes] stand for, in 32 bits: [..., 2, page, dim]."""
    v, e = _views(pages, c)
    if e is None:
        return v.float()
    return v.view(torch.float8_e4m3fn).float() * _two_to(e.int() - 127).unsqueeze(-1)


def _random_pages(g, n, c, gain=1.0):
    """A pool of n pages of every KV head, filled: uint8 [n, kv_heads, bytes]."""
    H = c["kv_heads"]
    pages = torch.empty(n, H, _page_bytes(c), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (H * 2 * c["page"] * c["dim"]))
    for a in range(0, n, step):
        b = min(n, a + step)
        x = torch.randn(b - a, H, 2, c["page"], c["dim"], generator=g, device="cuda")
        x[:, :, 0] *= gain
        v, e = _views(pages[a:b], c)
        if e is None:
            v.copy_(x)
        else:
            codes, ex = _quantise(x)
            v.copy_(codes)
            e.copy_(ex)
    return pages


def _cache_handle(s, c):
    from paper_2607_26475_b200 import binding as dd
    kind = dd.DD_CACHE_E4M3 if c["cache"] == "e4m3" else {"bf16": dd.DD_CACHE_BF16, "fp16": dd.DD_CACHE_FP16}[c["type"]]
    return dd.PagedCache(s["pages"], s["table"], cache_format=kind, head_dim=c["dim"], page_tokens=c["page"])


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 17)
    kind, H, d, op = TYPES[c["type"]], c["kv_heads"], c["dim"], c["op"]
    s = {"c": c}
    if op == "rope":
        n = c["tokens"]
        x = torch.randn(n, c["heads"] + 2 * H, d, generator=g, device="cuda").to(kind)      # q, k and v of one projection
        s["q"], s["k"] = x[:, :c["heads"]], x[:, c["heads"]:c["heads"] + H]
        s["positions"] = torch.randint(0, c["far"], (n,), generator=g, device="cuda").to(torch.int32)
        s["q_out"] = torch.empty(n, c["heads"], d, dtype=kind, device="cuda")
        s["k_out"] = torch.empty(n, H, d, dtype=kind, device="cuda")
        turns, s["amplitude"] = _turns(c, c["far"])
        s["turns"] = torch.from_numpy(turns).cuda()
        if own:
            s["rope"] = _rope_handle(c, c["layout"])
        return s
    if op == "append":
        news = _new_tokens(c)
        n, first = sum(news), c["start"] // c["page"]
        M = first + _append_pages(c)
        x = torch.randn(n + c["pad"], c["heads"] + 2 * H, d, generator=g, device="cuda").to(kind)
        s["q"], s["k"], s["v"] = x[:, :c["heads"]], x[:, c["heads"]:c["heads"] + H], x[:, c["heads"] + H:]
        B = c["requests"]
        s["positions"] = torch.tensor([c["start"] + i for m in news for i in range(m)] + [-1] * c["pad"], dtype=torch.int32).cuda()
        s["requests"] = torch.tensor([b for b, m in enumerate(news) for _ in range(m)] + [0] * c["pad"], dtype=torch.int32).cuda()
        # pages before the first written one are not touched: their table entries name one page of the pool
        used = M - first
        s["pages"] = _random_pages(g, B * used + 1, c)
        table = torch.full((B, M), B * used, dtype=torch.int32, device="cuda")
        table[:, first:] = torch.randperm(B * used, generator=g, device="cuda").to(torch.int32).view(B, used)
        s["table"] = table
        s["idx"] = torch.arange(first, M, dtype=torch.int32, device="cuda").expand(B, H, used).contiguous()
        s["q_out"] = torch.zeros(n + c["pad"], c["heads"], d, dtype=kind, device="cuda")
        s["back"] = torch.empty(B, H, 2, used * c["page"], d, dtype=kind, device="cuda")
        turns, s["amplitude"] = _turns(c, FAR)
        s["turns"] = torch.from_numpy(turns).cuda()
        s["n"] = n
        if own:
            s["rope"] = _rope_handle(c, "half") if c["rope"] else None
            s["handle"] = _cache_handle(s, c)
        return s
    if op == "read":
        B, M, k = c["requests"], c["pages"], c["picked"]
        s["pages"] = _random_pages(g, B * M, c)
        if c["host"]:
            s["pages"] = s["pages"].cpu().pin_memory()
        s["table"] = torch.randperm(B * M, generator=g, device="cuda").to(torch.int32).view(B, M)
        s["idx"] = torch.rand(B, H, M, generator=g, device="cuda").argsort(-1)[..., :k].sort(-1).values.to(torch.int32)
        s["out"] = torch.empty(B, H, 2, k * c["page"], d, dtype=kind, device="cuda")
        if own:
            s["handle"] = _cache_handle(s, c)
        return s
    B, lens = c["requests"], _lens(c)
    M = max(1, -(-c["ctx"] // c["page"]))
    need = [-(-m // c["page"]) for m in lens]
    total = sum(need)
    s["pages"] = _random_pages(g, total + 1, c, gain=1.5)        # scores of a spread that a trained model's have
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, M), total, dtype=torch.int32, device="cuda")
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    s["table"] = table
    s["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    s["q"] = torch.randn(B, c["tokens"], c["heads"], d, generator=g, device="cuda").to(kind)
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(B, c["tokens"], c["heads"], dtype=torch.float32, device="cuda")
    if own:
        s["handle"] = _cache_handle(s, c)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _rotate(x, positions, turns, amplitude, layout, backward):
    """Rows x [tokens, heads, dim] turned by their positions, in 32 bits (the angles in 64)."""
    half = turns.numel()
    a = positions.double().unsqueeze(-1) * turns
    a = (a - a.floor()) * (2 * math.pi)
    cos, sin = (a.cos() * amplitude).float().unsqueeze(1), (a.sin() * amplitude).float().unsqueeze(1)
    if backward:
        sin = -sin
    x = x.float()
    head, rest = x[..., :2 * half], x[..., 2 * half:]
    u, w = (head[..., :half], head[..., half:]) if layout == "half" else (head[..., 0::2], head[..., 1::2])
    y = (u * cos - w * sin, w * cos + u * sin)
    turned = torch.cat(y, -1) if layout == "half" else torch.stack(y, -1).flatten(-2)
    return torch.cat((turned, rest), -1)


def _plain_rope(s):
    c = s["c"]
    q = _rotate(s["q"], s["positions"], s["turns"], s["amplitude"], c["layout"], c["backward"])
    k = _rotate(s["k"], s["positions"], s["turns"], s["amplitude"], c["layout"], c["backward"])
    return {"q": q.to(TYPES[c["type"]]), "k": k.to(TYPES[c["type"]])}


def _plain_read(s, idx):
    c = s["c"]
    phys = s["table"].long().unsqueeze(1).expand(-1, c["kv_heads"], -1).gather(2, idx.long())
    h = torch.arange(c["kv_heads"], device=phys.device).view(1, -1, 1)
    if not s["pages"].is_cuda:
        got = s["pages"][phys.cpu(), h.cpu()].cuda()
    else:
        got = s["pages"][phys, h]
    v = _values(got, c).transpose(2, 3)                           # [B, H, 2, picked, page, dim]
    return v.reshape(v.shape[0], v.shape[1], 2, -1, c["dim"]).to(TYPES[c["type"]])


def _plain_append(s):
    c, n = s["c"], s["n"]
    k, v, at = s["k"][:n].float(), s["v"][:n].float(), s["positions"][:n].long()
    if c["rope"]:
        k = _rotate(s["k"][:n], at, s["turns"], s["amplitude"], "half", False)
        s["q_out"][:n] = _rotate(s["q"][:n], at, s["turns"], s["amplitude"], "half", False).to(s["q_out"].dtype)
    block = s["table"][s["requests"][:n].long(), at // c["page"]].long()
    off = at % c["page"]
    held, ex = _views(s["pages"], c)
    if ex is None:
        held[block, :, 0, off], held[block, :, 1, off] = k.to(held.dtype), v.to(held.dtype)
    else:
        for_k, for_v = _quantise(k), _quantise(v)
        held[block, :, 0, off], held[block, :, 1, off] = for_k[0], for_v[0]
        ex[block, :, 0, off], ex[block, :, 1, off] = for_k[1], for_v[1]
    out = {"cache": _plain_read(s, s["idx"])}
    if c["rope"]:
        out["q"] = s["q_out"]
    return out


def _plain_attn(s):
    c = s["c"]
    B, Tq, H, d = c["requests"], c["tokens"], c["kv_heads"], c["dim"]
    G = c["heads"] // H
    kv = _values(s["pages"][s["table"].long()], c)                # [B, M, H, 2, page, dim]
    k = kv[:, :, :, 0].transpose(1, 2).reshape(B, H, -1, d)
    v = kv[:, :, :, 1].transpose(1, 2).reshape(B, H, -1, d)
    q = s["q"].float().view(B, Tq, H, G, d).transpose(1, 2).reshape(B, H, Tq * G, d)
    z = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    last = (s["lens"].view(B, 1) - Tq + torch.arange(Tq, device=q.device)).repeat_interleave(G, 1).view(B, 1, -1, 1)
    at = torch.arange(k.shape[2], device=q.device)
    seen = at <= last
    if c["window"]:
        seen = seen & (at > last - c["window"])
    z = z.masked_fill(~seen, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    v = v.masked_fill(~(at < s["lens"].view(B, 1, 1)).unsqueeze(-1), 0.0)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.view(B, H, Tq, G, d).transpose(1, 2).reshape(B, Tq, H * G, d)
    lse = (top + torch.log(total)).view(B, H, Tq, G).transpose(1, 2).reshape(B, Tq, H * G)
    return {"out": o.to(s["q"].dtype), "lse": lse}


def run(s):
    c = s["c"]
    if not own:
        return {"rope": _plain_rope, "append": _plain_append, "attn": _plain_attn,
                "read": lambda s: {"out": _plain_read(s, s["idx"])}}[c["op"]](s)
    if c["op"] == "rope":
        s["rope"].apply(s["positions"], s["q"], s["k"], s["q_out"], s["k_out"], backward=c["backward"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["op"] == "append":
        if c["rope"]:
            s["handle"].append(s["k"], s["v"], s["positions"], s["requests"], rope=s["rope"], q=s["q"], q_out=s["q_out"])
        else:
            s["handle"].append(s["k"], s["v"], s["positions"], s["requests"])
        s["handle"].read(s["idx"], s["back"])
        return {"cache": s["back"], "q": s["q_out"]} if c["rope"] else {"cache": s["back"]}
    if c["op"] == "read":
        s["handle"].read(s["idx"], s["out"])
        return {"out": s["out"]}
    s["handle"].decode_attn(s["q"], s["lens"], s["out"], s["lse"], window=c["window"])
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------------ the definition, 64 bits
def _e4m3_table():
    """What each of the 256 codes stands for."""
    v = []
    for code in range(256):
        sign, e, m = -1.0 if code & 128 else 1.0, (code >> 3) & 15, code & 7
        v.append(float("nan") if code & 127 == 127 else sign * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)))
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def _exact_page(raw, c):
    """Pages [..., bytes] -> [..., 2, page, dim] in 64 bits."""
    if c["cache"] != "e4m3":
        return raw.contiguous().view(TYPES[c["type"]]).double().unflatten(-1, (2, c["page"], c["dim"]))
    n = 2 * c["page"] * c["dim"]
    codes = _e4m3_table()[raw[..., :n].long()].unflatten(-1, (2, c["page"], c["dim"]))
    scale = torch.pow(torch.full((), 2.0, dtype=torch.float64, device="cuda"),
                      raw[..., n:].double() - 127.0).unflatten(-1, (2, c["page"]))
    return codes * scale.unsqueeze(-1)


def _exact_e4m3(x):
    """Rows x [..., dim] as a quantised cache holds them: to the nearest multiple of the step at each value's binade
    (three bits behind the leading one, no finer than 2^-9 of the row's scale), ties to the even multiple."""
    two = torch.full((), 2.0, dtype=torch.float64, device="cuda")
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0))
    e = torch.where(top > 448.0 * torch.pow(two, e), e + 1, torch.where(top <= 448.0 * torch.pow(two, e - 1), e - 1, e))
    scale = torch.pow(two, e.clamp(min=-127.0))
    y = x / scale
    step = torch.pow(two, torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * scale


def _exact_turn(x, positions, c, layout, backward):
    """The rotation as a complex product."""
    turns, amplitude = _turns(c, FAR)
    angle = 2 * math.pi * torch.remainder(positions.double().unsqueeze(-1) * torch.from_numpy(turns).cuda(), 1.0)
    turn = torch.polar(torch.full_like(angle, amplitude), -angle if backward else angle).unsqueeze(1)
    r = 2 * turns.size
    y = x.double().clone()
    if layout == "half":
        z = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * turn
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    else:
        z = torch.complex(y[..., 0:r:2].contiguous(), y[..., 1:r:2].contiguous()) * turn
        y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
    return y


def exact(c, seed):
    s = prepare(c, seed)
    H, d, T = c["kv_heads"], c["dim"], c.get("page", 0)
    if c["op"] == "rope":
        return {x: _exact_turn(s[x], s["positions"], c, c["layout"], c["backward"]) for x in ("q", "k")}
    if c["op"] in ("read", "append"):
        table, idx, raw = s["table"].cpu().long(), s["idx"].cpu().long(), s["pages"]
        B, k = idx.shape[0], idx.shape[2]
        out = torch.empty(B, H, 2, k, T, d, dtype=torch.float64, device="cuda")
        for b in range(B):
            for h in range(H):
                out[b, h] = _exact_page(raw[table[b][idx[b, h]].to(raw.device), h].cuda(), c).transpose(0, 1)
        out = out.view(B, H, 2, k * T, d)
        if c["op"] == "read":
            return {"out": out}
        n, first = s["n"], c["start"] // T * T
        k64 = _exact_turn(s["k"][:n], s["positions"][:n], c, "half", False) if c["rope"] else s["k"][:n].double()
        v64 = s["v"][:n].double()
        if c["cache"] == "e4m3":
            k64, v64 = _exact_e4m3(k64), _exact_e4m3(v64)
        at = 0
        for b, m in enumerate(_new_tokens(c)):
            a = c["start"] - first
            out[b, :, 0, a:a + m], out[b, :, 1, a:a + m] = k64[at:at + m].transpose(0, 1), v64[at:at + m].transpose(0, 1)
            at += m
        if not c["rope"]:
            return {"cache": out}
        q = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        q[:n] = _exact_turn(s["q"][:n], s["positions"][:n], c, "half", False)
        return {"cache": out, "q": q}
    B, Tq, G = c["requests"], c["tokens"], c["heads"] // H
    out = torch.zeros(B, Tq, c["heads"], d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, Tq, c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lens(c)):
        if n == 0:
            continue
        blocks = s["table"][b, :-(-n // T)].long()
        for h in range(H):
            kv = _exact_page(s["pages"][blocks, h], c).transpose(0, 1).reshape(2, -1, d)
            for t in range(Tq):
                end = n - Tq + t + 1
                begin = max(0, end - c["window"]) if c["window"] else 0
                if end <= 0:
                    continue
                z = s["q"][b, t, h * G:(h + 1) * G].double() @ kv[0, begin:end].T / math.sqrt(d)
                out[b, t, h * G:(h + 1) * G] = torch.softmax(z, -1) @ kv[1, begin:end]
                lse[b, t, h * G:(h + 1) * G] = torch.logsumexp(z, -1)
    return {"out": out, "lse": lse}
