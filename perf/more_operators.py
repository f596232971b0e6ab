"""What a paged key-value cache in 4 bits costs, and attention that reads only the pages chosen for each query.

Four operators, each with its plain form in elementary torch operations:

  append   new keys and values written into 4-bit pages, with the rotation of queries and keys in the same pass; the pages
           are then read back
  attn     attention of one or a few new tokens over every token of a 4-bit cache
  select   the landmarks of the pages that the newest tokens lie in brought up to date, and for every query token and KV head
           the pages with the highest scores of query and landmark
  sparse   attention of every query token over the pages listed for it, straight from the pool (4-bit, e4m3 or 16-bit pages)

Pages. 16-bit and e4m3 pages: see perf/operators.py. A 4-bit page is a run of tiles of 16 tokens of one KV head. A tile holds the
codes of K, row by row, two to a byte, the lower half first; the codes of V, [token / 8][dim / 8 parts][token % 8 / 2][token % 2]
[dim / 8 codes]; the scales of K [token][dim / 16], e4m3 codes; the scales of V [dim / 16][token]; one exponent byte per token for K,
the same for V. A value is (code - 8) * scale * 2^(byte - 127). The byte is the smallest with which the row's largest magnitude
is at most 7 * 448; a scale is that of its 16 elements over 7, rounded, and at least 2^-4.

Landmarks. The mean of a page's valid keys as 8-bit whole numbers with one power of two: [block][head][dim codes, exponent
byte + 64, 15 bytes of nothing]. A score is <codes of the summed query heads, codes of the landmark> * 2^exponent: exact in 32
bits, so the chosen set is defined to the last page.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
FAR = 1 << 20                      # the longest context, in tokens
LM_PAD = 16                        # bytes behind the codes of a landmark


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decode step of a batch of 8: queries and keys turned, the new entries quantised into their pages
        dict(name="append4_step_b8", op="append", requests=8, tokens=1, start=32767, heads=32, kv_heads=8, dim=128, page=16,
             cache="int4", type="bf16", rope=True, pad=0),
        # eight prompts of 4096 tokens written into the cache
        dict(name="append4_prompt_8x4k", op="append", requests=8, tokens=4096, start=0, heads=32, kv_heads=8, dim=128,
             page=16, cache="int4", type="bf16", rope=True, pad=0),
        # ragged chunks of prompts that go on in the middle of a page, padded to a fixed number of tokens
        dict(name="append4_chunks_odd", op="append", requests=5, tokens=613, start=1003, heads=16, kv_heads=4, dim=64,
             page=32, cache="int4", type="fp16", rope=False, pad=37),
        # one short request, latency alone
        dict(name="attn4_b1_4k", op="attn", requests=1, ctx=4096, ragged=False, tokens=1, heads=32, kv_heads=8, dim=128,
             page=16, cache="int4", type="bf16", window=0),
        # a batch of 8 at 32K context, output token and speculated token together
        dict(name="attn4_b8_32k", op="attn", requests=8, ctx=32768, ragged=False, tokens=2, heads=32, kv_heads=8, dim=128,
             page=16, cache="int4", type="bf16", window=0),
        # a ragged batch of short and long requests
        dict(name="attn4_ragged_b48", op="attn", requests=48, ctx=32768, ragged=True, tokens=1, heads=32, kv_heads=8,
             dim=128, page=16, cache="int4", type="bf16", window=0),
        # one request of a million tokens
        dict(name="attn4_b1_1m", op="attn", requests=1, ctx=FAR, ragged=False, tokens=1, heads=32, kv_heads=8, dim=128,
             page=16, cache="int4", type="bf16", window=0),
        # one decode step of a batch of 8 at 32K context: budget 2048 tokens, the first page and the last 8 always kept
        dict(name="select_step_b8", op="select", requests=8, ctx=32768, ragged=False, tokens=1, heads=32, kv_heads=8, dim=128,
             page=16, cache="int4", type="bf16", picked=128, first=1, recent=8),
        # a chunk of 2048 prompt tokens at the end of 32K, budget 1024
        dict(name="select_chunk_2k", op="select", requests=1, ctx=32768, ragged=False, tokens=2048, heads=32, kv_heads=8,
             dim=128, page=16, cache="same", type="bf16", picked=64, first=1, recent=2),
        # the attention of that decode step
        dict(name="sparse_step_b8", op="sparse", requests=8, ctx=32768, ragged=False, tokens=1, heads=32, kv_heads=8, dim=128,
             page=16, cache="int4", type="bf16", picked=128, first=1, recent=8),
        # the attention of that chunk, 16-bit pages
        dict(name="sparse_chunk_2k", op="sparse", requests=1, ctx=32768, ragged=False, tokens=2048, heads=32, kv_heads=8,
             dim=128, page=16, cache="same", type="bf16", picked=64, first=1, recent=2),
        # a ragged, padded batch of chunks, e4m3 pages of 32 tokens, a group of five query heads
        dict(name="sparse_ragged_odd", op="sparse", requests=13, ctx=5003, ragged=True, tokens=37, heads=20, kv_heads=4, dim=64,
             page=32, cache="e4m3", type="fp16", picked=24, first=0, recent=1),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "select", "sparse", "sparse"])
    dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    kind = rng.choice(["bf16", "bf16", "fp16"])
    page = rng.choice([16, 16, 32, 64])
    c = dict(op=op, heads=kv_heads * rng.choice([1, 2, 4, 5, 8]), kv_heads=kv_heads, dim=dim, page=page, cache="int4", type=kind)
    if op == "append":
        requests = _log(rng, 1, 64)
        return dict(c, heads=kv_heads * rng.choice([1, 2, 4]), requests=requests, tokens=_log(rng, 1, 32768 // requests),
                    start=_log(rng, 1, 4096) - 1, rope=rng.random() < 0.6, pad=rng.choice([0, 0, rng.randint(1, 50)]))
    if op == "attn":
        requests = _log(rng, 1, 64)
        return dict(c, requests=requests, ctx=_log(rng, 1, 262144 // requests), ragged=rng.random() < 0.6,
                    tokens=rng.choice([1, 1, 2, 3]), window=rng.choice([0, 0, 0, _log(rng, 16, 4096)]))
    requests = _log(rng, 1, 32)
    tokens = rng.choice([1, 1, 2, _log(rng, 3, 2048 // requests)])
    ctx = max(tokens, _log(rng, 16, min(262144 // requests, (1 << 26) // (requests * tokens))))
    pages = -(-ctx // page)
    picked = _log(rng, 2, max(2, min(pages, 128)))
    return dict(c, heads=kv_heads * rng.choice([1, 2, 4]), requests=requests, ctx=ctx, ragged=rng.random() < 0.6, tokens=tokens,
                cache=rng.choice(["int4", "int4", "e4m3", "same"]), picked=picked, first=rng.choice([0, 0, 1]),
                recent=rng.choice([1, 1, min(4, picked - 1)]))


# ------------------------------------------------------------------------------------------------ sizes
def _page_bytes(c):
    if c["cache"] == "int4":
        return c["page"] * c["dim"] + c["page"] // 16 * (2 * c["dim"] + 32)
    e = 1 if c["cache"] == "e4m3" else 2
    return 2 * c["page"] * c["dim"] * e + (2 * c["page"] if e == 1 else 0)


def _new_tokens(c):
    """Tokens that each request of an append brings: all alike, or ragged where the call is padded."""
    if not c["pad"]:
        return [c["tokens"]] * c["requests"]
    r = random.Random(c["tokens"] * 131 + c["requests"])
    return [r.randint(1, c["tokens"]) for _ in range(c["requests"])]


def _lens(c):
    """Context length of every request: all alike, or from empty to the longest."""
    if not c["ragged"]:
        return [c["ctx"]] * c["requests"]
    r = random.Random(c["ctx"] * 131 + c["requests"])
    lens = [_log(r, 1, c["ctx"] + 1) - 1 for _ in range(c["requests"])]
    lens[0] = c["ctx"]
    return lens


def _append_pages(c):
    """Pages of a request's table in an append case that are written (and read back)."""
    return (c["start"] + c["tokens"] - 1) // c["page"] + 1 - c["start"] // c["page"]


def work(c):
    d, H, T = c["dim"], c["kv_heads"], c["page"]
    if c["op"] == "append":
        n = sum(_new_tokens(c))
        b = n * H * (2 * d * 2 + _page_bytes(c) // T) + (2 * n * c["heads"] * d * 2 if c["rope"] else 0) + 8 * n
        back = c["requests"] * H * _append_pages(c) * (_page_bytes(c) + 2 * T * d * 2)
        return {"bytes": b + back, "flops": 0}
    spans = [[p for p in range(n - c["tokens"], n) if p >= 0] for n in _lens(c)]
    rows = sum(map(len, spans)) * c["heads"]
    if c["op"] == "attn":
        seen = [[min(p + 1, c["window"] or p + 1) for p in s] for s in spans]
        read = sum(s[-1] + 1 - max(0, s[0] + 1 - (c["window"] or s[0] + 1)) for s in spans if s)
        return {"bytes": read * H * (_page_bytes(c) // T) + rows * (2 * d * 2 + 4) + 4 * c["requests"],
                "flops": 4 * d * c["heads"] * sum(map(sum, seen))}
    pages = sum(s[-1] // T + 1 for s in spans if s)                          # visible to a request's last token
    scored = sum(p // T + 1 for s in spans for p in s)
    if c["op"] == "select":
        fresh = sum(s[-1] // T + 1 - s[0] // T for s in spans if s)
        return {"bytes": pages * H * (d + 1) + fresh * H * (_page_bytes(c) // 2 + d + 1) + rows * d * 2 + rows // c["heads"] * H * c["picked"] * 4,
                "flops": 2 * d * H * scored + rows * d}
    chosen = sum(min(c["picked"], p // T + 1) for s in spans for p in s)
    return {"bytes": min(chosen, pages) * H * _page_bytes(c) + rows * (2 * d * 2 + 4) + rows // c["heads"] * H * c["picked"] * 4,
            "flops": 4 * d * c["heads"] * chosen * T}


# ------------------------------------------------------------------------------------------------ pages
def _two_to(e):
    """2^e in 64 bits, from its bits (exp2 and pow may be off by one step on a GPU, which a tie would show)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantise4(x):
    """Rows x [..., dim] -> (codes 1 ... 15 [..., dim], scales as e4m3 codes [..., dim / 16], exponent bytes [...]). The
    seventh is taken by a tensor: a division by a number is a product with its inverse, which ties would show."""
    x = x.double() if x.dtype is torch.float64 else x.float()
    m, e = torch.frexp(x.abs().amax(-1))             # the largest = m * 2^e, m in [1/2, 1); 7 * 448 = 0.765625 * 2^12
    e = torch.where(m > 0, (e - 12 + (m > 0.765625).to(e.dtype)).clamp(min=-127), torch.full_like(e, -127))
    y = (x * _two_to(-e).to(x.dtype).unsqueeze(-1)).unflatten(-1, (-1, 16))
    top = y.abs().amax(-1)
    scale = (top / torch.full_like(top, 7.0)).clamp(min=2.0 ** -4).float().to(torch.float8_e4m3fn)
    code = torch.round(y / scale.to(x.dtype).unsqueeze(-1)).clamp(-7, 7).flatten(-2)
    return (code + 8).to(torch.uint8), scale.view(torch.uint8), (e + 127).to(torch.uint8)


def _quantise8(v):
    """Codes and exponent bytes of rows v [..., dim] of an e4m3 page (32 bits)."""
    m, x = torch.frexp(v.abs().amax(-1))             # 448 = 0.875 * 2^9
    e = torch.where(m > 0, (x - 8 - (m <= 0.875).to(x.dtype)).clamp(min=-127), torch.full_like(x, -127))
    return (v * _two_to(-e).float().unsqueeze(-1)).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _tiles(pages, c):
    """Parts of 4-bit pages [..., bytes], each with the tile in front: K rows [16, dim / 2], V [2, 8, 4, 2, dim / 16], scales of
    K [16, dim / 16], of V [dim / 16, 16], exponents [2, 16]."""
    d = c["dim"]
    t = pages.unflatten(-1, (c["page"] // 16, -1))
    return (t[..., :8 * d].unflatten(-1, (16, d // 2)), t[..., 8 * d:16 * d].unflatten(-1, (2, 8, 4, 2, d // 16)),
            t[..., 16 * d:17 * d].unflatten(-1, (16, d // 16)), t[..., 17 * d:18 * d].unflatten(-1, (d // 16, 16)),
            t[..., 18 * d:].unflatten(-1, (2, 16)))


def _pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpack(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def _views(pages, c):
    """K and V parts of 16-bit or e4m3 pages [..., bytes]: (values or codes [..., 2, page, dim], exponent bytes or None)."""
    if c["cache"] == "e4m3":
        n = 2 * c["page"] * c["dim"]
        return (pages[..., :n].unflatten(-1, (2, c["page"], c["dim"])), pages[..., n:].unflatten(-1, (2, c["page"])))
    return pages.view(TYPES[c["type"]]).unflatten(-1, (2, c["page"], c["dim"])), None


def _values(pages, c):
    """What pages [..., bytes] stand for, in 32 bits: [..., 2, page, dim]."""
    if c["cache"] != "int4":
        v, e = _views(pages, c)
        return v.float() if e is None else v.view(torch.float8_e4m3fn).float() * _two_to(e.int() - 127).float().unsqueeze(-1)
    k, v, ks, vs, ex = _tiles(pages, c)
    v = _unpack(v).movedim(-4, -2)                                # [..., 2, 4, 2, 8, dim / 8]
    codes = torch.stack((_unpack(k), v.flatten(-2).flatten(-4, -2)), -4).flatten(-3, -2)      # [..., 2, page, dim] by tiles: K and V in front
    scale = torch.stack((ks, vs.transpose(-1, -2)), -4).flatten(-3, -2).contiguous().view(torch.float8_e4m3fn).float()
    scale = scale * _two_to(ex.movedim(-2, -3).flatten(-2).int() - 127).float().unsqueeze(-1)
    return (codes.float() - 8).unflatten(-1, (-1, 16)).mul_(scale.unsqueeze(-1)).flatten(-2)


def _random_pages(g, n, c, gain=1.0):
    """A pool of n pages of every KV head, filled: uint8 [n, kv_heads, bytes]."""
    H, T, d = c["kv_heads"], c["page"], c["dim"]
    pages = torch.empty(n, H, _page_bytes(c), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (H * 2 * T * d))
    for a in range(0, n, step):
        b = min(n, a + step)
        x = torch.randn(b - a, H, 2, T, d, generator=g, device="cuda")
        x[:, :, 0] *= gain
        if c["cache"] == "int4":
            codes, scale, ex = _quantise4(x)
            k, v, ks, vs, e = _tiles(pages[a:b], c)
            k.copy_(_pack(codes[:, :, 0]).unflatten(-2, (-1, 16)))
            v.copy_(_pack(codes[:, :, 1]).unflatten(-1, (8, -1)).unflatten(-3, (-1, 2, 4, 2)).movedim(-2, -4))
            ks.copy_(scale[:, :, 0].unflatten(-2, (-1, 16)))
            vs.copy_(scale[:, :, 1].unflatten(-2, (-1, 16)).transpose(-1, -2))
            e.copy_(ex.unflatten(-1, (-1, 16)).movedim(-2, -3))
            continue
        v, e = _views(pages[a:b], c)
        if e is None:
            v.copy_(x)
        else:
            codes, ex = _quantise8(x)
            v.copy_(codes)
            e.copy_(ex)
    return pages


def _landmark(keys, valid):
    """Landmarks [..., dim + 16] of keys [..., tokens, dim]; valid [..., tokens]. The sum, the mean and its codes in 64 bits."""
    keys = torch.where(valid.unsqueeze(-1), keys.double(), torch.zeros((), dtype=torch.float64, device=keys.device))
    mean = keys.sum(-2) / valid.sum(-1, keepdim=True).clamp(min=1)
    codes, e = _whole(mean, -64)
    tail = torch.zeros(*codes.shape[:-1], LM_PAD, dtype=torch.uint8, device=codes.device)
    tail[..., 0] = (e + 64).to(torch.uint8)
    return torch.cat((codes.to(torch.int8).view(torch.uint8), tail), -1)


def _whole(x, least):
    """Rows x [..., dim] (64 bits) as whole numbers up to 127 times 2^e: (numbers in 32 bits, e)."""
    m, e = torch.frexp(x.abs().amax(-1))             # 127 = 0.9921875 * 2^7
    e = torch.where(m > 0, (e - 7 + (m > 0.9921875).to(e.dtype)).clamp(min=least), torch.full_like(e, least)).clamp(max=63)
    return torch.round(x * _two_to(-e).unsqueeze(-1)).clamp(-127, 127).float(), e


# ------------------------------------------------------------------------------------------------ inputs
def _turns(c):
    """Turns per position of every rotated pair."""
    return 500000.0 ** (-2.0 * np.arange(c["dim"] // 2, dtype=np.float64) / c["dim"]) / (2 * np.pi)


def _cache_handle(s, c):
    from paper_2607_26475_b200 import binding as dd
    kind = {"int4": getattr(dd, "DD_CACHE_INT4", None), "e4m3": dd.DD_CACHE_E4M3,
            "same": {"bf16": dd.DD_CACHE_BF16, "fp16": dd.DD_CACHE_FP16}[c["type"]]}[c["cache"]]
    return dd.PagedCache(s["pages"], s["table"], cache_format=kind, head_dim=c["dim"], page_tokens=c["page"])


def _filled(s, c, g, lens):
    """A pool that holds requests of these lengths, one page to spare, and their tables."""
    M = max(1, -(-c["ctx"] // c["page"]))
    need = [-(-m // c["page"]) for m in lens]
    total = sum(need)
    s["pages"] = _random_pages(g, total + 1, c, gain=1.5)        # scores of a spread that a trained model's have
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((c["requests"], M), total, dtype=torch.int32, device="cuda")
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    s["table"] = table
    s["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 29)
    kind, H, d, B, n = TYPES[c["type"]], c["kv_heads"], c["dim"], c["requests"], c["tokens"]
    s = {"c": c}
    if c["op"] == "append":
        news = _new_tokens(c)
        total, first = sum(news), c["start"] // c["page"]
        used = _append_pages(c)
        x = torch.randn(total + c["pad"], c["heads"] + 2 * H, d, generator=g, device="cuda").to(kind)
        s["q"], s["k"], s["v"] = x[:, :c["heads"]], x[:, c["heads"]:c["heads"] + H], x[:, c["heads"] + H:]
        s["positions"] = torch.tensor([c["start"] + i for m in news for i in range(m)] + [-1] * c["pad"], dtype=torch.int32).cuda()
        s["requests"] = torch.tensor([b for b, m in enumerate(news) for _ in range(m)] + [0] * c["pad"], dtype=torch.int32).cuda()
        # pages before the first written one are not touched: their table entries name one page of the pool
        s["pages"] = _random_pages(g, B * used + 1, c)
        table = torch.full((B, first + used), B * used, dtype=torch.int32, device="cuda")
        table[:, first:] = torch.randperm(B * used, generator=g, device="cuda").to(torch.int32).view(B, used)
        s["table"] = table
        s["idx"] = torch.arange(first, first + used, dtype=torch.int32, device="cuda").expand(B, H, used).contiguous()
        s["q_out"] = torch.zeros(total + c["pad"], c["heads"], d, dtype=kind, device="cuda")
        s["back"] = torch.empty(B, H, 2, used * c["page"], d, dtype=kind, device="cuda")
        s["turns"] = torch.from_numpy(_turns(c)).cuda()
        s["n"] = total
        if own:
            from paper_2607_26475_b200 import binding as dd
            s["rope"] = dd.Rope(head_dim=d, base=500000.0) if c["rope"] else None
    elif c["op"] == "attn":
        _filled(s, c, g, _lens(c))
        s["q"] = torch.randn(B, n, c["heads"], d, generator=g, device="cuda").to(kind)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(B, n, c["heads"], dtype=torch.float32, device="cuda")
    else:
        _filled(s, c, g, _lens(c))
        M = s["table"].shape[1]
        s["q"] = torch.randn(B * n, c["heads"], d, generator=g, device="cuda").to(kind)
        # the newest tokens of every request; what would lie before its beginning is padding
        at = s["lens"].view(B, 1) - n + torch.arange(n, dtype=torch.int32, device="cuda")
        s["positions"] = at.clamp(min=-1).flatten().contiguous()
        s["requests"] = torch.arange(B, dtype=torch.int32, device="cuda").repeat_interleave(n)
        s["idx"] = torch.full((B * n, H, c["picked"]), -1, dtype=torch.int32, device="cuda")
        if c["op"] == "select":
            total = s["pages"].shape[0]
            s["landmarks"] = torch.zeros(total, H, d + LM_PAD, dtype=torch.uint8, device="cuda")
            last = torch.full((total,), c["page"], dtype=torch.int64, device="cuda")          # tokens that each page holds
            for b, m in enumerate(_lens(c)):
                if m % c["page"]:
                    last[s["table"][b, m // c["page"]].long()] = m % c["page"]
            step = max(1, (1 << 26) // (H * c["page"] * d))
            for a in range(0, total - 1, step):
                e = min(total - 1, a + step)
                valid = torch.arange(c["page"], device="cuda") < last[a:e].view(-1, 1, 1)
                s["landmarks"][a:e] = _landmark(_values(s["pages"][a:e], c)[:, :, 0], valid.expand(-1, H, -1))
        else:
            # what a selection gives: neighbours share most of their pages
            mine = torch.div(s["positions"], c["page"], rounding_mode="floor").view(B, n, 1, 1)
            p = torch.arange(M, device="cuda")
            like = torch.randn(B, 1, H, M, generator=g, device="cuda") + 0.3 * torch.randn(B, n, H, M, generator=g, device="cuda")
            like = torch.where((p < c["first"]) | (p > mine - c["recent"]), torch.full_like(like, 1e9), like)
            like = torch.where(p <= mine, like, torch.full_like(like, -1e9))
            k = min(c["picked"], M)
            top, got = like.topk(k, dim=-1)
            got = torch.where(top > -1e8, got, torch.full_like(got, M)).sort(-1).values
            s["idx"].view(B, n, H, -1)[..., :k] = torch.where(got < M, got, torch.full_like(got, -1)).to(torch.int32)
            s["out"] = torch.zeros_like(s["q"])
            s["lse"] = torch.zeros(B * n, c["heads"], dtype=torch.float32, device="cuda")
    if own:
        s["handle"] = _cache_handle(s, c)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _rotate(x, positions, turns):
    """Rows x [tokens, heads, dim] turned by their positions, in 64 bits: a code hangs on which side of a border a value falls."""
    a = positions.double().unsqueeze(-1) * turns
    a = (a - a.floor()) * (2 * math.pi)
    cos, sin = a.cos().unsqueeze(1), a.sin().unsqueeze(1)
    u, w = x.double().chunk(2, -1)
    return torch.cat((u * cos - w * sin, w * cos + u * sin), -1)


def _plain_append(s):
    c, n = s["c"], s["n"]
    k, v, at = s["k"][:n].float(), s["v"][:n].float(), s["positions"][:n].long()
    if c["rope"]:
        k = _rotate(s["k"][:n], at, s["turns"])
        s["q_out"][:n] = _rotate(s["q"][:n], at, s["turns"]).to(s["q_out"].dtype)
    block = s["table"][s["requests"][:n].long(), at // c["page"]].long()
    tile, tok = at % c["page"] // 16, at % 16
    hk, hv, hks, hvs, hex_ = _tiles(s["pages"], c)
    (kc, ks, ke), (vc, vs, ve) = _quantise4(k), _quantise4(v)
    hk[block, :, tile, tok], hks[block, :, tile, tok], hex_[block, :, tile, 0, tok] = _pack(kc), ks, ke
    hv[block, :, tile, tok // 8, :, tok % 8 // 2, tok % 2] = _pack(vc).unflatten(-1, (8, -1))
    hvs[block, :, tile, :, tok], hex_[block, :, tile, 1, tok] = vs, ve
    phys = s["table"].long().unsqueeze(1).expand(-1, c["kv_heads"], -1).gather(2, s["idx"].long())
    got = _values(s["pages"][phys, torch.arange(c["kv_heads"], device=phys.device).view(1, -1, 1)], c)
    out = {"cache": got.transpose(2, 3).flatten(3, 4).to(TYPES[c["type"]])}
    if c["rope"]:
        out["q"] = s["q_out"]
    return out


def _all_tokens(s):
    """Every token of every request's table: K and V [B, H, tokens, dim] in 32 bits."""
    c = s["c"]
    kv = _values(s["pages"][s["table"].long()], c)                # [B, M, H, 2, page, dim]
    return kv[:, :, :, 0].transpose(1, 2).flatten(2, 3), kv[:, :, :, 1].transpose(1, 2).flatten(2, 3)


def _attend(q, k, v, seen, dim):
    """q [B, H, rows, dim] over k, v [B, H, tokens, dim] where seen [B, 1 or H, rows, tokens]."""
    z = torch.matmul(q, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(dim)).masked_fill_(~seen, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = z.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o, (top + torch.log(total)).squeeze(-1)


def _plain_attn(s):
    c = s["c"]
    B, n, H, d = c["requests"], c["tokens"], c["kv_heads"], c["dim"]
    G = c["heads"] // H
    k, v = _all_tokens(s)
    q = s["q"].float().view(B, n, H, G, d).transpose(1, 2).reshape(B, H, n * G, d)
    last = (s["lens"].view(B, 1) - n + torch.arange(n, device=q.device)).repeat_interleave(G, 1).view(B, 1, -1, 1)
    at = torch.arange(k.shape[2], device=q.device)
    seen = at <= last
    if c["window"]:
        seen = seen & (at > last - c["window"])
    o, lse = _attend(q, k, v, seen, d)
    o = o.view(B, H, n, G, d).transpose(1, 2).reshape(B, n, H * G, d)
    return {"out": o.to(s["q"].dtype), "lse": lse.view(B, H, n, G).transpose(1, 2).reshape(B, n, H * G)}


def _plain_select(s):
    c = s["c"]
    B, n, H, d, T = c["requests"], c["tokens"], c["kv_heads"], c["dim"], c["page"]
    M, dev = s["table"].shape[1], s["q"].device
    # landmarks of the pages that hold the newest tokens
    lens = s["lens"].view(B, 1).long()
    fresh = (lens - n).clamp(min=0) // T + torch.arange((n + T - 2) // T + 1, device=dev)
    live = (fresh * T < lens).view(B, -1, 1, 1)
    block = s["table"].long().gather(1, fresh.clamp(max=M - 1))
    block = torch.where(live[..., 0, 0], block, torch.full_like(block, s["pages"].shape[0] - 1))
    valid = fresh.unsqueeze(-1) * T + torch.arange(T, device=dev) < lens.unsqueeze(-1)
    new = _landmark(_values(s["pages"][block], c)[:, :, :, 0], valid.unsqueeze(2).expand(-1, -1, H, -1))
    s["landmarks"][block] = torch.where(live, new, s["landmarks"][block])
    # scores
    q, _ = _whole(s["q"].double().view(B, n, H, -1, d).sum(3), -120)
    lm = s["landmarks"][s["table"].long()]                        # [B, M, H, dim + 16]
    codes = lm[..., :d].contiguous().view(torch.int8).float()
    z = torch.matmul(q.transpose(1, 2), codes.permute(0, 2, 3, 1)) * _two_to(lm[..., d].int() - 64).float().transpose(1, 2).unsqueeze(2)
    mine = torch.div(s["positions"], T, rounding_mode="floor").view(B, 1, n, 1)
    p = torch.arange(M, device=dev)
    z = torch.where((p < c["first"]) | (p > mine - c["recent"]), torch.full_like(z, math.inf), z)
    z = torch.where(p <= mine, z, torch.full_like(z, -math.inf))
    k = min(c["picked"], M)
    top, got = z.sort(dim=-1, descending=True, stable=True)
    got = torch.where(top[..., :k] > -math.inf, got[..., :k], torch.full_like(got[..., :k], M)).sort(-1).values
    idx = torch.full((B, H, n, c["picked"]), -1, dtype=torch.int32, device=dev)
    idx[..., :k] = torch.where(got < M, got, torch.full_like(got, -1)).to(torch.int32)
    return {"idx": idx.transpose(1, 2).reshape(B * n, H, -1), "landmarks": s["landmarks"]}


def _plain_sparse(s):
    c = s["c"]
    B, n, H, d, T = c["requests"], c["tokens"], c["kv_heads"], c["dim"], c["page"]
    G, M = c["heads"] // H, s["table"].shape[1]
    idx = s["idx"].view(B, n, H, -1).transpose(1, 2).long()
    listed_ = torch.zeros(B, H, n, M + 1, dtype=torch.bool, device=idx.device).scatter_(3, torch.where(idx < 0, torch.full_like(idx, M), idx), True)
    at = torch.arange(M * T, device=idx.device)
    seen = listed_[..., :M].repeat_interleave(T, 3) & (at <= s["positions"].view(B, 1, n, 1))
    k, v = _all_tokens(s)
    q = s["q"].float().view(B, n, H, G, d).transpose(1, 2).reshape(B, H, n * G, d)
    o, lse = _attend(q, k, v, seen.repeat_interleave(G, 2), d)
    o = o.view(B, H, n, G, d).transpose(1, 2).reshape(B * n, H * G, d)
    lse = lse.view(B, H, n, G).transpose(1, 2).reshape(B * n, H * G)
    there = (s["positions"] >= 0).view(-1, 1)
    return {"out": torch.where(there.unsqueeze(-1), o.to(s["q"].dtype), s["out"]), "lse": torch.where(there, lse, s["lse"])}


def run(s):
    c = s["c"]
    if not own:
        return {"append": _plain_append, "attn": _plain_attn, "select": _plain_select, "sparse": _plain_sparse}[c["op"]](s)
    cache = s["handle"]
    if c["op"] == "append":
        if c["rope"]:
            cache.append(s["k"], s["v"], s["positions"], s["requests"], rope=s["rope"], q=s["q"], q_out=s["q_out"])
        else:
            cache.append(s["k"], s["v"], s["positions"], s["requests"])
        cache.read(s["idx"], s["back"])
        return {"cache": s["back"], "q": s["q_out"]} if c["rope"] else {"cache": s["back"]}
    if c["op"] == "attn":
        cache.decode_attn(s["q"], s["lens"], s["out"], s["lse"], window=c["window"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "select":
        cache.update_landmarks(s["landmarks"], s["lens"], n_last=c["tokens"])
        cache.select(s["q"], s["landmarks"], s["positions"], s["idx"], s["requests"], first_pages=c["first"], recent_pages=c["recent"])
        return {"idx": s["idx"], "landmarks": s["landmarks"]}
    cache.sparse_attn(s["q"], s["idx"], s["positions"], s["out"], s["lse"], s["requests"])
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------------ the definition, 64 bits
def _e4m3_table():
    """What each of the 256 codes stands for."""
    v = []
    for code in range(256):
        sign, e, m = -1.0 if code & 128 else 1.0, (code >> 3) & 15, code & 7
        v.append(float("nan") if code & 127 == 127 else sign * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)))
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def _places4(T, d):
    """Where in a 4-bit page each element lies: byte of its code, shift of it, byte of its scale and of its exponent, [2, T, d]."""
    kv, t, x = np.meshgrid(np.arange(2), np.arange(T), np.arange(d), indexing="ij")
    tile, r, size = t // 16 * (18 * d + 32), t % 16, d // 8
    k_at = r * (d // 2) + x // 2
    v_at = 8 * d + (((r // 8) * 8 + x // size) * 4 + r % 8 // 2) * size + (r % 2) * (size // 2) + x % size // 2
    code = tile + np.where(kv == 0, k_at, v_at)
    scale = tile + 16 * d + np.where(kv == 0, r * (d // 16) + x // 16, d + x // 16 * 16 + r)
    return [torch.from_numpy(a).cuda() for a in (code, 4 * (x % 2), scale, tile + 18 * d + 16 * kv + r)]


def _exact_page(raw, c):
    """Pages [..., bytes] -> [..., 2, page, dim] in 64 bits."""
    T, d = c["page"], c["dim"]
    if c["cache"] == "int4":
        code, shift, scale, ex = _places4(T, d)
        number = ((raw[..., code] >> shift.to(torch.uint8)) & 15).double() - 8
        return number * _e4m3_table()[raw[..., scale].long()] * _two_to(raw[..., ex].int() - 127)
    if c["cache"] != "e4m3":
        return raw.contiguous().view(TYPES[c["type"]]).double().unflatten(-1, (2, T, d))
    n = 2 * T * d
    codes = _e4m3_table()[raw[..., :n].long()].unflatten(-1, (2, T, d))
    return codes * _two_to(raw[..., n:].int() - 127).unflatten(-1, (2, T)).unsqueeze(-1)


def _exact_rows4(x):
    """Rows x [..., dim] as a 4-bit cache holds them: the nearest of 15 multiples of the group's step, the even one of two."""
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 3136.0))
    e = torch.where(top > 3136.0 * _two_to(e), e + 1, torch.where(top <= 3136.0 * _two_to(e - 1), e - 1, e)).clamp(min=-127.0)
    y = (x / _two_to(e)).unflatten(-1, (-1, 16))
    top = y.abs().amax(-1, keepdim=True)
    want = (top / torch.full_like(top, 7.0)).clamp(min=2.0 ** -4)
    unit = _two_to(torch.floor(torch.log2(want)) - 3)
    step = torch.round(want / unit) * unit
    below = torch.floor(y / step)
    rest = y - below * step - step / 2
    number = below + ((rest > 0) | ((rest == 0) & (torch.remainder(below, 2.0) == 1))).double()
    return (number.clamp(-7, 7) * step).flatten(-2) * _two_to(e)


def _exact_turn(x, positions, c):
    """The rotation as a complex product."""
    angle = 2 * math.pi * torch.remainder(positions.double().unsqueeze(-1) * torch.from_numpy(_turns(c)).cuda(), 1.0)
    y = x.double()
    z = torch.complex(y[..., :c["dim"] // 2].contiguous(), y[..., c["dim"] // 2:].contiguous()) * torch.polar(torch.ones_like(angle), angle).unsqueeze(1)
    return torch.cat((z.real, z.imag), -1)


def _exact_whole(x, least):
    """A row as whole numbers up to 127 times the smallest power of two that allows it (not below 2^least)."""
    top, e = float(x.abs().max()), least
    while top > 127.0 * 2.0 ** e and e < 63:
        e += 1
    return torch.round(x / 2.0 ** e).clamp(-127, 127), e


def _exact_select(s, c):
    """Token by token and head by head, from the stored keys and landmarks."""
    H, d, T, B, n = c["kv_heads"], c["dim"], c["page"], c["requests"], c["tokens"]
    lens, G = _lens(c), c["heads"] // c["kv_heads"]
    lm = s["landmarks"].clone()
    idx = torch.full((B * n, H, c["picked"]), -1, dtype=torch.int32)
    for b, m in enumerate(lens):
        if m == 0:
            continue
        for p in range(max(0, m - n) // T, (m - 1) // T + 1):
            block = int(s["table"][b, p])
            keys = _exact_page(s["pages"][block], c)[:, 0, :min(T, m - p * T)].mean(1)
            for h in range(H):
                number, e = _exact_whole(keys[h], -64)
                lm[block, h] = 0
                lm[block, h, :d] = number.to(torch.int8).view(torch.uint8)
                lm[block, h, d] = e + 64
        mine = lm[s["table"][b, :(m - 1) // T + 1].long()]
        codes = mine[..., :d].contiguous().view(torch.int8).double() * _two_to(mine[..., d:d + 1].int() - 64)
        for t in range(max(0, n - m), n):
            q = s["q"][b * n + t].double().view(H, G, d).sum(1)
            own_page = (m - n + t) // T
            for h in range(H):
                z = (codes[:own_page + 1, h] @ _exact_whole(q[h], -120)[0]).cpu().numpy()
                z[:c["first"]] = math.inf
                z[max(0, own_page + 1 - c["recent"]):] = math.inf
                best = np.sort(np.argsort(-z, kind="stable")[:c["picked"]])
                idx[b * n + t, h, :best.size] = torch.from_numpy(best.astype(np.int32))
    return {"idx": idx.cuda(), "landmarks": lm}


def exact(c, seed):
    s = prepare(c, seed)
    H, d, T, B = c["kv_heads"], c["dim"], c["page"], c["requests"]
    if c["op"] == "select":                          # a chunk's tokens one by one take minutes
        return _exact_select(s, c) if B * c["tokens"] * H <= 1024 else None
    if c["op"] == "append":
        raw, idx = s["pages"], s["idx"]
        out = torch.empty(B, H, 2, idx.shape[2], T, d, dtype=torch.float64, device="cuda")
        for b in range(B):
            for h in range(H):
                out[b, h] = _exact_page(raw[s["table"][b][idx[b, h].long()].long(), h], c).transpose(0, 1)
        out = out.view(B, H, 2, -1, d)
        n, first = s["n"], c["start"] // T * T
        k64 = _exact_rows4(_exact_turn(s["k"][:n], s["positions"][:n], c) if c["rope"] else s["k"][:n].double())
        v64 = _exact_rows4(s["v"][:n].double())
        at = 0
        for b, m in enumerate(_new_tokens(c)):
            a = c["start"] - first
            out[b, :, 0, a:a + m], out[b, :, 1, a:a + m] = k64[at:at + m].transpose(0, 1), v64[at:at + m].transpose(0, 1)
            at += m
        if not c["rope"]:
            return {"cache": out}
        q = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        q[:n] = _exact_turn(s["q"][:n], s["positions"][:n], c)
        return {"cache": out, "q": q}
    n, G = c["tokens"], c["heads"] // H
    q = s["q"].view(B, n, c["heads"], d)
    if c["op"] == "attn":
        out = torch.zeros(B, n, c["heads"], d, dtype=torch.float64, device="cuda")
        lse = torch.full((B, n, c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    else:
        out, lse = s["out"].double().view(B, n, -1, d), s["lse"].double().view(B, n, -1)
    lens = _lens(c)
    for b, m in enumerate(lens):
        if m == 0:
            continue
        blocks = s["table"][b, :-(-m // T)].long()
        for h in range(H):
            kv = _exact_page(s["pages"][blocks, h], c).transpose(0, 1).reshape(2, -1, d)
            rows = slice(h * G, (h + 1) * G)
            if c["op"] == "attn":
                for t in range(n):
                    end = m - n + t + 1
                    begin = max(0, end - c["window"]) if c["window"] else 0
                    if end > 0:
                        z = q[b, t, rows].double() @ kv[0, begin:end].T / math.sqrt(d)
                        out[b, t, rows] = torch.softmax(z, -1) @ kv[1, begin:end]
                        lse[b, t, rows] = torch.logsumexp(z, -1)
                continue
            # every listed page gathered, some tokens at a time
            live = [t for t in range(n) if m - n + t >= 0]
            for a in range(0, len(live), 64):
                t = torch.tensor(live[a:a + 64], device="cuda")
                pages = s["idx"].view(B, n, H, -1)[b, t, h].long()                              # [t, picked]
                tok = pages.unsqueeze(-1) * T + torch.arange(T, device="cuda")
                hidden = ((pages.unsqueeze(-1) < 0) | (tok > (m - n + t).view(-1, 1, 1))).flatten(1)
                tok = tok.clamp(min=0).flatten(1)
                z = torch.einsum("tgd,tnd->tgn", q[b, t, rows].double(), kv[0][tok]) / math.sqrt(d)
                z = z.masked_fill(hidden.unsqueeze(1), -math.inf)
                out[b, t, rows] = torch.einsum("tgn,tnd->tgd", torch.softmax(z, -1), kv[1][tok])
                lse[b, t, rows] = torch.logsumexp(z, -1)
    if c["op"] == "sparse":
        return {"out": out.view(B * n, -1, d), "lse": lse.view(B * n, -1)}
    return {"out": out, "lse": lse}
