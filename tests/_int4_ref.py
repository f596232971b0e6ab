"""Plain 64-bit definitions of the 4-bit cache and of attention over listed pages, on the CPU (numpy), for the tests of their
kernels."""
import math

import numpy as np
import torch

from tests import _cache_ref as ref

E4M3 = ref.CODES[:127]             # 0 ... 448, ascending


def page_bytes(fmt, T, d):
    return T // 16 * (18 * d + 32) if fmt == "int4" else ref.page_bytes(fmt, T, d)


def nearest(table, x):
    """Index of the entry of an ascending table nearest to x >= 0, the even index of two."""
    hi = np.searchsorted(table, x, side="left").clip(0, len(table) - 1)
    lo = np.maximum(hi - 1, 0)
    a, b = x - table[lo], table[hi] - x
    return np.where(table[hi] == x, hi, np.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi))


def quantise(x):
    """Rows x [..., d] (64 bits) -> (codes [..., d] 1 ... 15, scales [..., d / 16] as e4m3 codes, exponent bytes [...])."""
    fin = np.where(np.isfinite(x), np.abs(x), 0.0)
    amax = fin.max(-1)
    e = np.full(amax.shape, -127, dtype=np.int64)
    for at in np.ndindex(amax.shape):
        if amax[at] > 0:
            k = math.floor(math.log2(amax[at] / 3136.0)) - 1
            while 3136.0 * 2.0 ** k < amax[at]:
                k += 1
            e[at] = max(-127, k)
    shape = x.shape[:-1] + (x.shape[-1] // 16, 16)
    y = (np.where(np.isfinite(x), x, 0.0) * np.exp2(-e.astype(np.float64))[..., None]).reshape(shape)
    scale = nearest(E4M3, np.maximum(np.abs(y).max(-1) / 7.0, 2.0 ** -4))
    bad = ~np.isfinite(x).reshape(shape).all(-1)
    n = np.rint(y / E4M3[scale][..., None]).clip(-7, 7)              # rint: the even one of two
    n = np.where(bad[..., None], 0.0, n)
    return (n + 8).astype(np.uint8).reshape(x.shape), np.where(bad, 127, scale).astype(np.uint8), (e + 127).astype(np.uint8)


def places(T, d):
    """Where in a page each element lies: byte and shift of its code, byte of its scale and of its exponent, each [2, T, d]."""
    kv, t, x = np.meshgrid(np.arange(2), np.arange(T), np.arange(d), indexing="ij")
    tile, r, part = t // 16 * (18 * d + 32), t % 16, d // 8
    k_at = r * d // 2 + x // 2
    v_at = 8 * d + (r // 8) * 4 * d + (x // part) * d // 2 + (r % 8 // 2) * d // 8 + (r % 2) * d // 16 + x % part // 2
    scale = tile + 16 * d + np.where(kv == 0, r * (d // 16) + x // 16, d + x // 16 * 16 + r)
    return tile + np.where(kv == 0, k_at, v_at), 4 * (x % 2), scale, tile + 18 * d + 16 * kv + r


def decode_pages(raw, fmt, T, d):
    """Pages uint8 [..., bytes] -> [..., 2, T, d] in 64 bits."""
    if fmt != "int4":
        return ref.decode_pages(raw, fmt, T, d)
    code, shift, scale, ex = places(T, d)
    n = (raw[..., code].astype(np.int64) >> shift & 15) - 8
    return n * ref.CODES[raw[..., scale]] * np.exp2(raw[..., ex].astype(np.float64) - 127)


def encode_pages(v, fmt):
    """Values [..., 2, T, d] (64 bits) -> pages uint8 [..., bytes]."""
    if fmt != "int4":
        return ref.encode_pages(v, fmt)
    T, d = v.shape[-2:]
    codes, scales, ex = quantise(v)
    code, shift, scale, e = places(T, d)
    raw = np.zeros(v.shape[:-3] + (page_bytes(fmt, T, d),), dtype=np.uint8)
    for s in (0, 4):                                                 # one nibble of every byte at a time
        m = shift == s
        raw[..., code[m]] |= codes[..., m] << s
    raw[..., scale[..., ::16]] = scales
    raw[..., e[..., 0]] = ex
    return raw


def rows_of(raw, table_row, h, n, fmt, T, d):
    """K and V [n, d] of the first n tokens of a request, KV head h."""
    pages = raw[table_row[:-(-n // T)], h]
    return np.moveaxis(decode_pages(pages, fmt, T, d), 0, 1).reshape(2, -1, d)[:, :n]


def attend(q, K, V, scale):
    """q [G, d] over K, V [n, d]: out, lse, and what roundings are measured by (sum of weight * |V|, largest sum |q||k| * scale)."""
    z = q @ K.T * scale
    m = z.max(-1, keepdims=True)
    p = np.exp(z - m)
    total = p.sum(-1, keepdims=True)
    return p @ V / total, (m + np.log(total))[:, 0], p @ np.abs(V) / total, (np.abs(q) @ np.abs(K).T).max(-1) * scale


def attention(q, raw, table, lens, fmt, T, window=0, scale=None):
    """q [B, Tq, Hq, d]: attention of each request's last Tq tokens over all its tokens; see attend."""
    B, Tq, Hq, d = q.shape
    H = raw.shape[1]
    G = Hq // H
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, absum = np.zeros(q.shape), np.zeros(q.shape)
    lse, unit = np.full((B, Tq, Hq), -np.inf), np.zeros((B, Tq, Hq))
    for b in range(B):
        n = int(lens[b])
        for h in range(H if n > 0 else 0):
            K, V = rows_of(raw, table[b], h, n, fmt, T, d)
            for t in range(Tq):
                end = n - Tq + t + 1
                begin = max(0, end - window) if window else 0
                if end > 0:
                    r = np.s_[b, t, h * G:(h + 1) * G]
                    out[r], lse[r], absum[r], unit[r] = attend(q[r], K[begin:end], V[begin:end], scale)
    return out, lse, absum, unit


def listed_attention(q, raw, table, requests, positions, idx, fmt, T, scale=None):
    """q [N, Hq, d] over the pages idx [N, H, k]; tokens that see nothing: zeros and -inf."""
    N, Hq, d = q.shape
    H = raw.shape[1]
    G = Hq // H
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, absum = np.zeros(q.shape), np.zeros(q.shape)
    lse, unit = np.full((N, Hq), -np.inf), np.zeros((N, Hq))
    pages = decode_pages(raw, fmt, T, d)                             # [blocks, H, 2, T, d]
    for n in range(N):
        pos = int(positions[n])
        for h in range(H if pos >= 0 else 0):
            ks, vs = [], []
            for p in idx[n, h][:pos // T + 1]:
                if 0 <= p <= pos // T:
                    blk = int(table[int(requests[n]), p])
                    kv = pages[blk, h][:, :min(T, pos + 1 - p * T)]
                    ks.append(kv[0])
                    vs.append(kv[1])
            if ks:
                r = np.s_[n, h * G:(h + 1) * G]
                out[r], lse[r], absum[r], unit[r] = attend(q[r], np.concatenate(ks), np.concatenate(vs), scale)
    return out, lse, absum, unit


def whole(x, least):
    """A row as whole numbers within 127 times 2^e: (numbers, e)."""
    x = np.where(np.isfinite(x), x, 0.0)
    top, e = np.abs(x).max(), least
    while e < 63 and top > 127.0 * 2.0 ** e:
        e += 1
    return np.rint(x * 2.0 ** -e).clip(-127, 127), e


def landmark(keys):
    """Bytes of the landmark of keys [n, d]."""
    d = keys.shape[1]
    with np.errstate(invalid="ignore"):
        n, e = whole(keys.sum(0) / len(keys), -64)
    out = np.zeros(d + 16, dtype=np.uint8)
    out[:d], out[d] = n.astype(np.int8).view(np.uint8), e + 64
    return out


def select(q, landmarks, k, first, recent, own):
    """Pages of one token and head: q [G, d], landmarks uint8 [own + 1, d + 16] of its visible pages."""
    d = q.shape[1]
    c, _ = whole(q.sum(0), -120)
    z = landmarks[:, :d].view(np.int8).astype(np.float64) @ c * np.exp2(landmarks[:, d].astype(np.float64) - 64)
    z[:first] = np.inf
    z[max(0, own + 1 - recent):] = np.inf
    best = np.sort(np.argsort(-z, kind="stable")[:k])
    return np.concatenate([best, np.full(k - len(best), -1)]).astype(np.int32)


STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}             # half a step of the type, relative
BITS = {"bf16": 8, "fp16": 11}
TINY = {"bf16": 2.0 ** -134, "fp16": 2.0 ** -25}
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def check(got, lse, want, want_lse, absum, unit, fmt, kind, n_max):
    """Results lie within the output's own rounding of something within `slack` of the definition. slack: a score is d products
    added in fp32 (each addition off by 2^-24 of a partial sum, at most sum |q||k|) and two multiplications, and both weight and
    denominator carry it; weights are two 16-bit parts (2^-16 for bf16 pages, 2^-22 for half queries) or, for quantised pages with bf16
    queries, one half (2^-11); sums of n terms 2^-24 each."""
    d = got.shape[-1]
    g = got.detach().cpu().double().numpy()
    dz = (d + 8) * 2.0 ** -24 * unit + 2.0 ** -21 * (1 + np.where(np.isfinite(want_lse), np.abs(want_lse), 0.0))
    weight = 2.0 ** -16 if fmt == "bf16" else 2.0 ** -11 if kind == "bf16" else 2.0 ** -22
    rel = weight + 2 * dz + n_max * 2.0 ** -29 + 2.0 ** -16
    slack = rel[..., None] * np.maximum(absum, absum.max(-1, keepdims=True) * 2.0 ** -10)
    half = np.maximum(np.exp2(np.frexp(np.abs(want) + slack)[1] - BITS[kind] - 1.0), TINY[kind])
    assert np.all(np.isfinite(g)), "a value that nobody sees was used"
    off = np.abs(g - want) - half
    assert np.all(off <= slack), f"{(off[off > slack] / slack[off > slack]).max()} times the slack"
    if lse is not None:
        l = lse.detach().cpu().double().numpy()
        empty = ~np.isfinite(want_lse)
        assert np.array_equal(empty, np.isneginf(l))
        assert np.all(np.abs(l[~empty] - want_lse[~empty]) <= (dz + 2.0 ** -20 + n_max * 2.0 ** -33)[~empty])
        assert np.all(g[empty] == 0.0)
