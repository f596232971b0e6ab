"""Plain 64-bit definitions of the paged-cache operators, on the CPU (numpy), for the tests of their kernels."""
import math

import numpy as np
import torch

CODES = np.array([(float("nan") if c & 127 == 127 else (-1.0 if c & 128 else 1.0) *
                   ((c & 7) * 2.0 ** -9 if (c >> 3) & 15 == 0 else (8 + (c & 7)) * 2.0 ** (((c >> 3) & 15) - 10)))
                  for c in range(256)])
_POS = CODES[:127]                 # 0 ... 448, ascending: code c stands for _POS[c]


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().double().numpy()


def turns_of(rot, base, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=32.0):
    """Turns per position of every pair."""
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if scaling == "linear":
            f = f / factor
        if scaling == "parts":
            kept = min(1.0, max(0.0, (original_len * f / (2 * math.pi) - low) / (high - low)))
            f = (1 - kept) * f / factor + kept * f
        out.append(f / (2 * math.pi))
    return np.array(out)


def rotate(x, positions, turns, layout, amplitude=1.0, backward=False):
    """Rows x [N, H, d] (64 bits) turned by their positions."""
    r = 2 * len(turns)
    part = positions.astype(np.float64)[:, None] * turns[None, :]
    a = 2 * np.pi * (part - np.floor(part))[:, None, :]
    c, s = np.cos(a) * amplitude, np.sin(a) * amplitude * (-1.0 if backward else 1.0)
    y = x.copy()
    iu, iw = (np.arange(r // 2), np.arange(r // 2) + r // 2) if layout == "half" else (np.arange(0, r, 2), np.arange(1, r, 2))
    y[..., iu] = x[..., iu] * c - x[..., iw] * s
    y[..., iw] = x[..., iw] * c + x[..., iu] * s
    return y


def quantise(x):
    """Rows x [..., d] (64 bits) -> (codes uint8, exponent bytes uint8)."""
    fin = np.where(np.isfinite(x), np.abs(x), 0.0)
    amax = fin.max(-1)
    e = np.full(amax.shape, -127, dtype=np.int64)
    for at in np.ndindex(amax.shape):
        if amax[at] > 0:
            k = math.floor(math.log2(amax[at] / 448.0)) - 1
            while 448.0 * 2.0 ** k < amax[at]:
                k += 1
            e[at] = max(-127, k)
    y = x * np.exp2(-e.astype(np.float64))[..., None]
    mag = np.where(np.isfinite(y), np.abs(y), 0.0)
    hi = np.searchsorted(_POS, mag, side="left").clip(0, 126)          # first code value >= mag
    lo = np.maximum(hi - 1, 0)
    dlo, dhi = mag - _POS[lo], _POS[hi] - mag
    code = np.where((dlo < dhi) | ((dlo == dhi) & (lo % 2 == 0)), lo, hi)
    code = np.where(_POS[hi] == mag, hi, code)
    code = np.where(np.signbit(x), code | 128, code).astype(np.uint8)
    code = np.where(np.isfinite(x), code, 127).astype(np.uint8)
    return code, (e + 127).astype(np.uint8)


def page_bytes(fmt, T, d):
    return 2 * T * d + 2 * T if fmt == "e4m3" else 4 * T * d


def decode_pages(raw, fmt, T, d):
    """Pages uint8 [..., bytes] -> [..., 2, T, d] in 64 bits."""
    if fmt == "e4m3":
        n = 2 * T * d
        v = CODES[raw[..., :n]].reshape(raw.shape[:-1] + (2, T, d))
        return v * np.exp2(raw[..., n:].astype(np.float64) - 127).reshape(raw.shape[:-1] + (2, T))[..., None]
    t = torch.from_numpy(np.ascontiguousarray(raw)).view(torch.bfloat16 if fmt == "bf16" else torch.float16)
    return t.double().numpy().reshape(raw.shape[:-1] + (2, T, d))


def encode_pages(v, fmt):
    """Values [..., 2, T, d] (64 bits, of the format's precision for 16-bit ones) -> pages uint8 [..., bytes]."""
    lead = v.shape[:-3]
    if fmt == "e4m3":
        code, ex = quantise(v)
        return np.concatenate([code.reshape(lead + (-1,)), ex.reshape(lead + (-1,))], -1)
    t = torch.from_numpy(v).to(torch.bfloat16 if fmt == "bf16" else torch.float16).contiguous()
    return t.view(torch.uint8).numpy().reshape(lead + (-1,)) if t.dim() else t


def attention(q, raw, table, lens, fmt, T, window=0, scale=None):
    """q [B, Tq, Hq, d] (64 bits), raw pages uint8 [n_blocks, H, bytes]; returns out, lse, and what the rounding of weights is
    measured by: sum of weight * |V|, and the largest score error unit (sum |q||k| * scale) of each row."""
    B, Tq, Hq, d = q.shape
    H = raw.shape[1]
    G = Hq // H
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, absum = np.zeros(q.shape), np.zeros(q.shape)
    lse, unit = np.full((B, Tq, Hq), -np.inf), np.zeros((B, Tq, Hq))
    for b in range(B):
        n = int(lens[b])
        if n <= 0:
            continue
        pages = raw[table[b, :(n + T - 1) // T]]
        for h in range(H):
            kv = np.moveaxis(decode_pages(pages[:, h], fmt, T, d), 0, 1).reshape(2, -1, d)
            for t in range(Tq):
                end = n - Tq + t + 1
                begin = max(0, end - window) if window else 0
                if end <= 0:
                    continue
                K, V = kv[0, begin:end], kv[1, begin:end]
                for j in range(G):
                    row = q[b, t, h * G + j]
                    z = K @ row * scale
                    m = z.max()
                    p = np.exp(z - m)
                    lse[b, t, h * G + j] = m + math.log(p.sum())
                    p /= p.sum()
                    out[b, t, h * G + j] = p @ V
                    absum[b, t, h * G + j] = p @ np.abs(V)
                    unit[b, t, h * G + j] = (np.abs(K) @ np.abs(row)).max() * scale
    return out, lse, absum, unit
