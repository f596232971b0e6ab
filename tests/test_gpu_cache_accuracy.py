"""Attention over the cache to within the rounding of its own output: nothing before that may cost a visible part of it.

A result is the correctly rounded value of something that lies within `slack` of the definition; slack counts the fp32
arithmetic and the weights. Weights are held as two 16-bit parts (off by (2^-8)^2 = 2^-16 of a weight for bf16 pages, by
2^-22 for half queries), for e4m3 pages with bf16 queries as one half (2^-11, an eighth of the output's half step)."""
import numpy as np
import pytest
import torch

from tests import _cache_ref as ref
from tests._cache_ref import f64
from tests.test_gpu_cache import TINY, check_attn, dd, make_attn, run_attn  # noqa: F401  (dd is the fixture)

pytestmark = pytest.mark.gpu

BITS = {"bf16": 8, "fp16": 11}


def half_step(x, kind):
    """Half of the distance between neighbours of the type at magnitude |x|."""
    return np.maximum(np.exp2(np.frexp(np.abs(x))[1] - BITS[kind] - 1.0), TINY[kind])


CASES = [  # lens, H, G, d, T, fmt, query type, Tq, window, scale
    ([2, 3, 7, 40, 1], 2, 4, 128, 16, "bf16", "bf16", 1, 0, 0.0),
    ([300, 17, 2], 1, 4, 128, 16, "bf16", "bf16", 2, 0, 0.0),
    ([300, 17, 2], 1, 16, 128, 16, "bf16", "bf16", 1, 20, 0.0),
    ([77, 5], 2, 5, 64, 32, "bf16", "bf16", 3, 0, 0.0),
    ([4000], 2, 4, 128, 16, "bf16", "bf16", 1, 0, 0.3),
    ([2, 3, 7, 40, 1], 2, 4, 128, 16, "fp16", "fp16", 1, 0, 0.02),
    ([300, 17, 2], 1, 12, 64, 16, "fp16", "fp16", 2, 0, 0.02),
    ([2, 3, 7, 40, 1], 2, 4, 128, 16, "e4m3", "fp16", 1, 0, 0.02),
    ([300, 17, 2], 1, 12, 64, 16, "e4m3", "fp16", 2, 0, 0.02),
    ([2, 3, 7, 40, 1], 2, 4, 128, 16, "e4m3", "bf16", 1, 0, 0.0),
    ([300, 17, 2], 1, 12, 64, 16, "e4m3", "bf16", 2, 0, 0.0),
]


@pytest.mark.parametrize("lens,H,G,d,T,fmt,kind,Tq,window,scale", CASES)
def test_only_the_output_is_rounded_visibly(dd, lens, H, G, d, T, fmt, kind, Tq, window, scale):
    gen = torch.Generator().manual_seed(sum(lens) + G + d)
    cache, raw, table, q = make_attn(dd, gen, lens, H, G, d, T, fmt, kind, Tq)
    out, lse = run_attn(cache, q, lens, window, scale)
    want, want_lse, absum, unit = ref.attention(f64(q), raw, table.numpy(), lens, fmt, T, window, scale or None)
    # a score: d products added in fp32 (each addition off by 2^-24 of a partial sum, at most sum |q||k|), two multiplications;
    # weight and denominator both carry it
    dz = (d + 8) * 2.0 ** -24 * unit + 2.0 ** -21 * (1 + np.where(np.isfinite(want_lse), np.abs(want_lse), 0.0))
    weight = 2.0 ** -11 if (fmt, kind) == ("e4m3", "bf16") else 2.0 ** -16 if fmt == "bf16" else 2.0 ** -22
    rel = weight + 2 * dz + max(lens) * 2.0 ** -29 + 2.0 ** -16
    slack = rel[..., None] * np.maximum(absum, absum.max(-1, keepdims=True) * 2.0 ** -10)
    off = np.abs(f64(out) - want) - half_step(np.abs(want) + slack, kind)
    assert np.all(off <= slack), f"{(off / slack).max()} times the slack"


@pytest.mark.parametrize("d,G", [(128, 4), (64, 16)])
def test_keys_of_the_smallest_exponent_count(dd, d, G):
    """A key row whose exponent byte is 0 holds code * 2^-127; large queries make scores of ordinary size of it."""
    gen = torch.Generator().manual_seed(d)
    lens, T = [70, 3], 16
    cache, raw, table, q = make_attn(dd, gen, lens, 1, G, d, T, "e4m3", "bf16", 1, poison=False)
    raw[:, :, 2 * T * d:2 * T * d + T] = np.random.RandomState(d).randint(0, 2, (raw.shape[0], 1, T))      # 2^-127 and 2^-126
    cache.data.copy_(torch.from_numpy(raw).cuda())
    q = (q.float() * 2.0 ** 120).to(torch.bfloat16)
    out, lse = run_attn(cache, q, lens)
    want_lse = ref.attention(f64(q), raw, table.numpy(), lens, "e4m3", T)[1]
    assert np.ptp(want_lse - np.log(np.array(lens))[:, None, None]) > 0.05              # scores that are not all zero
    check_attn(out, lse, q, raw, table, lens, "e4m3", "bf16", T)


@pytest.mark.parametrize("lens,M,G,Tq,fmt", [([50, 7], 0, 4, 1, "bf16"), ([50, 7], 0, 4, 2, "fp16"), ([600], 0, 16, 1, "bf16"), ([600], 0, 4, 1, "fp16"),
                                             ([3000, 40], 1200, 4, 1, "bf16"), ([3000, 40], 1200, 12, 2, "fp16")])
def test_infinite_values_that_are_seen_stay_infinite(dd, lens, M, G, Tq, fmt):
    """A value of +inf or -inf under any positive weight makes that channel +inf or -inf, both make it NaN, and the other
    channels do not notice. Weights down to 2^-12 of the largest."""
    gen = torch.Generator().manual_seed(sum(lens) + G)
    d, T = 128, 16
    cache, raw, table, q = make_attn(dd, gen, lens, 1, G, d, T, fmt, fmt, Tq, poison=False)
    if M:                                                           # a wide table: the flat list and its joining kernel
        table = torch.cat([table, torch.zeros(len(lens), M - table.shape[1], dtype=torch.int32)], 1)
        cache = dd.PagedCache(cache.data, table.cuda(), cache_format=cache.cache_format, head_dim=d, page_tokens=T)
    kv = ref.decode_pages(raw, fmt, T, d)
    for b, n in enumerate(lens):
        for at, channel, v in ((0, 3, np.inf), (n // 2, 3, np.inf), (1, 9, -np.inf), (n - Tq - 1, 70, np.inf), (0, 70, -np.inf), (2, 100, np.nan)):
            kv[table[b, at // T], 0, 1, at % T, channel] = v
    raw = ref.encode_pages(kv, fmt)
    cache.data.copy_(torch.from_numpy(raw).cuda())
    scale = 0.1 / np.sqrt(d)                                        # scores within about +-2
    out, lse = run_attn(cache, q, lens, 0, scale)
    with np.errstate(invalid="ignore"):
        want = ref.attention(f64(q), raw, table.numpy(), lens, fmt, T, 0, scale)[0]
    g = f64(out)
    assert np.all(np.isposinf(want[..., 3])) and np.all(np.isneginf(want[..., 9])) and np.all(np.isnan(want[..., (70, 100)]))
    assert np.array_equal(np.isposinf(g), np.isposinf(want)) and np.array_equal(np.isneginf(g), np.isneginf(want))
    assert np.array_equal(np.isnan(g), np.isnan(want))
    fine = np.isfinite(want)
    assert np.abs(g[fine] - want[fine]).max() < 0.02
    assert cache.device_error() == (0, 0)


@pytest.mark.parametrize("lens,G,Tq,power", [([300, 5], 4, 1, 117), ([300, 5], 16, 2, 117), ([9000, 40], 4, 1, 113), ([300, 5], 4, 1, -100)])
def test_values_near_the_ends_of_bf16(dd, lens, G, Tq, power):
    """The weighted sum stays within fp32 as long as the number of tokens times the largest value does."""
    gen = torch.Generator().manual_seed(sum(lens) + G)
    cache, raw, table, q = make_attn(dd, gen, lens, 1, G, 128, 16, "bf16", "bf16", Tq, poison=False)
    kv = ref.decode_pages(raw, "bf16", 16, 128)
    kv[:, :, 1] *= 2.0 ** power                                     # 2^117: sums of 300 values reach 2^127.6 at most
    raw = ref.encode_pages(kv, "bf16")
    cache.data.copy_(torch.from_numpy(raw).cuda())
    out, lse = run_attn(cache, q, lens)
    check_attn(out, lse, q, raw, table, lens, "bf16", "bf16", 16)
