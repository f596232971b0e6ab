"""Rotary positions, cache writes, cache reads and attention over the whole cache, against plain 64-bit definitions.

Tolerances count the roundings: half a step of the output type (eps / 2 relative: bf16 2^-8, half 2^-11), of the weights
(to bf16 or half before the second product), of a quantised value (2^-4 of it, or half of the smallest step of its row), and
fp32 arithmetic in between as derived at each comparison."""
import math

import numpy as np
import pytest
import torch

from tests import _cache_ref as ref
from tests._cache_ref import f64

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"bf16": 2.0 ** -134, "fp16": 2.0 ** -25}          # half of the smallest subnormal


@pytest.fixture(scope="module")
def dd():
    from paper_2607_26475_b200 import binding
    return binding


def fmt_code(dd, fmt):
    return {"bf16": dd.DD_CACHE_BF16, "fp16": dd.DD_CACHE_FP16, "e4m3": dd.DD_CACHE_E4M3}[fmt]


def rope_of(dd, d, rot, layout="half", scaling="none", amplitude=1.0):
    kw = dict(none={}, linear=dict(factor=4.0), ntk=dict(factor=8.0), parts=dict(factor=8.0, original_len=8192.0, low=1.0, high=4.0))[scaling]
    mode = dict(none=dd.DD_ROPE_NONE, linear=dd.DD_ROPE_LINEAR, ntk=dd.DD_ROPE_NTK, parts=dd.DD_ROPE_BY_PARTS)[scaling]
    args = {{"low": "low_turns", "high": "high_turns"}.get(k, k): v for k, v in kw.items()}
    r = dd.Rope(head_dim=d, rot_dim=rot, base=10000.0, layout=dd.DD_ROPE_HALF if layout == "half" else dd.DD_ROPE_INTERLEAVED,
                scaling=mode, amplitude=amplitude, **args)
    return r, ref.turns_of(rot, 10000.0, scaling, **kw)


# ---------------------------------------------------------------------------------------------- rotary positions
ROPE_CASES = [  # N, Hq, Hkv, d, rot, layout, type, scaling, amplitude, backward
    (1, 1, 1, 128, 128, "half", "bf16", "none", 1.0, False),
    (8, 32, 8, 128, 128, "half", "bf16", "parts", 1.2, False),
    (37, 5, 1, 128, 64, "interleaved", "fp16", "ntk", 1.0, True),
    (300, 4, 2, 64, 16, "half", "fp16", "linear", 0.5, False),
    (65, 3, 3, 64, 64, "interleaved", "bf16", "none", 1.0, False),
    (1000, 8, 1, 128, 32, "half", "bf16", "none", 1.0, True),
    (2500, 40, 8, 128, 128, "interleaved", "bf16", "parts", 1.0, False),
]


@pytest.mark.parametrize("N,Hq,Hkv,d,rot,layout,kind,scaling,amplitude,backward", ROPE_CASES)
def test_rope_matches_its_definition(dd, N, Hq, Hkv, d, rot, layout, kind, scaling, amplitude, backward):
    g = torch.Generator().manual_seed(N * 7 + d)
    x = torch.randn(N, Hq + 2 * Hkv, d, generator=g).to(TYPES[kind]).cuda()
    q, k = x[:, :Hq], x[:, Hq:Hq + Hkv]                             # slices of one projection
    pos = torch.randint(0, 1 << 22, (N,), generator=g).to(torch.int32)
    pos[0] = 2 ** 31 - 1
    if N > 3:
        pos[1], pos[2], pos[3] = 0, 1, -1                            # a padding token
    r, turns = rope_of(dd, d, rot, layout, scaling, amplitude)
    q_out, k_out = torch.full((N, Hq, d), 7.0, dtype=TYPES[kind], device="cuda"), torch.full((N, Hkv, d), 7.0, dtype=TYPES[kind], device="cuda")
    r.apply(pos.cuda(), q, k, q_out, k_out, backward=backward)
    for src, got in ((q, q_out), (k, k_out)):
        want = ref.rotate(f64(src), pos.numpy(), turns, layout, amplitude, backward)
        # sine and cosine 2 ulp each, their correction, two products and a sum: below 2^-21 of the pair's magnitude
        mag = np.abs(f64(src)).max() * 2 * abs(amplitude)
        got = f64(got)
        live = pos.numpy() >= 0
        assert np.all(np.abs(got - want)[live] <= STEP[kind] * np.abs(want)[live] + 2.0 ** -21 * mag + TINY[kind])
        assert np.all(got[~live] == 7.0)
        if rot < d:
            assert np.array_equal(got[live][..., rot:], f64(src)[live][..., rot:])
    # in place gives the same bits; so does q or k alone
    q2, k2 = q.clone(), k.clone()
    r.apply(pos.cuda(), q2, k2, backward=backward)
    live = pos >= 0
    assert torch.equal(q2[live], q_out[live]) and torch.equal(k2[live], k_out[live]) and torch.equal(q2[~live], q[~live])
    only = torch.full_like(k_out, 7.0)
    r.apply(pos.cuda(), None, k, None, only, backward=backward)
    assert torch.equal(only, k_out)


def test_rope_backward_is_the_gradient(dd):
    """<g, rope(x)> changes by <rope_backward(g), dx> for a change dx of x: exact but for the roundings of the two results."""
    N, H, d = 50, 4, 128
    gen = torch.Generator().manual_seed(3)
    x, gr, dx = (torch.randn(N, H, d, generator=gen).to(torch.float16).cuda() for _ in range(3))
    pos = torch.randint(0, 100000, (N,), generator=gen).to(torch.int32).cuda()
    r, turns = rope_of(dd, d, 64, "half", "parts", 1.3)
    grad = torch.empty_like(x)
    r.apply(pos, gr, None, grad, None, backward=True)
    for h in (1.0, -0.5):
        y0 = ref.rotate(f64(x), pos.cpu().numpy(), turns, "half", 1.3)
        y1 = ref.rotate(f64(x) + h * f64(dx), pos.cpu().numpy(), turns, "half", 1.3)
        want = ((y1 - y0) * f64(gr)).sum(-1) / h
        got = (f64(grad) * f64(dx)).sum(-1)
        bound = ((STEP["fp16"] + 2.0 ** -20) * np.abs(f64(grad)) * np.abs(f64(dx))).sum(-1) + 2.0 ** -20 * np.abs(f64(dx)).sum(-1) * 5
        assert np.all(np.abs(got - want) <= bound)


# ---------------------------------------------------------------------------------------------- writing and reading back
def random_pages(gen, n, H, fmt, T, d, gain=1.0):
    v = torch.randn(n, H, 2, T, d, generator=gen) * gain
    if fmt != "e4m3":
        return ref.encode_pages(v.to(TYPES[fmt]).double().numpy(), fmt)
    return ref.encode_pages(v.to(torch.bfloat16).double().numpy(), fmt)


def pool_of(raw, gap=0, pinned=False):
    """The pages uint8 [n, H, bytes] on the device (or page-locked), with a gap of `gap` bytes behind every page."""
    n, H, size = raw.shape
    t = torch.full((n, H, size + gap), 0xA5, dtype=torch.uint8)
    t[:, :, :size] = torch.from_numpy(raw)
    t = t.pin_memory() if pinned else t.cuda()
    return t, t[:, :, :size]


SPECIAL = [0.0, -0.0, 448.0, -449.0, 1.75, 1.7578125, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -11, 21.0, 1e-30, 2.0 ** -133, 3e38, -3e38]


@pytest.mark.parametrize("fmt,kind,T,d,H,gap,pinned", [
    ("e4m3", "bf16", 16, 128, 2, 0, False), ("e4m3", "fp16", 64, 64, 3, 48, False), ("e4m3", "bf16", 32, 64, 1, 0, True),
    ("bf16", "bf16", 16, 128, 2, 16, False), ("fp16", "fp16", 256, 64, 1, 0, False), ("bf16", "bf16", 16, 128, 8, 0, True)])
def test_append_writes_the_defined_bytes_and_nothing_else(dd, fmt, kind, T, d, H, gap, pinned):
    gen = torch.Generator().manual_seed(T + d)
    B, M, N = 3, 4, 41
    raw = random_pages(gen, B * M + 2, H, fmt, T, d)
    whole, pool = pool_of(raw, gap, pinned)
    table = torch.randperm(B * M + 2, generator=gen)[:B * M].view(B, M).to(torch.int32)
    table[1, 3] = -1                                                # pages that do not exist
    table[2, 3] = B * M + 2
    x = torch.randn(N, 2 * H, d, generator=gen) * torch.exp2(torch.randint(-12, 12, (N, 2 * H, 1), generator=gen).float())
    if kind == "bf16":
        for i, s in enumerate(SPECIAL):
            x[i, :, i % d] = s
    x[20] = 0.0
    x[21, 0, 3], x[21, 1, 5], x[22, 0, :] = float("inf"), float("nan"), float("-inf")
    x = x.to(TYPES[kind]).cuda()
    k, v = x[:, :H], x[:, H:]
    place = torch.randperm(B * M * T, generator=gen)[:N]
    req, pos = (place // (M * T)).to(torch.int32), (place % (M * T)).to(torch.int32)
    pos[30] = -1                                                    # padding
    req[31], req[32] = -1, B                                        # requests that do not exist
    pos[33] = M * T                                                 # behind the table
    cache = dd.PagedCache(pool, table.cuda(), cache_format=fmt_code(dd, fmt), head_dim=d, page_tokens=T)
    cache.append(k, v, pos.cuda(), req.cuda())
    torch.cuda.synchronize()
    want = raw.copy()
    skipped = 0
    for n in range(N):
        b, p = int(req[n]), int(pos[n])
        if p < 0 or b < 0 or b >= B or p >= M * T or not 0 <= int(table[b, p // T]) < B * M + 2:
            skipped += p >= 0
            continue
        blk, off = int(table[b, p // T]), p % T
        for h in range(H):
            for kv, src in ((0, k), (1, v)):
                row = f64(src[n, h])
                if fmt == "e4m3":
                    code, ex = ref.quantise(row)
                    want[blk, h, (kv * T + off) * d:(kv * T + off + 1) * d] = code
                    want[blk, h, 2 * T * d + kv * T + off] = ex
                else:
                    want[blk, h, (kv * T + off) * 2 * d:(kv * T + off + 1) * 2 * d] = src[n, h].cpu().view(torch.uint8).numpy()
    got = whole.cpu().numpy()
    assert np.array_equal(got[:, :, :want.shape[2]], want)
    assert np.all(got[:, :, want.shape[2]:] == 0xA5)
    code, detail = cache.device_error()
    assert skipped >= 3 and code == dd.DD_ERR_INDEX_RANGE
    bad = {-1, B, M, B * M + 2}
    assert detail in bad
    assert cache.device_error() == (0, 0)


@pytest.mark.parametrize("fmt,kind,d,rot,layout", [("e4m3", "bf16", 128, 128, "half"), ("e4m3", "fp16", 64, 32, "interleaved"), ("bf16", "bf16", 128, 64, "interleaved"),
                                                   ("fp16", "fp16", 64, 64, "half")])
def test_append_turns_keys_and_queries_on_the_way(dd, fmt, kind, d, rot, layout):
    gen = torch.Generator().manual_seed(d + rot)
    B, H, G, T, M, per = 3, 2, 4, 16, 8, 33
    raw = random_pages(gen, B * M, H, fmt, T, d)
    whole, pool = pool_of(raw)
    table = torch.randperm(B * M, generator=gen).view(B, M).to(torch.int32)
    x = torch.randn(B * per, H * G + 2 * H, d, generator=gen).to(TYPES[kind]).cuda()
    q, k, v = x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:]
    pos = torch.stack([torch.randperm(M * T, generator=gen)[:per] for _ in range(B)]).to(torch.int32).flatten()
    r, turns = rope_of(dd, d, rot, layout, "parts", 1.1)
    cache = dd.PagedCache(pool, table.cuda(), cache_format=fmt_code(dd, fmt), head_dim=d, page_tokens=T)
    q_out = torch.empty_like(q)
    cache.append(k, v, pos.cuda(), rope=r, q=q, q_out=q_out)              # requests: 33 tokens of each in turn
    alone = torch.empty_like(q)
    r.apply(pos.cuda(), q, None, alone, None)
    assert torch.equal(alone, q_out)                                      # the same rotation in either call
    got = ref.decode_pages(whole.cpu().numpy(), fmt, T, d)
    want_k = ref.rotate(f64(k), pos.numpy(), turns, layout, 1.1)
    want_v = f64(v)
    fp32 = 2.0 ** -21 * 2 * 1.1 * np.abs(f64(k)).max()
    for n in range(B * per):
        blk, off = int(table[n // per, int(pos[n]) // T]), int(pos[n]) % T
        for h in range(H):
            for kv, want, slack in ((0, want_k[n, h], fp32), (1, want_v[n, h], 0.0)):
                here = got[blk, h, kv, off]
                if fmt == "e4m3":
                    scale = 2.0 ** math.ceil(math.log2((np.abs(want).max() + slack) / 448.0))
                    tol = 2.0 ** -4 * np.abs(want) + 2.0 ** -10 * scale + slack * 1.1
                else:
                    tol = STEP[kind] * np.abs(want) + slack + TINY[kind]
                assert np.all(np.abs(here - want) <= tol), (n, h, kv)


@pytest.mark.parametrize("fmt,out,T,d,H,k,pinned", [
    ("e4m3", "bf16", 16, 128, 8, 7, False), ("e4m3", "fp16", 64, 64, 2, 3, False), ("bf16", "bf16", 16, 128, 2, 5, True), ("e4m3", "bf16", 16, 128, 4, 60, True), ("e4m3", "fp16", 32, 64, 3, 9, True), ("e4m3", "bf16", 64, 128, 1, 4, True),
    ("fp16", "fp16", 32, 64, 1, 1, False), ("bf16", "bf16", 256, 128, 1, 2, False), ("e4m3", "fp16", 128, 128, 1, 9, False)])
def test_read_brings_back_what_the_pages_stand_for(dd, fmt, out, T, d, H, k, pinned):
    gen = torch.Generator().manual_seed(T * d + k)
    B, M = 2, 64 if k > 10 else 12
    raw = random_pages(gen, B * M, H, fmt, T, d, gain=3.0)
    if fmt == "e4m3":                                             # scales over the whole range, and codes of every value but NaN
        raw[0, 0, :2 * T * d] = (np.arange(2 * T * d) % 254 + (np.arange(2 * T * d) % 254 >= 127)).astype(np.uint8)
        raw[0, 0, 2 * T * d:] = np.arange(2 * T) * 7 % 240 if out == "bf16" else 120 + np.arange(2 * T) % 9
    _, pool = pool_of(raw, 32, pinned)
    table = torch.randperm(B * M, generator=gen).view(B, M).to(torch.int32)
    table[0, 0] = 0
    table[1, 1] = B * M
    idx = torch.stack([torch.stack([torch.randperm(M, generator=gen)[:k] for _ in range(H)]) for _ in range(B)]).to(torch.int32)
    idx[0, 0, 0] = 0
    if k > 2:
        idx[0, 0, 1], idx[1, 0, 1], idx[1, 0, 2] = M, 1, -1       # out of range, a table entry out of range, negative
        idx[0, 0, 2] = 0                                          # the same page twice
    else:
        table[1, 1] = 5
    cache = dd.PagedCache(pool, table.cuda(), cache_format=fmt_code(dd, fmt), head_dim=d, page_tokens=T)
    got = torch.full((B, H, 2, k * T, d), 7.0, dtype=TYPES[out], device="cuda")
    cache.read(idx.cuda(), got)
    torch.cuda.synchronize()
    want = torch.zeros(B, H, 2, k * T, d, dtype=TYPES[out])
    for b in range(B):
        for h in range(H):
            for j in range(k):
                p = int(idx[b, h, j])
                blk = int(table[b, p]) if 0 <= p < M else -1
                if 0 <= blk < B * M:
                    v = ref.decode_pages(raw[blk, h], fmt, T, d)
                    want[b, h, :, j * T:(j + 1) * T] = torch.from_numpy(v).to(TYPES[out])
    assert torch.equal(got.cpu().view(torch.int16), want.view(torch.int16))
    code, detail = cache.device_error()
    if k > 2:
        assert code == dd.DD_ERR_INDEX_RANGE and detail in (M, -1, B * M)
    else:
        assert code == 0


# ---------------------------------------------------------------------------------------------- attention
def make_attn(dd, gen, lens, H, G, d, T, fmt, kind, Tq, gap=0, poison=True, shared=False, gain=1.5):
    """A cache whose pages behind each request's end hold NaN patterns, and queries."""
    B = len(lens)
    need = [max(0, -(-n // T)) for n in lens]
    M = max(1, max(need)) + 1
    total = sum(need) + 1
    raw = random_pages(gen, total, H, fmt, T, d, gain)
    table = torch.full((B, M), -7, dtype=torch.int32)             # entries behind the end are never read
    order = torch.randperm(total, generator=gen).to(torch.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    if shared and B > 1:                                          # requests that share their first pages
        m = min(need[0], need[1]) // 2
        table[1, :m] = table[0, :m]
    if poison:
        for b, n in enumerate(lens):
            if n > 0 and n % T:
                blk, off = int(table[b, need[b] - 1]), n % T
                if fmt == "e4m3":
                    page = raw[blk]
                    for kv in range(2):
                        page[:, (kv * T + off) * d:(kv + 1) * T * d] = 0x7f
                        page[:, 2 * T * d + kv * T + off:2 * T * d + (kv + 1) * T] = 255
                else:
                    for kv in range(2):
                        raw[blk][:, (kv * T + off) * 2 * d:(kv + 1) * T * 2 * d] = 0xff
    whole, pool = pool_of(raw, gap)
    cache = dd.PagedCache(pool, table.cuda(), cache_format=fmt_code(dd, fmt), head_dim=d, page_tokens=T)
    q = torch.randn(B, Tq, H * G, d, generator=gen).to(TYPES[kind]).cuda()
    return cache, raw, table, q


def check_attn(got, lse, q, raw, table, lens, fmt, kind, T, window=0, scale=None):
    d = q.shape[-1]
    want, want_lse, absum, unit = ref.attention(f64(q), raw, table.numpy(), lens, fmt, T, window, scale)
    # a score: 128 products added in fp32 in some order (each addition off by 2^-24 of a partial sum, at most sum |q||k|),
    # a multiplication by the scale and by log2 e; twice, since the weight and the denominator both carry it
    dz = (d + 8) * 2.0 ** -24 * unit + 2.0 ** -21 * (1 + np.where(np.isfinite(want_lse), np.abs(want_lse), 0.0))
    weight = STEP["bf16"] if fmt == "bf16" else STEP["fp16"]
    n_max = max(1, max(lens))
    rel = weight + 2 * dz + n_max * 2.0 ** -31 * 4 + 2.0 ** -16
    tol = STEP[kind] * np.abs(want) + rel[..., None] * (1 + STEP[kind]) * np.maximum(absum, absum.max(-1, keepdims=True) * 2.0 ** -10) + TINY[kind]
    g = f64(got)
    # a result beyond the type's largest value (65504 for half) is its infinity; within the tolerance of it, either
    limit = torch.finfo(TYPES[kind]).max
    beyond = np.abs(want) > limit + tol
    assert np.all(g[beyond] == np.sign(want[beyond]) * np.inf)
    near = ~beyond & (np.abs(want) + tol > limit) & np.isinf(g)
    g = np.where(beyond | near, want, g)
    assert np.all(np.isfinite(g)), "a value behind the end of a request was used"
    worst = np.max((np.abs(g - want)) / tol)
    assert worst <= 1.0, f"{worst} times the bound"
    if lse is not None:
        l = f64(lse)
        empty = ~np.isfinite(want_lse)
        assert np.array_equal(empty, np.isneginf(l))
        assert np.all(np.abs(l[~empty] - want_lse[~empty]) <= (dz + 2.0 ** -20 + n_max * 2.0 ** -33)[~empty])
        assert np.all(g[empty] == 0.0)


def run_attn(cache, q, lens, window=0, scale=0.0, with_lse=True):
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:3], 7.0, dtype=torch.float32, device="cuda") if with_lse else None
    cache.decode_attn(q, torch.tensor(lens, dtype=torch.int32).cuda(), out, lse, window=window, scale=scale)
    torch.cuda.synchronize()
    return out, lse


ATTN_CASES = [  # lens, H, G, d, T, fmt, query type, Tq, window
    ([1], 1, 1, 128, 16, "bf16", "bf16", 1, 0),
    ([5, 0, 16, 17, 1, 31], 2, 4, 128, 16, "e4m3", "bf16", 1, 0),
    ([5, 0, 16, 17, 1, 31], 2, 4, 128, 16, "bf16", "bf16", 2, 0),
    ([1000], 8, 4, 128, 16, "bf16", "bf16", 1, 0),
    ([4096, 4095], 8, 4, 128, 16, "e4m3", "bf16", 2, 0),
    ([777, 130, 2049], 2, 8, 128, 32, "e4m3", "fp16", 1, 0),
    ([777, 130, 2049], 2, 8, 64, 64, "fp16", "fp16", 2, 0),
    ([300, 299, 64, 3], 1, 5, 64, 16, "e4m3", "bf16", 3, 0),
    ([300, 299, 64, 3], 3, 16, 128, 16, "bf16", "bf16", 1, 0),
    ([300, 299, 64, 3], 3, 16, 128, 16, "e4m3", "bf16", 2, 0),
    ([100, 2, 40], 2, 24, 64, 256, "bf16", "bf16", 1, 0),
    ([512, 90, 33], 1, 6, 128, 16, "fp16", "fp16", 7, 0),
    ([1000, 15, 200, 0], 2, 2, 128, 16, "bf16", "bf16", 2, 64),
    ([1000, 15, 200, 0], 2, 2, 64, 32, "e4m3", "fp16", 4, 17),
    ([1000, 15, 200, 0], 1, 8, 128, 16, "e4m3", "bf16", 1, 1),
    ([3000] + [7] * 40 + [0] * 300 + [900], 1, 4, 128, 16, "e4m3", "bf16", 1, 0),
    ([20000], 1, 1, 64, 128, "bf16", "bf16", 1, 0),
]


@pytest.mark.parametrize("lens,H,G,d,T,fmt,kind,Tq,window", ATTN_CASES)
def test_decode_attention_matches_its_definition(dd, lens, H, G, d, T, fmt, kind, Tq, window):
    gen = torch.Generator().manual_seed(sum(lens) + G)
    cache, raw, table, q = make_attn(dd, gen, lens, H, G, d, T, fmt, kind, Tq, gap=16 * (len(lens) % 2), shared=True)
    out, lse = run_attn(cache, q, lens, window)
    assert cache.device_error() == (0, 0)
    check_attn(out, lse, q, raw, table, lens, fmt, kind, T, window)
    again, _ = run_attn(cache, q, lens, window, with_lse=False)       # the same bits every time, with or without lse
    assert torch.equal(out, again)


def test_attention_of_many_shapes(dd):
    """Seeded random launch shapes."""
    rng = np.random.RandomState(5)
    for i in range(40):
        fmt = ["bf16", "fp16", "e4m3", "e4m3"][rng.randint(4)]
        kind = fmt if fmt != "e4m3" else ["bf16", "fp16"][rng.randint(2)]
        B, H, G, d, T = rng.randint(1, 6), rng.randint(1, 4), rng.randint(1, 12), [64, 128][rng.randint(2)], [16, 32, 64][rng.randint(3)]
        Tq, window = rng.randint(1, 4), [0, 0, int(rng.randint(1, 300))][rng.randint(3)]
        lens = [int(2 ** rng.uniform(0, 11)) - 1 for _ in range(B)]
        gen = torch.Generator().manual_seed(i)
        cache, raw, table, q = make_attn(dd, gen, lens, H, G, d, T, fmt, kind, Tq)
        scale = [0.0, 0.05][rng.randint(2)]
        out, lse = run_attn(cache, q, lens, window, scale)
        check_attn(out, lse, q, raw, table, lens, fmt, kind, T, window, scale or None)


def test_infinities_and_nan_reach_only_the_rows_that_see_them(dd):
    """The newest token's value holds an infinity and a NaN: the query token before it must not notice; a window hides an
    old one from everybody, or from the later query token only."""
    gen = torch.Generator().manual_seed(0)
    for fmt, kind in (("bf16", "bf16"), ("e4m3", "fp16")):
        lens, H, G, d, T, Tq = [100, 37], 2, 4, 128, 16, 2
        cache, raw, table, q = make_attn(dd, gen, lens, H, G, d, T, fmt, kind, Tq)
        clean = raw.copy()
        for b, n in enumerate(lens):
            for at in (n - 1, n - 22):                              # the last token, and one that the window ends at
                blk, off = int(table[b, at // T]), at % T
                if fmt == "e4m3":
                    raw[blk, :, (T + off) * d + 5] = 0x7f
                else:
                    raw[blk, :, ((T + off) * d + 5) * 2:((T + off) * d + 6) * 2] = np.frombuffer(np.uint16(0x7f80).tobytes(), np.uint8)
        cache.data.copy_(torch.from_numpy(raw).cuda())
        out, _ = run_attn(cache, q, lens, window=21)                # token 0 sees n-22 .. n-2, token 1 sees n-21 .. n-1
        assert bool(torch.isfinite(out[:, :, :, :5]).all()) and bool(torch.isfinite(out[:, :, :, 6:]).all())
        assert not bool(torch.isfinite(out[:, :, :, 5]).any())
        out, _ = run_attn(cache, q, lens, window=20)                # now n-22 is hidden from both
        assert bool(torch.isfinite(out[:, 0]).all()) and not bool(torch.isfinite(out[:, 1, :, 5]).any())
        want, _, _, _ = ref.attention(f64(q), clean, table.numpy(), lens, fmt, T, 20)
        assert np.abs(f64(out)[:, 0] - want[:, 0]).max() < 0.05


def test_weights_of_every_size(dd):
    """Scores whose spread leaves one token with all the weight, far apart scales of V, and equal scores."""
    gen = torch.Generator().manual_seed(9)
    H, G, d, T, n = 1, 4, 128, 16, 700
    for fmt, kind, gain in (("bf16", "bf16", 40.0), ("e4m3", "bf16", 40.0), ("fp16", "fp16", 40.0), ("e4m3", "fp16", 0.0)):
        cache, raw, table, q = make_attn(dd, gen, [n], H, G, d, T, fmt, kind, 1, poison=False, gain=gain)
        v = ref.decode_pages(raw, fmt, T, d)
        v[:, :, 1] = np.random.RandomState(1).randn(*v[:, :, 1].shape)
        spread = 30 if fmt != "fp16" else 6
        v[:, :, 1] *= np.exp2(np.random.RandomState(2).randint(-spread, spread, v[:, :, 1].shape[:-1]))[..., None]
        if fmt != "e4m3":
            v = torch.from_numpy(v).to(TYPES[fmt]).double().numpy()
        raw[:] = ref.encode_pages(v, fmt)
        cache.data.copy_(torch.from_numpy(raw).cuda())
        out, lse = run_attn(cache, q, [n])
        check_attn(out, lse, q, raw, table, [n], fmt, kind, T)
    # all values zero (the smallest exponent byte): zeros, and the right lse
    cache, raw, table, q = make_attn(dd, gen, [n], H, G, d, T, "e4m3", "bf16", 1, poison=False)
    v = ref.decode_pages(raw, "e4m3", T, d)
    v[:, :, 1] = 0.0
    raw[:] = ref.encode_pages(v, "e4m3")
    cache.data.copy_(torch.from_numpy(raw).cuda())
    out, lse = run_attn(cache, q, [n])
    check_attn(out, lse, q, raw, table, [n], "e4m3", "bf16", T)
    assert bool((out == 0).all())


def test_bad_lengths_and_tables_are_reported(dd):
    gen = torch.Generator().manual_seed(1)
    cache, raw, table, q = make_attn(dd, gen, [64, 64], 1, 4, 128, 16, "bf16", "bf16", 1)
    M = table.shape[1]
    out, lse = run_attn(cache, q, [-5, 64])
    assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, -5)
    check_attn(out, lse, q, raw, table, [0, 64], "bf16", "bf16", 16)
    cache.block_table[:, M - 1] = 0
    out, lse = run_attn(cache, q, [64, M * 16 + 1])
    assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, M * 16 + 1)
    check_attn(out, lse, q, raw, cache.block_table.cpu(), [64, M * 16], "bf16", "bf16", 16)
    for bad in (-1, raw.shape[0], 2 ** 31 - 1):
        keep = int(table[0, 1])
        cache.block_table[0, 1] = bad
        out, lse = run_attn(cache, q, [64, 64])
        assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, bad)
        zeros = np.concatenate([raw, np.zeros_like(raw[:1])])     # the page reads as zeros
        t = table.clone()
        t[0, 1] = raw.shape[0]
        check_attn(out, lse, q, zeros, t, [64, 64], "bf16", "bf16", 16)
        cache.block_table[0, 1] = keep


def test_strided_queries_and_outputs(dd):
    gen = torch.Generator().manual_seed(2)
    lens = [200, 33, 90]
    cache, raw, table, q = make_attn(dd, gen, lens, 2, 3, 64, 16, "e4m3", "bf16", 2)
    B, Tq, Hq, d = q.shape
    wide = torch.randn(B, Tq, Hq + 4, d, generator=gen).to(torch.bfloat16).cuda()
    wide[:, :, :Hq] = q
    room = torch.full((B, Tq, Hq + 1, d + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    out = room[:, :, :Hq, :d]
    cache.decode_attn(wide[:, :, :Hq], torch.tensor(lens, dtype=torch.int32).cuda(), out)
    check_attn(out, None, q, raw, table, lens, "e4m3", "bf16", 16)
    assert bool((room[:, :, Hq:] == 7.0).all()) and bool((room[..., d:] == 7.0).all())
    same = q[:1, :1].expand(B, Tq, Hq, d)                        # one query for everybody
    with pytest.raises(dd.DDError):
        cache.decode_attn(q, torch.tensor(lens, dtype=torch.int32).cuda(), same)      # rows of the output would overlap
    out2, out3 = torch.empty_like(q), torch.empty_like(q)
    cache.decode_attn(same, torch.tensor(lens, dtype=torch.int32).cuda(), out2)
    cache.decode_attn(same.contiguous(), torch.tensor(lens, dtype=torch.int32).cuda(), out3)
    assert torch.equal(out2, out3)


def test_workspace_too_small_and_wrong_memory_are_refused(dd):
    gen = torch.Generator().manual_seed(4)
    cache, raw, table, q = make_attn(dd, gen, [40], 1, 4, 128, 16, "bf16", "bf16", 1)
    lens = torch.tensor([40], dtype=torch.int32).cuda()
    out = torch.full_like(q, 7.0)
    need = cache.workspace(4).numel()
    with pytest.raises(dd.DDError) as e:
        cache.decode_attn(q, lens, out, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert str(need) in str(e.value)
    for kw in (dict(q=q.cpu()), dict(lens=lens.cpu()), dict(out=out.cpu()), dict(ws=torch.empty(need, dtype=torch.uint8)),
               dict(lse=torch.zeros(1, 1, 4))):
        with pytest.raises(dd.DDError) as e:
            cache.decode_attn(kw.get("q", q), kw.get("lens", lens), kw.get("out", out), kw.get("lse"), workspace=kw.get("ws"))
        assert e.value.code == dd.DD_ERR_INVALID_ARG
    pageable = dd.PagedCache(torch.from_numpy(raw), table.cuda(), head_dim=128)
    kv, pos = torch.zeros(1, 1, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for call in (lambda: pageable.append(kv, kv, pos), lambda: pageable.read(pos.view(1, 1, 1), torch.empty(1, 1, 2, 16, 128, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(dd.DDError) as e:
            call()
        assert e.value.code == dd.DD_ERR_NOT_PINNED
    pinned = dd.PagedCache(torch.from_numpy(raw).pin_memory(), table.cuda(), head_dim=128)
    with pytest.raises(dd.DDError):
        pinned.decode_attn(q, lens, out)
    off = torch.zeros(129, dtype=torch.bfloat16, device="cuda")[1:].view(1, 1, 128)
    with pytest.raises(dd.DDError):
        cache.append(off, kv, pos)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


# ---------------------------------------------------------------------------------------------- as they are used
def test_decode_steps_through_the_cache(dd):
    """Three decode steps of a batch: turn and append, attend, read the newest page back; every step against the
    definitions run on the cache's own bytes."""
    gen = torch.Generator().manual_seed(11)
    B, H, G, d, T, M = 3, 2, 4, 128, 16, 12
    raw = random_pages(gen, B * M, H, "e4m3", T, d)
    whole, pool = pool_of(raw)
    table = torch.randperm(B * M, generator=gen).view(B, M).to(torch.int32)
    cache = dd.PagedCache(pool, table.cuda(), cache_format=dd.DD_CACHE_E4M3, head_dim=d, page_tokens=T)
    r, turns = rope_of(dd, d, 128)
    lens = torch.tensor([15, 100, 0], dtype=torch.int32)
    for step in range(3):
        x = torch.randn(B, H * G + 2 * H, d, generator=gen).to(torch.bfloat16).cuda()
        q, k, v = x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:]
        turned = torch.empty(B, H * G, d, dtype=torch.bfloat16, device="cuda")
        cache.append(k, v, lens.cuda(), rope=r, q=q, q_out=turned)
        lens += 1
        out = torch.empty(B, 1, H * G, d, dtype=torch.bfloat16, device="cuda")
        lse = torch.empty(B, 1, H * G, device="cuda")
        cache.decode_attn(turned.view(B, 1, H * G, d), lens.cuda(), out, lse)
        now = whole.cpu().numpy()
        check_attn(out, lse, turned.view(B, 1, H * G, d), now, table, lens.tolist(), "e4m3", "bf16", T)
        last = ((lens - 1) // T).view(B, 1, 1).expand(B, H, 1).contiguous().cuda()
        back = torch.empty(B, H, 2, T, d, dtype=torch.bfloat16, device="cuda")
        cache.read(last, back)
        for b in range(B):
            off = int(lens[b] - 1) % T
            assert torch.equal(back[b, :, 1, off].double().cpu(), torch.from_numpy(ref.decode_pages(now[table[b, (int(lens[b]) - 1) // T]], "e4m3", T, d)[:, 1, off]))
            want = ref.rotate(f64(k[b:b + 1]), lens[b:b + 1].numpy() - 1, turns, "half")[0]
            assert np.all(np.abs(f64(back[b, :, 0, off]) - want) <= 2.0 ** -4 * np.abs(want) + 2.0 ** -10 * np.abs(want).max(-1, keepdims=True) / 224 + 1e-5)
    assert cache.device_error() == (0, 0)


@pytest.mark.parametrize("M", [5, 40, 600])                       # a warp a unit, clusters, the flat list
def test_captured_steps_replayed_with_other_lengths(dd, M):
    """Two graphs of the same cache hold an append and an attention each; replayed in turn with other lengths and rows
    than at capture, they give the eager calls' bits. The two graphs take workspaces of their own."""
    gen = torch.Generator().manual_seed(12)
    B, H, G, d, T = 4, 2, 4, 128, 16
    raw = random_pages(gen, B * M, H, "bf16", T, d)
    _, pool = pool_of(raw)
    table = torch.randperm(B * M, generator=gen).view(B, M).to(torch.int32).cuda()
    cache = dd.PagedCache(pool, table, head_dim=d, page_tokens=T)
    r, _ = rope_of(dd, d, 128)
    x = torch.zeros(B, H * G + 2 * H, d, dtype=torch.bfloat16, device="cuda")
    pos, lens = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.ones(B, dtype=torch.int32, device="cuda")
    turned, out = torch.empty(B, H * G, d, dtype=torch.bfloat16, device="cuda"), torch.empty(B, 1, H * G, d, dtype=torch.bfloat16, device="cuda")

    def step(out):
        cache.append(x[:, H * G:H * G + H], x[:, H * G + H:], pos, rope=r, q=x[:, :H * G], q_out=turned)
        cache.decode_attn(turned.view(B, 1, H * G, d), lens, out)

    step(out)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        o = torch.empty_like(out)
        gph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gph):
            step(o)
        graphs.append((gph, o))
    for rep in range(4):
        gph, o = graphs[rep % 2]
        x.copy_(torch.randn(x.shape, generator=gen).to(torch.bfloat16))
        p = torch.randint(0, M * T, (B,), generator=gen).to(torch.int32)
        pos.copy_(p)
        lens.copy_(p + 1)
        gph.replay()
        torch.cuda.synchronize()
        step(out)
        torch.cuda.synchronize()
        assert torch.equal(o, out)
    assert cache.device_error() == (0, 0)


def test_calls_on_several_streams_at_once(dd):
    gen = torch.Generator().manual_seed(13)
    lens = [3000, 100, 1, 700]
    cache, raw, table, q = make_attn(dd, gen, lens, 2, 4, 128, 16, "e4m3", "bf16", 1)
    l = torch.tensor(lens, dtype=torch.int32).cuda()
    want = torch.empty_like(q)
    cache.decode_attn(q, l, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = [torch.zeros_like(q) for _ in range(16)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        s = streams[i % 4]
        if i % 2:
            with torch.cuda.stream(s):
                cache.decode_attn(q, l, o)
        else:
            cache.decode_attn(q, l, o, stream=s if i % 4 else s.cuda_stream)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, want)


def test_a_layer_of_the_store_seen_as_a_cache(dd):
    """The method's store layout [B, Hkv, P, 2, T, d]: pages read through the cache are the pages that the sparse path
    gathers, and attention over all of it is the sparse attention with every page selected."""
    gen = torch.Generator().manual_seed(14)
    B, H, P, T, d, G = 2, 8, 24, 16, 128, 4
    kv = torch.randn(B, H, P, 2, T, d, generator=gen).to(torch.bfloat16)
    dev = kv.cuda()
    cache = dd.PagedCache.of_store(dev)
    idx = torch.stack([torch.stack([torch.randperm(P, generator=gen)[:9].sort().values for _ in range(H)]) for _ in range(B)]).to(torch.int32).cuda()
    ctx = dd.Context(n_layers=1, batch=B, max_pages=P, k_pages=9, n_q_tokens=1)
    ctx.gather_kv_from_host(kv.pin_memory(), idx, None, 0)
    got = torch.empty(B, H, 2, 9 * T, d, dtype=torch.bfloat16, device="cuda")
    cache.read(idx, got)
    assert torch.equal(got, ctx.slot_tensor(0))
    ctx.close()
    lens = torch.tensor([P * T, P * T - 21], dtype=torch.int32).cuda()
    every = torch.arange(P, dtype=torch.int32).expand(B, H, P).contiguous().cuda()
    ctx = dd.Context(n_layers=1, batch=B, max_pages=P, k_pages=P, n_q_tokens=1)
    ctx.gather_kv_from_host(dev, every, None, 0)
    q = torch.randn(B, 1, H * G, d, generator=gen).to(torch.bfloat16).cuda()
    sparse, full = torch.empty_like(q), torch.empty_like(q)
    ctx.sparse_decode_attn(q, 0, every, lens, sparse)
    cache.decode_attn(q, lens, full)
    ctx.close()
    # each side rounds its weights to bf16 and its result to bf16
    v = dev[:, :, :, 1].abs().amax().item()
    assert float((sparse.float() - full.float()).abs().max()) <= 2 * (2.0 ** -8 + 2.0 ** -8) * v
    raw = kv.contiguous().view(torch.uint8).reshape(B * H * P, 1, 8192).numpy()
    table = cache.block_table.cpu()
    flat = np.stack([raw[:, 0][h * P + np.arange((B - 1) * H * P + P)] for h in range(H)], 1)     # [block, head, bytes]
    check_attn(full, None, q, flat, table, lens.tolist(), "bf16", "bf16", T)


def test_offsets_beyond_32_bits(dd):
    """Pages at the far end of a pool of 4.8 GB: written, attended to and read back."""
    gen = torch.Generator().manual_seed(15)
    n, T, d, H, G = 580000, 16, 128, 2, 4
    pool = torch.empty(n, H, 4128, dtype=torch.uint8, device="cuda")
    assert pool.numel() > 1 << 32
    far = torch.tensor([[n - 1, n - 5, n - 3, n - 2], [0, n - 4, 1, 2]], dtype=torch.int32)
    wide = torch.full((2, 9), -1, dtype=torch.int32)               # a table with rows longer than the cache's
    wide[:, :4] = far
    cache = dd.PagedCache(pool, wide.cuda()[:, :4], cache_format=dd.DD_CACHE_E4M3)
    k, v = (torch.randn(2 * 64, H, d, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    cache.append(k, v, torch.arange(64, dtype=torch.int32).repeat(2).cuda())
    q = torch.randn(2, 1, H * G, d, generator=gen).to(torch.bfloat16).cuda()
    out, lse = run_attn(cache, q, [64, 49])
    used = far.flatten().long()
    raw = pool[used.cuda()].cpu().numpy()
    table = torch.arange(8).view(2, 4)
    for i in range(8):
        want = torch.stack([k.view(2, 4, T, H, d)[i // 4, i % 4], v.view(2, 4, T, H, d)[i // 4, i % 4]], 0)     # [2, T, H, d]
        for h in range(H):
            assert np.array_equal(raw[i, h], ref.encode_pages(f64(want[:, :, h]), "e4m3"))
    check_attn(out, lse, q, raw, table, [64, 49], "e4m3", "bf16", T)
    idx = torch.arange(4, dtype=torch.int32).expand(2, H, 4).contiguous().cuda()
    back = torch.empty(2, H, 2, 64, d, dtype=torch.bfloat16, device="cuda")
    cache.read(idx, back)
    want = ref.decode_pages(raw.reshape(2, 4, H, 4128), "e4m3", T, d).transpose(0, 2, 3, 1, 4, 5).reshape(2, H, 2, 64, d)
    assert np.array_equal(f64(back), want)
    assert cache.device_error() == (0, 0)


def test_output_in_place_of_the_queries(dd):
    """Every row of the queries is read before its place is written, whichever way the work is split."""
    gen = torch.Generator().manual_seed(16)
    for lens, H, G in (([4000, 17, 0], 2, 4), ([100, 90], 1, 8), ([3000] * 12, 8, 4)):
        cache, raw, table, q = make_attn(dd, gen, lens, H, G, 128, 16, "bf16", "bf16", 1)
        l = torch.tensor(lens, dtype=torch.int32).cuda()
        out = torch.empty_like(q)
        cache.decode_attn(q, l, out)
        same = q.clone()
        cache.decode_attn(same, l, same)
        assert torch.equal(out, same)


def test_every_way_to_split_the_work_gives_the_definition(dd):
    """Table widths on both sides of each rule: one warp a unit, clusters of 2, 4 and 8 blocks, the flat list; few units and many;
    lengths below what the table could hold."""
    gen = torch.Generator().manual_seed(17)
    for lens, H, G, Tq, fmt in (([128], 1, 4, 1, "bf16"), ([129, 3], 1, 4, 2, "bf16"), ([512], 2, 3, 1, "e4m3"), ([513, 5], 1, 16, 1, "bf16"), ([1025], 4, 8, 1, "e4m3"),
                                ([4096, 0, 33], 1, 2, 3, "bf16"), ([8192], 1, 4, 1, "e4m3"), ([8193], 1, 4, 1, "e4m3"), ([700] * 40, 2, 4, 1, "bf16"),
                                ([2000] * 9, 2, 24, 1, "e4m3")):
        cache, raw, table, q = make_attn(dd, gen, lens, H, G, 128, 16, fmt, "bf16", Tq)
        out, lse = run_attn(cache, q, lens)
        check_attn(out, lse, q, raw, table, lens, fmt, "bf16", 16)
        short = [max(0, n - 300) for n in lens]
        out, lse = run_attn(cache, q, short)
        keep = raw.copy()
        check_attn(out, lse, q, keep, table, short, fmt, "bf16", 16)
        assert cache.device_error() == (0, 0)


@pytest.mark.parametrize("fmt,kind,Tq", [("e4m3", "bf16", 1), ("e4m3", "fp16", 2), ("bf16", "bf16", 1)])
def test_long_requests_over_few_pages(dd, fmt, kind, Tq):
    """A request of 1.25 million tokens whose table names 61 pages over and over: the definition is attention over the 61
    pages' tokens, each weighted by how often it is seen."""
    gen = torch.Generator().manual_seed(18)
    T, d, H, G, n_pages, M = 16, 128, 1, 4, 61, 78200
    lens = M * T - 5
    raw = random_pages(gen, n_pages, H, fmt, T, d, gain=1.5)
    _, pool = pool_of(raw)
    table = (torch.arange(M, dtype=torch.int32) * 7 % n_pages).view(1, M)
    cache = dd.PagedCache(pool, table.cuda(), cache_format=fmt_code(dd, fmt), head_dim=d, page_tokens=T)
    q = torch.randn(1, Tq, G, d, generator=gen).to(TYPES[kind]).cuda()
    out, lse = run_attn(cache, q, [lens])
    again, _ = run_attn(cache, q, [lens])
    assert torch.equal(out, again) and cache.device_error() == (0, 0)
    kv = ref.decode_pages(raw[:, 0], fmt, T, d)                     # [pages, 2, T, d]
    K, V = kv[:, 0].reshape(-1, d), kv[:, 1].reshape(-1, d)
    for t in range(Tq):
        seen = np.zeros((n_pages, T))
        end = lens - Tq + t + 1
        np.add.at(seen, table[0, :end // T].numpy(), 1.0)
        seen[int(table[0, end // T]), :end % T] += 1.0
        for h in range(G):
            row = f64(q[0, t, h])
            z = K @ row / math.sqrt(d)
            p = np.exp(z - z.max()) * seen.reshape(-1)
            want_lse = z.max() + math.log(p.sum())
            p /= p.sum()
            want, absum = p @ V, p @ np.abs(V)
            unit = (np.abs(K) @ np.abs(row)).max() / math.sqrt(d)
            # as for shorter requests; a warp adds up to 40 tiles before its sums are merged, 2048 merges of fp32 partials follow
            dz = (d + 8) * 2.0 ** -24 * unit + 2.0 ** -21 * (1 + abs(want_lse))
            rel = (STEP["bf16"] if fmt == "bf16" else STEP["fp16"]) + 2 * dz + lens * 2.0 ** -31 * 4 + 2.0 ** -12
            tol = STEP[kind] * np.abs(want) + rel * np.maximum(absum, absum.max() * 2.0 ** -10)
            assert np.all(np.abs(f64(out[0, t, h]) - want) <= tol)
            assert abs(float(lse[0, t, h]) - want_lse) <= dz + 2.0 ** -12
