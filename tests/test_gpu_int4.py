"""The 4-bit cache: bytes written, values read back, attention over it, against plain 64-bit definitions."""
import numpy as np
import pytest
import torch

from tests import _cache_ref as ref
from tests import _int4_ref as ref4
from tests._cache_ref import f64
from tests._int4_ref import BITS, TINY, TYPES, check
from tests.test_gpu_cache import SPECIAL, dd, pool_of, rope_of  # noqa: F401  (dd is the fixture)

pytestmark = pytest.mark.gpu


def random_pages(gen, n, H, fmt, T, d, gain=1.0):
    v = torch.randn(n, H, 2, T, d, generator=gen) * gain
    return ref4.encode_pages(v.to(TYPES[fmt] if fmt in TYPES else torch.bfloat16).double().numpy(), fmt)


def format_code(dd, fmt):
    return {"bf16": dd.DD_CACHE_BF16, "fp16": dd.DD_CACHE_FP16, "e4m3": dd.DD_CACHE_E4M3, "int4": dd.DD_CACHE_INT4}[fmt]


def poison(raw, blk, off, fmt, T, d):
    """Tokens from `off` on of a page hold the bits that would do the most harm."""
    page = raw[blk]
    if fmt == "int4":
        code, _, scale, ex = ref4.places(T, d)
        page[:, np.unique(code[:, off:])] = 0xff
        page[:, np.unique(scale[:, off:])] = 0x7f
        page[:, np.unique(ex[:, off:])] = 255
    elif fmt == "e4m3":
        for kv in range(2):
            page[:, (kv * T + off) * d:(kv + 1) * T * d] = 0x7f
            page[:, 2 * T * d + kv * T + off:2 * T * d + (kv + 1) * T] = 255
    else:
        for kv in range(2):
            page[:, (kv * T + off) * 2 * d:(kv + 1) * T * 2 * d] = 0xff


def make(dd, gen, lens, H, d, T, fmt, gap=0, spare=1, gain=1.5, shared=False):
    """A cache whose pages behind each request's end are poisoned: (cache, raw pages, table)."""
    B, need = len(lens), [max(0, -(-n // T)) for n in lens]
    M, total = max(1, max(need)) + spare, sum(need) + 1
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
    for b, n in enumerate(lens):
        if n > 0 and n % T:
            poison(raw, int(table[b, need[b] - 1]), n % T, fmt, T, d)
    _, pool = pool_of(raw, gap)
    return dd.PagedCache(pool, table.cuda(), cache_format=format_code(dd, fmt), head_dim=d, page_tokens=T), raw, table


# ---------------------------------------------------------------------------------------------- writing and reading back
def put(want, blk, h, kv, off, x, T, d):
    """Row x of token `off` into a page of the definition."""
    code, shift, scale, ex = ref4.places(T, d)
    c, s, e = ref4.quantise(x)
    page = want[blk, h]
    for sh in (0, 4):
        m = shift[kv, off] == sh
        page[code[kv, off, m]] = (page[code[kv, off, m]] & (0xf0 if sh == 0 else 0x0f)) | (c[m] << sh)
    page[scale[kv, off, ::16]] = s
    page[ex[kv, off, 0]] = e


@pytest.mark.parametrize("kind,T,d,H,gap,pinned", [("bf16", 16, 128, 2, 0, False), ("fp16", 64, 64, 3, 48, False), ("bf16", 32, 64, 1, 0, True),
                                                   ("bf16", 256, 128, 1, 16, False), ("fp16", 16, 128, 8, 0, False)])
def test_append_writes_the_defined_bytes_and_nothing_else(dd, kind, T, d, H, gap, pinned):
    gen = torch.Generator().manual_seed(T + d)
    B, M, N = 3, 4, 61
    raw = random_pages(gen, B * M + 2, H, "int4", T, d)
    whole, pool = pool_of(raw, gap, pinned)
    table = torch.randperm(B * M + 2, generator=gen)[:B * M].view(B, M).to(torch.int32)
    table[1, 3], table[2, 3] = -1, B * M + 2                        # pages that do not exist
    x = torch.randn(N, 2 * H, d, generator=gen) * torch.exp2(torch.randint(-12, 12, (N, 2 * H, 1), generator=gen).float())
    if kind == "bf16":
        for i, s in enumerate(SPECIAL):
            x[i, :, i % d] = s
    x[20] = 0.0
    x[21, 0, 3], x[21, 1, 5], x[22, 0, :] = float("inf"), float("nan"), float("-inf")
    # every border: multiples of half a step up to the largest, for a scale that is exact
    x[23:40] = (torch.arange(d).remainder(29) - 14).float() / 2 * torch.exp2(torch.arange(17).float() - 8).view(-1, 1, 1)
    x[23:40, :, ::16] = (7 * torch.exp2(torch.arange(17).float() - 8)).view(-1, 1, 1)
    # sevenths on the borders of the scale's own rounding
    x[40:50] *= 2.0 ** -6
    x[40:50, :, ::16] = (7 * (1 + (2 * torch.arange(10) + 1) / 16.0)).view(-1, 1, 1)
    x = x.to(TYPES[kind]).cuda()
    k, v = x[:, :H], x[:, H:]
    place = torch.randperm(B * M * T, generator=gen)[:N]
    req, pos = (place // (M * T)).to(torch.int32), (place % (M * T)).to(torch.int32)
    pos[50], req[51], req[52], pos[53] = -1, -1, B, M * T          # padding; requests and a place that do not exist
    cache = dd.PagedCache(pool, table.cuda(), cache_format=dd.DD_CACHE_INT4, head_dim=d, page_tokens=T)
    cache.append(k, v, pos.cuda(), req.cuda())
    torch.cuda.synchronize()
    want = raw.copy()
    for n in range(N):
        b, p = int(req[n]), int(pos[n])
        if 0 <= p < M * T and 0 <= b < B and 0 <= int(table[b, p // T]) < B * M + 2:
            for h in range(H):
                put(want, int(table[b, p // T]), h, 0, p % T, f64(k[n, h]), T, d)
                put(want, int(table[b, p // T]), h, 1, p % T, f64(v[n, h]), T, d)
    got = whole.cpu().numpy()
    assert np.array_equal(got[:, :, :want.shape[2]], want)
    assert np.all(got[:, :, want.shape[2]:] == 0xA5)
    code, detail = cache.device_error()
    assert code == dd.DD_ERR_INDEX_RANGE and detail in {-1, B, M, B * M + 2}
    assert cache.device_error() == (0, 0)


@pytest.mark.parametrize("kind,d,rot,layout,far", [("bf16", 128, 128, "half", 128), ("fp16", 64, 32, "interleaved", 128), ("bf16", 128, 48, "half", 128),
                                                   ("bf16", 64, 16, "half", 128), ("fp16", 128, 64, "half", 1 << 21), ("bf16", 128, 128, "interleaved", 1 << 21)])
def test_turned_keys_are_held_as_the_64_bit_rotation_says(dd, kind, d, rot, layout, far):
    """Byte for byte, over enough rows to meet borders that the 32-bit rotation misses."""
    gen = torch.Generator().manual_seed(d + rot)
    H, G, T, N = 2, 4, 16, 4000
    M = far // T
    # one request whose table repeats a few blocks: tokens go to places of their own, at positions far apart
    blocks = N // T
    where = torch.randperm(min(M, 1 << 15), generator=gen)[:blocks]
    table = torch.zeros(1, M, dtype=torch.int32)
    if blocks <= M:
        pages = torch.randperm(M, generator=gen)[:blocks]
        table[0, pages] = torch.arange(blocks, dtype=torch.int32)
        pos = (pages.view(-1, 1) * T + torch.arange(T)).flatten().to(torch.int32)
        req = torch.zeros(N, dtype=torch.int32)
    else:                                                          # several requests of few pages
        B = -(-blocks // M)
        table = torch.arange(B * M, dtype=torch.int32).view(B, M)
        blocks = B * M
        pos = (torch.arange(N) % (M * T)).to(torch.int32)
        req = (torch.arange(N) // (M * T)).to(torch.int32)
    del where
    raw = np.zeros((blocks, H, ref4.page_bytes("int4", T, d)), dtype=np.uint8)
    whole, pool = pool_of(raw)
    x = torch.randn(N, H * G + 2 * H, d, generator=gen).to(TYPES[kind]).cuda()
    q, k, v = x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:]
    r, turns = rope_of(dd, d, rot, layout, "parts", 1.1)
    cache = dd.PagedCache(pool, table.cuda(), cache_format=dd.DD_CACHE_INT4, head_dim=d, page_tokens=T)
    q_out, alone = torch.empty_like(q), torch.empty_like(q)
    cache.append(k, v, pos.cuda(), req.cuda(), rope=r, q=q, q_out=q_out)
    r.apply(pos.cuda(), q, None, alone, None)
    assert torch.equal(alone, q_out)                               # the same rotation in either call
    # the amplitude is a 32-bit number of the call
    want_k = ref.rotate(f64(k), pos.numpy(), turns, layout, float(np.float32(1.1)))
    got = whole.cpu().numpy()
    code, shift, scale, ex = ref4.places(T, d)
    blk, off = table[req.long(), pos.long() // T].numpy(), pos.numpy() % T
    differ = 0
    for kv, rows in ((0, want_k), (1, f64(v))):
        c, s, e = ref4.quantise(rows)
        for h in range(H):
            page = got[blk, h]                                     # [N, bytes]
            n = np.arange(N)[:, None]
            assert np.array_equal(page[n, ex[kv, off, :1]][:, 0], e[:, h])
            differ += int((page[n, scale[kv, off, ::16]] != s[:, h]).sum())
            differ += int(((page[n, code[kv, off]] >> shift[kv, off] & 15) != c[:, h]).sum())
    # what is left is the difference of two 64-bit rotations (2^-50 of a step): none of 2 million codes
    assert differ == 0


@pytest.mark.parametrize("out,T,d,H,k,pinned", [("bf16", 16, 128, 2, 5, False), ("fp16", 64, 64, 3, 4, False), ("bf16", 256, 64, 1, 3, True), ("bf16", 16, 128, 8, 1, False)])
def test_read_brings_back_what_the_pages_stand_for(dd, out, T, d, H, k, pinned):
    gen = torch.Generator().manual_seed(T + k)
    B, M = 2, 6
    raw = random_pages(gen, B * M, H, "int4", T, d)
    code, _, scale, ex = ref4.places(T, d)
    raw[3][:, np.unique(code)] = np.arange(T * d, dtype=np.uint8)     # every pair of nibbles
    raw[4][:, np.unique(scale)] = np.arange(len(np.unique(scale)), dtype=np.uint8)   # every scale, NaN codes among them
    if out == "bf16":
        raw[5][:, np.unique(ex)] = (np.arange(2 * T, dtype=np.int64) * 37 % 240 + 1).astype(np.uint8)
    whole, pool = pool_of(raw, 32, pinned)
    table = torch.arange(B * M, dtype=torch.int32).view(B, M)
    table[1, 2] = B * M
    idx = torch.randint(0, M, (B, H, k), generator=gen).to(torch.int32)
    idx[0, 0, :min(k, 3)] = torch.tensor([3, 4, 5])[:min(k, 3)]
    if k > 3:
        idx[1, 0, 0], idx[1, 0, 1], idx[1, H - 1, 2] = 2, M, -1
    cache = dd.PagedCache(pool, table.cuda(), cache_format=dd.DD_CACHE_INT4, head_dim=d, page_tokens=T)
    got = torch.full((B, H, 2, k * T, d), 7.0, dtype=TYPES[out], device="cuda")
    cache.read(idx.cuda(), got)
    torch.cuda.synchronize()
    want = np.zeros((B, H, 2, k * T, d))
    for b in range(B):
        for h in range(H):
            for j in range(k):
                p = int(idx[b, h, j])
                blk = int(table[b, p]) if 0 <= p < M else -1
                if 0 <= blk < B * M:
                    want[b, h, :, j * T:(j + 1) * T] = ref4.decode_pages(raw[blk, h], "int4", T, d)
    got = f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    rounded = torch.from_numpy(want).to(TYPES[out]).double().numpy()
    assert np.array_equal(got[fine], rounded[fine])
    code, detail = cache.device_error()
    assert (code == dd.DD_ERR_INDEX_RANGE and detail in (M, -1, B * M)) if k > 3 else code in (0, dd.DD_ERR_INDEX_RANGE)


# ---------------------------------------------------------------------------------------------- attention
def run_attn(cache, q, lens, window=0, scale=0.0, with_lse=True):
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:3], 7.0, dtype=torch.float32, device="cuda") if with_lse else None
    cache.decode_attn(q, torch.tensor(lens, dtype=torch.int32).cuda(), out, lse, window=window, scale=scale)
    torch.cuda.synchronize()
    return out, lse


def check_attn(out, lse, q, raw, table, lens, kind, T, window=0, scale=None):
    check(out, lse, *ref4.attention(f64(q), raw, table.numpy(), lens, "int4", T, window, scale), "int4", kind, max(1, max(lens)))


def queries(gen, B, Tq, Hq, d, kind):
    return torch.randn(B, Tq, Hq, d, generator=gen).to(TYPES[kind]).cuda()


ATTN = [  # lens, H, G, d, T, query type, Tq, window, scale
    ([1], 1, 1, 128, 16, "bf16", 1, 0, 0.0),
    ([5, 0, 16, 17, 1, 31], 2, 4, 128, 16, "bf16", 1, 0, 0.0),
    ([5, 0, 16, 17, 1, 31], 2, 4, 64, 16, "fp16", 2, 0, 0.02),
    ([1000], 8, 4, 128, 16, "bf16", 1, 0, 0.0),
    ([4096, 4095], 8, 4, 128, 16, "bf16", 2, 0, 0.0),
    ([777, 130, 2049], 2, 8, 128, 32, "fp16", 1, 0, 0.02),
    ([777, 130, 2049], 2, 8, 64, 64, "bf16", 2, 0, 0.0),
    ([300, 299, 64, 3], 1, 5, 64, 16, "bf16", 3, 0, 0.0),
    ([300, 299, 64, 3], 3, 16, 128, 16, "bf16", 2, 0, 0.3),
    ([100, 2, 40], 2, 24, 64, 256, "fp16", 1, 0, 0.02),
    ([512, 90, 33], 1, 6, 128, 128, "bf16", 7, 0, 0.0),
    ([1000, 15, 200, 0], 2, 2, 128, 16, "bf16", 2, 64, 0.0),
    ([1000, 15, 200, 0], 2, 2, 64, 32, "fp16", 4, 17, 0.02),
    ([1000, 15, 200, 0], 1, 8, 128, 16, "bf16", 1, 1, 0.0),
    ([3000] + [7] * 40 + [0] * 300 + [900], 1, 4, 128, 16, "bf16", 1, 0, 0.0),
    ([20000], 1, 1, 64, 128, "bf16", 1, 0, 0.0),
    ([9, 70], 1, 40, 128, 16, "fp16", 2, 0, 0.02),
]


@pytest.mark.parametrize("lens,H,G,d,T,kind,Tq,window,scale", ATTN)
def test_attention_matches_its_definition(dd, lens, H, G, d, T, kind, Tq, window, scale):
    gen = torch.Generator().manual_seed(sum(lens) + G)
    cache, raw, table = make(dd, gen, lens, H, d, T, "int4", gap=16 * (len(lens) % 2), shared=True)
    q = queries(gen, len(lens), Tq, H * G, d, kind)
    out, lse = run_attn(cache, q, lens, window, scale)
    assert cache.device_error() == (0, 0)
    check_attn(out, lse, q, raw, table, lens, kind, T, window, scale or None)
    again, _ = run_attn(cache, q, lens, window, scale, with_lse=False)    # the same bits every time, with or without lse
    assert torch.equal(out, again)


@pytest.mark.parametrize("M", [5, 40, 600])                           # a warp a unit, clusters, the flat list
def test_every_split_of_the_work(dd, M):
    gen = torch.Generator().manual_seed(M)
    lens = [min(M * 16, n) for n in (M * 16, M * 8 + 3, 1, 17)]
    cache, raw, table = make(dd, gen, lens, 2, 128, 16, "int4", spare=0)
    q = queries(gen, 4, 1, 8, 128, "bf16")
    out, lse = run_attn(cache, q, lens)
    check_attn(out, lse, q, raw, table, lens, "bf16", 16)


def test_attention_of_many_shapes(dd):
    rng = np.random.RandomState(6)
    for i in range(30):
        B, H, G, d, T = rng.randint(1, 6), rng.randint(1, 4), rng.randint(1, 12), [64, 128][rng.randint(2)], [16, 32, 64][rng.randint(3)]
        Tq, window, kind = rng.randint(1, 4), [0, 0, int(rng.randint(1, 300))][rng.randint(3)], ["bf16", "fp16"][rng.randint(2)]
        lens = [int(2 ** rng.uniform(0, 11)) - 1 for _ in range(B)]
        gen = torch.Generator().manual_seed(i)
        cache, raw, table = make(dd, gen, lens, H, d, T, "int4")
        q = queries(gen, B, Tq, H * G, d, kind)
        out, lse = run_attn(cache, q, lens, window, 0.02)
        check_attn(out, lse, q, raw, table, lens, kind, T, window, 0.02)


def test_groups_and_rows_far_apart(dd):
    """Row exponents over the whole range of the type, and groups of a row at the largest ratio that scales allow."""
    gen = torch.Generator().manual_seed(9)
    rng = np.random.RandomState(1)
    T, d, n = 16, 128, 700
    for kind, spread in (("bf16", 30), ("fp16", 6)):
        cache, raw, table = make(dd, gen, [n], 1, d, T, "int4")
        v = rng.randn(*raw.shape[:2], 2, T, d)
        v[..., 16:32] *= 2.0 ** -11                                  # scales near 2^-4 next to ones near 448
        v[:, :, 1] *= np.exp2(rng.randint(-spread, spread, v[:, :, 1].shape[:-1]))[..., None]
        raw = ref4.encode_pages(v, "int4")
        cache.data.copy_(torch.from_numpy(raw).cuda())
        q = queries(gen, 1, 1, 4, d, kind)
        out, lse = run_attn(cache, q, [n])
        want = ref4.attention(f64(q), raw, table.numpy(), [n], "int4", T)
        limit = torch.finfo(TYPES[kind]).max
        assert np.abs(want[0]).max() < limit
        check(out, lse, *want, "int4", kind, n)
        # channels that only small groups feed, by their own measure: the definition's sum of weight * |V| of the channel
        rel = 2.0 ** -11 if kind == "bf16" else 2.0 ** -22
        dz = (d + 8) * 2.0 ** -24 * want[3] + 2.0 ** -21 * (1 + np.abs(want[1]))
        slack = (rel + 2 * dz + n * 2.0 ** -29 + 2.0 ** -16)[..., None] * want[2]
        half = np.maximum(np.exp2(np.frexp(np.abs(want[0]) + slack)[1] - BITS[kind] - 1.0), TINY[kind])
        assert np.all(np.abs(f64(out) - want[0])[..., 16:32] <= (half + slack)[..., 16:32])


def test_nan_groups_reach_only_the_rows_that_see_them(dd):
    """A group of the newest token's value is not finite: the query token before it must not notice; nor, with a window, of an old one."""
    gen = torch.Generator().manual_seed(0)
    lens, H, G, d, T, Tq = [100, 37], 2, 4, 128, 16, 2
    cache, raw, table = make(dd, gen, lens, H, d, T, "int4")
    q = queries(gen, 2, Tq, H * G, d, "bf16")
    clean = raw.copy()
    _, _, scale, _ = ref4.places(T, d)
    for b, n in enumerate(lens):
        for at in (n - 1, n - 22):
            raw[int(table[b, at // T]), :, scale[1, at % T, 5]] = 0x7f
    cache.data.copy_(torch.from_numpy(raw).cuda())
    out, _ = run_attn(cache, q, lens, window=21)                    # token 0 sees n-22 .. n-2, token 1 sees n-21 .. n-1
    assert bool(torch.isnan(out[..., :16]).all()) and bool(torch.isfinite(out[..., 16:]).all())
    out, lse = run_attn(cache, q, lens, window=20)                  # now n-22 is hidden from both
    want = ref4.attention(f64(q), clean, table.numpy(), lens, "int4", T, 20)
    assert bool(torch.isnan(out[:, 1, :, :16]).all())
    check(out[:, :1], lse[:, :1], *(w[:, :1] for w in want), "int4", "bf16", 100)


def test_bad_lengths_and_tables_are_reported(dd):
    gen = torch.Generator().manual_seed(1)
    cache, raw, table = make(dd, gen, [64, 64], 1, 128, 16, "int4")
    q, M = queries(gen, 2, 1, 4, 128, "bf16"), table.shape[1]
    out, lse = run_attn(cache, q, [-5, 64])
    assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, -5)
    check_attn(out, lse, q, raw, table, [0, 64], "bf16", 16)
    cache.block_table[:, M - 1] = 0
    out, lse = run_attn(cache, q, [64, M * 16 + 1])
    assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, M * 16 + 1)
    check_attn(out, lse, q, raw, cache.block_table.cpu(), [64, M * 16], "bf16", 16)
    for bad in (-1, raw.shape[0], 2 ** 31 - 1):
        keep = int(table[0, 1])
        cache.block_table[0, 1] = bad
        out, lse = run_attn(cache, q, [64, 64])
        assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, bad)
        zeros, t = np.concatenate([raw, np.zeros_like(raw[:1])]), table.clone()      # the page reads as zeros
        t[0, 1] = raw.shape[0]
        check_attn(out, lse, q, zeros, t, [64, 64], "bf16", 16)
        cache.block_table[0, 1] = keep
