"""Landmarks of a paged cache, the pages chosen for each query token, attention over listed pages, and all of them together, against
plain 64-bit definitions. Landmarks and chosen pages are whole numbers and have to be equal."""
import numpy as np
import pytest
import torch

from tests import _int4_ref as ref4
from tests._cache_ref import f64
from tests._int4_ref import TYPES, check
from tests.test_gpu_int4 import dd, format_code, make, random_pages, rope_of  # noqa: F401  (dd is the fixture)

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


# ---------------------------------------------------------------------------------------------- landmarks
@pytest.mark.parametrize("fmt,T,d,H,n_last", [("int4", 16, 128, 2, 0), ("int4", 64, 64, 3, 5), ("e4m3", 32, 128, 1, 40), ("e4m3", 16, 64, 2, 0),
                                              ("bf16", 16, 128, 8, 1), ("bf16", 256, 64, 1, 0), ("fp16", 16, 64, 2, 17), ("fp16", 32, 128, 2, 0)])
def test_landmarks_match_their_definition(dd, fmt, T, d, H, n_last):
    gen = torch.Generator().manual_seed(T + d + n_last)
    lens = [200, 0, 1, T, T + 1, 77]
    cache, raw, table = make(dd, gen, lens, H, d, T, fmt, gap=16)
    raw[int(table[0, 0])] = random_pages(gen, 1, H, fmt, T, d, 2.0 ** -9)[0]
    if fmt == "bf16":                                                # a channel that is not finite, and keys beyond 2^63
        page = np.zeros((T, d), np.float64)
        page[:, 3], page[:, 5] = 2.0 ** 90, 2.0 ** 69
        raw[int(table[0, 1]), 0, :T * d * 2] = torch.from_numpy(page).to(torch.bfloat16).view(torch.uint8).numpy().reshape(-1)
        raw[int(table[0, 2]), 0, 4:6] = np.frombuffer(np.uint16(0x7f80).tobytes(), np.uint8)
    cache.data.copy_(torch.from_numpy(raw).cuda())
    lm = torch.full((raw.shape[0], H, d + 16), 99, dtype=torch.uint8, device="cuda")
    cache.update_landmarks(lm, ints(lens), n_last=n_last)
    torch.cuda.synchronize()
    want = np.full(lm.shape, 99, dtype=np.uint8)
    for b, n in enumerate(lens):
        for p in range((max(0, n - n_last) if n_last else 0) // T, -(-n // T)):
            blk = int(table[b, p])
            for h in range(H):
                want[blk, h] = ref4.landmark(ref4.decode_pages(raw[blk, h], fmt, T, d)[0, :min(T, n - p * T)])
    assert np.array_equal(lm.cpu().numpy(), want)
    assert cache.device_error() == (0, 0)


@pytest.mark.parametrize("fmt,d,H", [("int4", 64, 8), ("bf16", 128, 7), ("fp16", 64, 3), ("e4m3", 128, 8)])
def test_landmarks_of_many_pages(dd, fmt, d, H):
    """More pages than fill the device, so that a warp has several: full ones out of a few blocks, ragged ends, an empty request, a bad entry."""
    T, M, full = 16, 3001, 40
    gen = torch.Generator().manual_seed(d + H)
    lens = [3000 * T + 5, 0, 1200 * T, 2999 * T + 1, 7, 2500 * T + 15, 3001 * T, 17]
    raw = random_pages(gen, full + len(lens), H, fmt, T, d)
    table = torch.randint(0, full, (len(lens), M), generator=gen, dtype=torch.int32)
    for b, n in enumerate(lens):
        if n % T:
            table[b, n // T] = full + b
    table[2, 77] = full + len(lens)                                  # behind the pool
    table[5, 2501:] = -9                                             # never read
    cache = dd.PagedCache(torch.from_numpy(raw).cuda(), table.cuda(), cache_format=format_code(dd, fmt), head_dim=d, page_tokens=T)
    lm = torch.full((raw.shape[0], H, d + 16), 99, dtype=torch.uint8, device="cuda")
    cache.update_landmarks(lm, ints(lens))
    torch.cuda.synchronize()
    want = np.full(lm.shape, 99, dtype=np.uint8)
    for blk in range(raw.shape[0]):
        n = T if blk < full else lens[blk - full] % T
        for h in range(H if n else 0):
            want[blk, h] = ref4.landmark(ref4.decode_pages(raw[blk, h], fmt, T, d)[0, :n])
    assert np.array_equal(lm.cpu().numpy(), want)
    assert cache.device_error()[1] == full + len(lens)


# ---------------------------------------------------------------------------------------------- selection
def random_landmarks(gen, n, H, d, ties=False):
    lm = torch.zeros(n, H, d + 16, dtype=torch.uint8)
    lm[..., :d] = torch.randint(-127, 128, (n, H, d), generator=gen).to(torch.int8).view(torch.uint8)
    lm[..., d] = torch.randint(55, 59, (n, H), generator=gen).to(torch.uint8)
    if ties:
        lm[...] = lm[:3].repeat(n // 3 + 1, 1, 1)[:n]
    return lm


def want_select(q, lm, table, requests, positions, k, first, recent, T):
    q, lm, t = f64(q), lm.numpy(), table.numpy()
    H = lm.shape[1]
    G = q.shape[1] // H
    out = np.full((q.shape[0], H, k), -1, dtype=np.int32)
    for n in range(q.shape[0]):
        if positions[n] >= 0:
            own = positions[n] // T
            for h in range(H):
                out[n, h] = ref4.select(q[n, h * G:(h + 1) * G], lm[t[requests[n], :own + 1], h], k, first, recent, own)
    return out


SELECT = [  # positions by request, H, G, d, T, type, k, first, recent, max_pages, ties
    ([[0]], 1, 1, 128, 16, "bf16", 1, 0, 1, 1, False),
    ([[1000], [17], [], [555]], 2, 4, 128, 16, "bf16", 8, 1, 2, 64, False),
    ([[1000, 1001], [2, 3], [400, 401]], 2, 3, 64, 16, "fp16", 13, 0, 1, 63, False),
    ([list(range(900, 1030)), [5]], 2, 4, 128, 16, "bf16", 20, 1, 1, 65, False),
    ([list(range(0, 300))], 1, 5, 64, 32, "fp16", 4, 1, 2, 33, False),
    ([list(range(50)), list(range(700, 719)), [31]], 3, 2, 128, 16, "bf16", 30, 2, 3, 45, False),
    ([[32000], [31000]], 2, 4, 128, 16, "bf16", 128, 1, 8, 2048, False),
    ([[50000]], 1, 8, 64, 16, "bf16", 128, 0, 1, 3200, False),
    ([[200000], [131072]], 1, 4, 128, 16, "bf16", 100, 1, 4, 12600, False),
    ([[700000]], 1, 4, 64, 16, "fp16", 300, 1, 4, 43760, False),
    ([[900000, 900001]], 1, 2, 64, 16, "bf16", 2000, 1, 4, 56300, False),
    ([[16 * 500 + 3, 16 * 499]], 2, 2, 128, 16, "bf16", 50, 1, 2, 501, True),
    ([list(range(3000, 3100))], 2, 2, 64, 16, "bf16", 50, 0, 1, 200, True),
    ([list(range(8000, 8400))], 4, 4, 128, 16, "bf16", 40, 1, 2, 540, False),
]


@pytest.mark.parametrize("where,H,G,d,T,kind,k,first,recent,max_pages,ties", SELECT)
def test_selection_matches_its_definition(dd, where, H, G, d, T, kind, k, first, recent, max_pages, ties):
    gen = torch.Generator().manual_seed(max_pages + k)
    B = len(where)
    positions = [p for w in where for p in w] + [-1, -5]
    requests = [b for b, w in enumerate(where) for _ in w] + [0, B - 1]
    n_blocks = B * max_pages
    table = torch.randperm(n_blocks, generator=gen).view(B, max_pages).to(torch.int32)
    lm = random_landmarks(gen, n_blocks, H, d, ties)
    pool = torch.zeros(16, dtype=torch.uint8, device="cuda")
    page = dd.lib.dd_cache_page_bytes(dd.DD_CACHE_INT4, T, d)
    pool = torch.zeros(n_blocks, H, page, dtype=torch.uint8, device="cuda") if n_blocks * H * page < 1 << 31 else None
    cache = dd.PagedCache(pool, table.cuda(), cache_format=dd.DD_CACHE_INT4, head_dim=d, page_tokens=T)
    q = torch.randn(len(positions), H * G + 1, d, generator=gen).to(TYPES[kind]).cuda()[:, :H * G]
    idx = torch.full((len(positions), H, k), 77, dtype=torch.int32, device="cuda")
    cache.select(q, lm.cuda(), ints(positions), idx, ints(requests), first_pages=first, recent_pages=recent)
    torch.cuda.synchronize()
    want = want_select(q, lm, table, requests, positions, k, first, recent, T)
    got = idx.cpu().numpy()
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]
    assert cache.device_error() == (0, 0)


def test_selection_in_pieces_and_without_requests(dd):
    """More tokens than the workspace holds at once; equal numbers of tokens per request need no list of requests."""
    gen = torch.Generator().manual_seed(3)
    B, per, H, d, T, M, k = 2, 96, 1, 64, 16, 9000, 12
    table = torch.randint(0, 500, (B, M), generator=gen).to(torch.int32)
    lm = random_landmarks(gen, 500, H, d)
    cache = dd.PagedCache(torch.zeros(500, H, 1184, dtype=torch.uint8, device="cuda"), table.cuda(), cache_format=dd.DD_CACHE_INT4, head_dim=d)
    assert dd.lib.dd_cache_select_workspace(B * per * 20, H, M) < B * per * 20 * M * 4
    positions = torch.randint(0, M * T, (B * per,), generator=gen).to(torch.int32)
    q = torch.randn(B * per, 2, d, generator=gen).to(torch.bfloat16).cuda()
    small = torch.empty(B * per, H, k, dtype=torch.int32, device="cuda")
    cache.select(q, lm.cuda(), positions.cuda(), small)
    requests = np.repeat(np.arange(B), per)
    want = want_select(q, lm, table, requests, positions.numpy(), k, 0, 1, T)      # blocks appear many times: ties
    assert np.array_equal(small.cpu().numpy(), want)
    many = torch.empty(B * per * 20, H, k, dtype=torch.int32, device="cuda")
    cache.select(q.repeat(20, 1, 1), lm.cuda(), positions.repeat(20).cuda(), many, ints(np.tile(requests, 20)))
    assert torch.equal(many.view(20, B * per, H, k), small.unsqueeze(0).expand(20, -1, -1, -1))


def test_queries_of_every_size(dd):
    """Rows far below and above one, with an infinity or NaN, and zeros (all scores equal: the lowest pages)."""
    gen = torch.Generator().manual_seed(4)
    H, G, d, M, k = 1, 2, 128, 70, 6
    table, lm = torch.arange(M, dtype=torch.int32).view(1, M), random_landmarks(gen, M, 1, d)
    lm[:, :, d] = torch.randint(0, 128, (M, 1), generator=gen).to(torch.uint8)       # exponents from -64 to 63
    cache = dd.PagedCache(torch.zeros(M, 1, 2336, dtype=torch.uint8, device="cuda"), table.cuda(), cache_format=dd.DD_CACHE_INT4)
    q = torch.randn(9, G, d, generator=gen)
    for n, s in enumerate([2.0 ** -126, 2.0 ** -100, 2.0 ** 50, 2.0 ** 70, 2.0 ** 120, 0.0]):
        q[n] *= s
    q = q.to(torch.bfloat16)
    q[6, 0, 5], q[7, 1, 9], q[8, :, 3] = float("nan"), float("inf"), 3e38
    idx = torch.empty(9, 1, k, dtype=torch.int32, device="cuda")
    cache.select(q.cuda(), lm.cuda(), ints([M * 16 - 1] * 9), idx)
    assert np.array_equal(idx.cpu().numpy(), want_select(q, lm, table, [0] * 9, [M * 16 - 1] * 9, k, 0, 1, 16))
    assert idx[5, 0].tolist() == [0, 1, 2, 3, 4, M - 1]


def test_bad_places_are_reported_by_the_selection(dd):
    gen = torch.Generator().manual_seed(5)
    M, d = 8, 64
    table, lm = torch.arange(2 * M, dtype=torch.int32).view(2, M), random_landmarks(gen, 2 * M, 1, d)
    cache = dd.PagedCache(torch.zeros(2 * M, 1, 1184, dtype=torch.uint8, device="cuda"), table.cuda(), cache_format=dd.DD_CACHE_INT4, head_dim=d)
    q = torch.randn(3, 1, d, generator=gen).to(torch.bfloat16).cuda()
    for pos, req, bad in (([100, M * 16, 3], [0, 0, 1], M * 16), ([100, 5, 3], [0, 2, 1], 2), ([100, 5, 3], [0, -1, 1], -1)):
        idx = torch.full((3, 1, 3), 77, dtype=torch.int32, device="cuda")
        cache.select(q, lm.cuda(), ints(pos), idx, ints(req))
        assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, bad)
        want = want_select(q, lm, table, [0, 0, 1], [pos[0], -1, pos[2]], 3, 0, 1, 16)
        assert np.array_equal(idx.cpu().numpy(), want)
    cache.block_table[0, 2] = 2 * M                                   # a page without a block scores 0
    idx = torch.empty(1, 1, 3, dtype=torch.int32, device="cuda")
    cache.select(q[:1], lm.cuda(), ints([100]), idx, ints([0]))
    assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, 2 * M)
    t, zeros = table.clone(), torch.cat([lm, torch.zeros_like(lm[:1])])
    t[0, 2] = 2 * M
    assert np.array_equal(idx.cpu().numpy(), want_select(q[:1], zeros, t, [0], [100], 3, 0, 1, 16))
    lens = ints([100, 3])
    out = cache.new_landmarks()
    cache.update_landmarks(out, lens)
    assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, 2 * M)
    cache.update_landmarks(out, ints([-3, M * 16]))
    assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, -3)


# ---------------------------------------------------------------------------------------------- attention over listed pages
def random_lists(gen, positions, H, k, T):
    """Ascending, some of the visible pages, the own one mostly; -1 behind."""
    idx = np.full((len(positions), H, k), -1, dtype=np.int32)
    for n, p in enumerate(positions):
        for h in range(H if p >= 0 else 0):
            own = p // T
            some = torch.randperm(own + 1, generator=gen)[:k].numpy()
            if own not in some and (n + h) % 3:
                some[0] = own
            idx[n, h, :len(some)] = np.sort(some)
    return idx


def run_listed(cache, q, idx, positions, requests, scale=0.0, with_lse=True):
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda") if with_lse else None
    cache.sparse_attn(q, ints(idx), ints(positions), out, lse, None if requests is None else ints(requests), scale=scale)
    torch.cuda.synchronize()
    return out, lse


def check_listed(out, lse, q, raw, table, requests, positions, idx, fmt, kind, T, scale=None):
    live = np.asarray(positions) >= 0
    want = ref4.listed_attention(f64(q), raw, table.numpy(), requests, positions, idx, fmt, T, scale)
    check(out[torch.from_numpy(live)], None if lse is None else lse[torch.from_numpy(live)], *(w[live] for w in want), fmt, kind, idx.shape[2] * T)
    assert bool((out[torch.from_numpy(~live)] == 7.0).all())          # padding: as it was
    if lse is not None:
        assert bool((lse[torch.from_numpy(~live)] == 7.0).all())


SPARSE = [  # positions by request, H, G, d, T, fmt, query type, k, scale
    ([[0]], 1, 1, 128, 16, "int4", "bf16", 1, 0.0),
    ([[300, 301], [15, 16]], 2, 4, 128, 16, "int4", "bf16", 6, 0.0),
    ([[300, 301], [15, 16]], 2, 4, 64, 16, "int4", "fp16", 6, 0.02),
    ([[2000], [1999], [700], [0]], 8, 4, 128, 16, "int4", "bf16", 40, 0.0),
    ([[2000], [1999], [700], [0]], 8, 4, 128, 16, "bf16", "bf16", 40, 0.0),
    ([[2000], [1999], [700], [0]], 2, 4, 128, 16, "e4m3", "bf16", 40, 0.0),
    ([[2000], [1999], [700], [0]], 2, 5, 64, 32, "e4m3", "fp16", 40, 0.02),
    ([list(range(200)), list(range(500, 533)), [7]], 2, 4, 128, 16, "int4", "bf16", 9, 0.0),
    ([list(range(200)), list(range(500, 533)), [7]], 2, 4, 128, 16, "bf16", "bf16", 9, 0.0),
    ([list(range(200)), list(range(500, 533)), [7]], 3, 2, 64, 64, "fp16", "fp16", 5, 0.02),
    ([list(range(200)), list(range(500, 533)), [7]], 1, 12, 128, 32, "e4m3", "bf16", 9, 0.0),
    ([list(range(90))], 2, 16, 128, 16, "int4", "bf16", 3, 0.3),
    ([list(range(90))], 1, 20, 64, 16, "fp16", "fp16", 3, 0.02),
    ([[4000, 4001], [3000, 3001]], 1, 8, 128, 256, "int4", "fp16", 12, 0.02),
    ([[4095]], 2, 4, 128, 16, "bf16", "bf16", 256, 0.0),               # all of them
    ([[9000]], 1, 4, 64, 16, "e4m3", "bf16", 500, 0.0),
    ([[9000]], 1, 4, 128, 16, "int4", "bf16", 560, 0.0),
]


@pytest.mark.parametrize("where,H,G,d,T,fmt,kind,k,scale", SPARSE)
def test_attention_over_listed_pages_matches_its_definition(dd, where, H, G, d, T, fmt, kind, k, scale):
    gen = torch.Generator().manual_seed(k + H + G)
    lens = [max(w) + 1 for w in where]
    cache, raw, table = make(dd, gen, lens, H, d, T, fmt, gap=16 * (k % 2))
    positions = [p for w in where for p in w] + [-1, -1]
    requests = [b for b, w in enumerate(where) for _ in w] + [0, 0]
    idx = random_lists(gen, positions, H, k, T)
    wide = torch.randn(len(positions), H * G + 3, d, generator=gen).to(TYPES[kind]).cuda()
    q = wide[:, 1:1 + H * G]
    out, lse = run_listed(cache, q, idx, positions, requests, scale)
    assert cache.device_error() == (0, 0)
    check_listed(out, lse, q, raw, table, requests, positions, idx, fmt, kind, T, scale or None)
    again, _ = run_listed(cache, q, idx, positions, requests, scale, with_lse=False)
    assert torch.equal(out, again)


def test_attention_over_lists_of_many_shapes(dd):
    rng = np.random.RandomState(7)
    for i in range(40):
        fmt = ["bf16", "fp16", "e4m3", "int4", "int4"][rng.randint(5)]
        kind = fmt if fmt in TYPES else ["bf16", "fp16"][rng.randint(2)]
        B, H, G, d, T = rng.randint(1, 5), rng.randint(1, 4), rng.randint(1, 12), [64, 128][rng.randint(2)], [16, 32, 64][rng.randint(3)]
        per, k = rng.randint(1, 24), int(2 ** rng.uniform(0, 6))
        lens = [int(2 ** rng.uniform(0, 11)) for _ in range(B)]
        gen = torch.Generator().manual_seed(i)
        cache, raw, table = make(dd, gen, lens, H, d, T, fmt)
        positions = [max(-1, n - per + t) for n in lens for t in range(per)]
        idx = random_lists(gen, positions, H, k, T)
        q = torch.randn(B * per, H * G, d, generator=gen).to(TYPES[kind]).cuda()
        out, lse = run_listed(cache, q, idx, positions, None, 0.02)
        check_listed(out, lse, q, raw, table, np.repeat(np.arange(B), per), positions, idx, fmt, kind, T, 0.02)


PAIRS = [  # tokens by request, H, G, d, T, fmt, query type, k
    ([list(range(200)), list(range(500, 633)), [7]], 8, 4, 128, 16, "int4", "bf16", 9),
    ([list(range(200)), list(range(500, 633)), [7]], 8, 4, 128, 16, "bf16", "bf16", 9),
    ([list(range(100, 400))], 8, 2, 64, 16, "e4m3", "fp16", 12),
    ([list(range(400))], 8, 3, 128, 32, "e4m3", "bf16", 5),
    ([list(range(150)), list(range(151))], 8, 1, 64, 64, "fp16", "fp16", 3),
    ([list(range(150)), list(range(151))], 8, 4, 64, 16, "int4", "fp16", 20),
    ([list(range(5000, 5300))], 8, 4, 64, 16, "int4", "bf16", 270),       # lists too long to be merged
]


@pytest.mark.parametrize("where,H,G,d,T,fmt,kind,k", PAIRS)
def test_neighbouring_tokens_together(dd, where, H, G, d, T, fmt, kind, k):
    """Enough tokens of few query heads that two of them share a unit: lists that overlap, tokens of different requests side by
    side, padding between them, an odd number of tokens, lists that do not ascend."""
    gen = torch.Generator().manual_seed(k + H + G)
    lens = [max(w) + 1 for w in where]
    cache, raw, table = make(dd, gen, lens, H, d, T, fmt)
    positions = [p for w in where for p in w]
    requests = [b for b, w in enumerate(where) for _ in w]
    for at in (0, 7, 50, 51):                                         # padding on either side of a pair, and a pair of it
        positions.insert(at, -1)
        requests.insert(at, 0)
    if len(positions) % 2 == 0:
        positions.append(-1)
        requests.append(0)
    n = len(positions)
    assert n // 2 * H >= 8 * 148 and n % 2 == 1
    idx = random_lists(gen, positions, H, k, T)
    for i in range(0, n - 1, 2):                                      # neighbours share most of their pages
        if positions[i] >= 0 and positions[i + 1] > positions[i] and requests[i] == requests[i + 1]:
            idx[i + 1] = idx[i]
            idx[i + 1, ::2, :1] = 0
            idx[i + 1] = np.sort(idx[i + 1].astype(np.uint32)).astype(np.int32)          # (-1 behind)
            for h in range(H):                                        # no page twice
                row = [p for j, p in enumerate(idx[i + 1, h]) if p >= 0 and p not in idx[i + 1, h, :j]]
                idx[i + 1, h] = row + [-1] * (k - len(row))
    idx[10:20] = idx[10:20, :, ::-1]                                  # holes in front, descending
    idx[30, :, 0] = positions[30] // T + 1                            # behind the token's own page
    q = torch.randn(n, H * G, d, generator=gen).to(TYPES[kind]).cuda()
    out, lse = run_listed(cache, q, idx, positions, requests, 0.02 if kind == "fp16" else 0.0)
    assert cache.device_error() == (0, 0)
    check_listed(out, lse, q, raw, table, requests, positions, idx, fmt, kind, T, 0.02 if kind == "fp16" else None)
    again, _ = run_listed(cache, q, idx, positions, requests, 0.02 if kind == "fp16" else 0.0, with_lse=False)
    assert torch.equal(out, again)
    # a few tokens alone take the other way: the same but for the order of the sums
    few = [i for i in range(60, 70) if positions[i] >= 0]
    part, _ = run_listed(cache, q[few], idx[few], [positions[i] for i in few], [requests[i] for i in few], 0.02 if kind == "fp16" else 0.0)
    assert float((part.float() - out[few].float()).abs().max()) <= 2 * ref4.STEP[kind] * float(out[few].float().abs().max())


@pytest.mark.parametrize("fmt", ["int4", "bf16", "e4m3"])
def test_a_neighbours_pages_do_not_reach_a_token(dd, fmt):
    """Pages that only the other token of a pair lists hold infinities and NaN."""
    gen = torch.Generator().manual_seed(5)
    H, G, d, T, k, n = 8, 4, 128, 16, 4, 300
    cache, raw, table = make(dd, gen, [2000], H, d, T, fmt)
    bad = [int(table[0, p]) for p in (3, 50)]
    for blk in bad:
        if fmt == "int4":
            _, _, scale, _ = ref4.places(T, d)
            raw[blk][:, np.unique(scale[1])] = 0x7f
        elif fmt == "e4m3":
            raw[blk][:, T * d:2 * T * d] = 0x7f
        else:
            raw[blk][:, T * d * 2:] = 0xff
    cache.data.copy_(torch.from_numpy(raw).cuda())
    idx = np.tile(np.array([10, 20, 60, 124], dtype=np.int32), (n, H, 1))
    idx[1::2, :, 0], idx[2::4, :, 2] = 3, 50
    q = torch.randn(n, H * G, d, generator=gen).to(torch.bfloat16).cuda()
    out, lse = run_listed(cache, q, idx, [1999] * n, [0] * n)
    seen = np.zeros(n, bool)
    seen[1::2] = seen[2::4] = True
    assert bool(torch.isnan(out[torch.from_numpy(seen)]).all())
    clean = ~seen
    check_listed(out[torch.from_numpy(clean)], lse[torch.from_numpy(clean)], q[torch.from_numpy(clean)], raw, table, [0] * int(clean.sum()),
                 [1999] * int(clean.sum()), idx[clean], fmt, "bf16", T)


@pytest.mark.parametrize("fmt", ["int4", "bf16", "e4m3"])
def test_odd_lists(dd, fmt):
    """No page at all, pages out of order, holes, pages behind the token's own, numbers out of range, one page twice."""
    gen = torch.Generator().manual_seed(8)
    H, G, d, T, n = 1, 4, 128, 16, 200
    cache, raw, table = make(dd, gen, [n], H, d, T, fmt)
    own = (n - 1) // T
    lists = [[-1, -1, -1, -1], [own, 3, 0, 7], [-1, 5, -1, own], [own + 1, 2, own, -1], [4, 4, 4, -1], [3, table.shape[1], 2, -1], [-9, 1, 2, 3]]
    idx = np.array(lists, dtype=np.int32)[:, None]
    q = torch.randn(len(lists), H * G, d, generator=gen).to(torch.bfloat16).cuda()
    out, lse = run_listed(cache, q, idx, [n - 1] * len(lists), [0] * len(lists))
    assert cache.device_error()[0] == dd.DD_ERR_INDEX_RANGE
    check_listed(out, lse, q, raw, table, [0] * len(lists), [n - 1] * len(lists), idx, fmt, "bf16", T)
    assert bool((out[0] == 0).all()) and bool(torch.isneginf(lse[0]).all())
    # a token that names no place is passed over, and reported
    for pos, req, bad in ((table.shape[1] * T, 0, table.shape[1] * T), (5, 1, 1), (5, -2, -2)):
        out, lse = run_listed(cache, q[:3], idx[:3], [n - 1, pos, n - 1], [0, req, 0])
        assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, bad)
        check_listed(out, lse, q[:3], raw, table, [0, 0, 0], [n - 1, -1, n - 1], idx[:3], fmt, "bf16", T)
    cache.block_table[0, 3] = -1                                      # the page reads as zeros
    out, lse = run_listed(cache, q[1:2], idx[1:2], [n - 1], [0])
    assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, -1)
    t, zeros = table.clone(), np.concatenate([raw, np.zeros_like(raw[:1])])
    t[0, 3] = raw.shape[0]
    check_listed(out, lse, q[1:2], zeros, t, [0], [n - 1], idx[1:2], fmt, "bf16", T)


def test_nothing_listed_gives_zeros_however_the_work_is_split(dd):
    gen = torch.Generator().manual_seed(2)
    for n_tokens, k in ((1, 3), (1, 64), (700, 9), (40, 64)):
        cache, raw, table = make(dd, gen, [2000], 2, 64, 16, "int4")
        q = torch.randn(n_tokens, 4, 64, generator=gen).to(torch.float16).cuda()
        out, lse = run_listed(cache, q, np.full((n_tokens, 2, k), -1), [1999] * n_tokens, [0] * n_tokens)
        assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())


# ---------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("fmt,kind,d", [("int4", "bf16", 128), ("int4", "fp16", 64), ("e4m3", "bf16", 128), ("bf16", "bf16", 128)])
def test_prompt_chunks_and_steps_through_the_cache(dd, fmt, kind, d):
    """Chunks of two prompts, then steps: append, landmarks, selection, attention over what was selected; each against the definition
    on the bytes that the cache holds by then."""
    gen = torch.Generator().manual_seed(d)
    B, H, G, T, M, k = 2, 2, 4, 16, 30, 5
    page = dd.lib.dd_cache_page_bytes({"int4": 4, "e4m3": 2, "bf16": 0}[fmt], T, d)
    pool = torch.zeros(B * M, H, page, dtype=torch.uint8, device="cuda")
    table = torch.randperm(B * M, generator=gen).view(B, M).to(torch.int32)
    cache = dd.PagedCache(pool, table.cuda(), cache_format={"int4": dd.DD_CACHE_INT4, "e4m3": dd.DD_CACHE_E4M3, "bf16": dd.DD_CACHE_BF16}[fmt], head_dim=d, page_tokens=T)
    rope, _ = rope_of(dd, d, d)
    lm, length = cache.new_landmarks(), np.zeros(B, dtype=np.int64)
    for per in (150, 37, 1, 1, 2, 1):
        new = [per, max(1, per - 3)]                                  # the second request's chunk is shorter: padding
        positions = np.concatenate([np.where(np.arange(per) < new[b], length[b] + np.arange(per), -1) for b in range(B)])
        x = torch.randn(B * per, H * G + 2 * H, d, generator=gen).to(TYPES[kind]).cuda()
        q = torch.zeros(B * per, H * G, d, dtype=TYPES[kind], device="cuda")
        cache.append(x[:, H * G:H * G + H], x[:, H * G + H:], ints(positions), rope=rope, q=x[:, :H * G], q_out=q)
        length += new
        cache.update_landmarks(lm, ints(length), n_last=per)
        idx = torch.empty(B * per, H, k, dtype=torch.int32, device="cuda")
        cache.select(q, lm, ints(positions), idx, first_pages=1, recent_pages=2)
        out, lse = torch.full_like(q, 7.0), torch.full((B * per, H * G), 7.0, dtype=torch.float32, device="cuda")
        cache.sparse_attn(q, idx, ints(positions), out, lse)
        torch.cuda.synchronize()
        raw, requests = pool.cpu().numpy(), np.repeat(np.arange(B), per)
        lm_want = np.zeros(lm.shape, dtype=np.uint8)
        for b in range(B):
            for p in range(-(-int(length[b]) // T)):
                for h in range(H):
                    lm_want[int(table[b, p]), h] = ref4.landmark(ref4.decode_pages(raw[int(table[b, p]), h], fmt, T, d)[0, :min(T, int(length[b]) - p * T)])
        assert np.array_equal(lm.cpu().numpy(), lm_want)
        want = want_select(q, lm.cpu(), table, requests, positions, k, 1, 2, T)
        assert np.array_equal(idx.cpu().numpy(), want)
        check_listed(out, lse, q, raw, table, requests, positions, want, fmt, kind, T)
    assert cache.device_error() == (0, 0)
    # with as many entries as there are pages the set is everything: the same as the attention over all of the cache
    every = torch.empty(B, H, M, dtype=torch.int32, device="cuda")
    last = ints(length - 1)
    cache.select(q.view(B, -1, H * G, d)[:, 0].contiguous(), lm, last, every)
    qq = torch.randn(B, H * G, d, generator=gen).to(TYPES[kind]).cuda()
    out, dense = torch.empty_like(qq), torch.empty_like(qq)
    cache.sparse_attn(qq, every, last, out)
    cache.decode_attn(qq.view(B, 1, H * G, d), ints(length), dense.view(B, 1, H * G, d))
    assert (f64(out) - f64(dense)).__abs__().max() <= 2 * 2.0 ** -8 * np.abs(f64(dense)).max()


def test_captured_step_replayed_with_other_lengths(dd):
    """A whole step in a graph: positions, lengths and queries are read when it runs."""
    gen = torch.Generator().manual_seed(6)
    B, H, G, d, T, M, k = 3, 2, 4, 128, 16, 50, 7
    raw = random_pages(gen, B * M, H, "int4", T, d)
    table = torch.randperm(B * M, generator=gen).view(B, M).to(torch.int32)

    def new():
        pool = torch.from_numpy(raw).cuda()
        c = dd.PagedCache(pool, table.cuda(), cache_format=dd.DD_CACHE_INT4, head_dim=d, page_tokens=T)
        lm = c.new_landmarks()
        c.update_landmarks(lm, ints([M * T] * B))
        return c, lm, pool
    rope, _ = rope_of(dd, d, d)
    x, positions, lens = torch.zeros(B, H * G + 2 * H, d, dtype=torch.bfloat16, device="cuda"), ints([0] * B), ints([1] * B)

    def step(c, lm, s):
        c.append(x[:, H * G:H * G + H], x[:, H * G + H:], positions, rope=rope, q=x[:, :H * G], q_out=s["q"])
        c.update_landmarks(lm, lens, n_last=1)
        c.select(s["q"], lm, positions, s["idx"])
        c.sparse_attn(s["q"], s["idx"], positions, s["out"], s["lse"])

    def outputs():
        return dict(q=torch.zeros(B, H * G, d, dtype=torch.bfloat16, device="cuda"), idx=torch.zeros(B, H, k, dtype=torch.int32, device="cuda"),
                    out=torch.zeros(B, H * G, d, dtype=torch.bfloat16, device="cuda"), lse=torch.zeros(B, H * G, device="cuda"))
    a, b = new(), new()
    s, e = outputs(), outputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a[0], a[1], s)
    torch.cuda.current_stream().wait_stream(side)
    step(b[0], b[1], e)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a[0], a[1], s)
    for at in ([0, 5, 799], [300, 17, 16], [511, 512, 40], [799, 799, 799]):
        x.copy_(torch.randn(x.shape, generator=gen))
        positions.copy_(ints(at))
        lens.copy_(positions + 1)
        graph.replay()
        step(b[0], b[1], e)
        torch.cuda.synchronize()
        assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
        for name in s:
            assert torch.equal(s[name], e[name]), name


def test_calls_on_several_streams_at_once(dd):
    gen = torch.Generator().manual_seed(11)
    H, G, d, T, k, n = 2, 4, 128, 16, 16, 30
    cache, raw, table = make(dd, gen, [4000], H, d, T, "int4")
    lm = cache.new_landmarks()
    cache.update_landmarks(lm, ints([4000]))
    positions = ints(torch.randint(0, 4000, (n,), generator=gen))
    qs = [torch.randn(n, H * G, d, generator=gen).to(torch.bfloat16).cuda() for _ in range(4)]
    torch.cuda.synchronize()

    def call(q, stream):
        idx, out = torch.empty(n, H, k, dtype=torch.int32, device="cuda"), torch.empty_like(q)
        cache.select(q, lm, positions, idx, stream=stream)
        cache.sparse_attn(q, idx, positions, out, stream=stream)
        return idx, out
    want = [call(q, None) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = [[call(q, s) for q, s in zip(qs, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    for g in got:
        for (i, o), (wi, wo) in zip(g, want):
            assert torch.equal(i, wi) and torch.equal(o, wo)


@pytest.mark.parametrize("n,k,ctx", [(2, 30, 2000), (40, 64, 4000), (320, 9, 2000)])      # a cluster a unit, the flat list, pairs
def test_output_in_place_of_the_queries(dd, n, k, ctx):
    gen = torch.Generator().manual_seed(n)
    H, G, d, T = 8, 4, 128, 16
    cache, raw, table = make(dd, gen, [ctx], H, d, T, "int4")
    positions = torch.randint(0, ctx, (n,), generator=gen).to(torch.int32)
    idx = ints(random_lists(gen, positions.tolist(), H, k, T))
    q = torch.randn(n, H * G, d, generator=gen).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)
    cache.sparse_attn(q, idx, positions.cuda(), out)
    cache.sparse_attn(q, idx, positions.cuda(), q)
    assert torch.equal(q, out)


def test_two_captured_steps_with_workspaces_of_their_own(dd):
    """Two graphs that replay at the same time on two streams, each with its own workspaces."""
    gen = torch.Generator().manual_seed(21)
    H, G, d, T, k, n = 2, 4, 128, 16, 40, 6
    cache, raw, table = make(dd, gen, [6000], H, d, T, "int4")
    lm = cache.new_landmarks()
    cache.update_landmarks(lm, ints([6000]))
    positions = ints(torch.randint(3000, 6000, (n,), generator=gen))
    qs = [torch.randn(n, H * G, d, generator=gen).to(torch.bfloat16).cuda() for _ in range(2)]
    want = []
    for q in qs:
        idx, out = torch.empty(n, H, k, dtype=torch.int32, device="cuda"), torch.empty_like(q)
        cache.select(q, lm, positions, idx)
        cache.sparse_attn(q, idx, positions, out)
        want.append((idx, out))
    torch.cuda.synchronize()
    graphs, got, spaces = [], [], []
    for q in qs:
        ws = torch.empty(dd.lib.dd_cache_select_workspace(n, H, table.shape[1]), dtype=torch.uint8, device="cuda")
        wa = torch.empty(dd.lib.dd_cache_sparse_attn_workspace(n, H * G, H, d, k), dtype=torch.uint8, device="cuda")
        idx, out = torch.zeros(n, H, k, dtype=torch.int32, device="cuda"), torch.zeros_like(q)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(5):
                cache.select(q, lm, positions, idx, workspace=ws)
                cache.sparse_attn(q, idx, positions, out, workspace=wa)
        graphs.append(g)
        got.append((idx, out))
        spaces.append((ws, wa))
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(4):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for (i, o), (wi, wo) in zip(got, want):
        assert torch.equal(i, wi) and torch.equal(o, wo)


def test_wrong_memory_and_small_workspaces_are_refused(dd):
    gen = torch.Generator().manual_seed(12)
    cache, raw, table = make(dd, gen, [64, 64], 2, 128, 16, "int4")
    q, idx, pos = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 3, dtype=torch.int32, device="cuda"), ints([63, 63])
    lm, out = cache.new_landmarks(), torch.full((2, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    need = dd.lib.dd_cache_sparse_attn_workspace(2, 4, 2, 128, 3)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    calls = [lambda: cache.sparse_attn(q, idx, pos, out, workspace=ws[:-1]), lambda: cache.sparse_attn(q, idx, pos, out, workspace=ws[8:]),
             lambda: cache.sparse_attn(q.cpu(), idx, pos, out), lambda: cache.sparse_attn(q, idx.cpu(), pos, out), lambda: cache.sparse_attn(q, idx, pos.cpu(), out),
             lambda: cache.sparse_attn(q, idx, pos, out.cpu()), lambda: cache.sparse_attn(q, idx, pos, out, torch.zeros(2, 4)),
             lambda: cache.sparse_attn(q, idx, pos, out, None, pos.cpu()), lambda: cache.sparse_attn(q, idx, pos, out, workspace=ws.cpu()),
             lambda: cache.select(q, lm, pos, idx, workspace=ws[:2 * 2 * 32 * 4 - 1]), lambda: cache.select(q, lm.cpu(), pos, idx),
             lambda: cache.select(q.cpu(), lm, pos, idx), lambda: cache.select(q, lm, pos, idx.cpu()), lambda: cache.select(q, lm, pos, idx, first_pages=3),
             lambda: cache.update_landmarks(lm.cpu(), ints([64, 64])), lambda: cache.update_landmarks(lm, ints([64, 64]).cpu())]
    for call in calls:
        with pytest.raises(dd.DDError) as e:
            call()
        assert e.value.code == dd.DD_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
    pinned = torch.from_numpy(raw).pin_memory()
    host = dd.PagedCache(pinned, table.cuda(), cache_format=dd.DD_CACHE_INT4)
    for call in (lambda: host.sparse_attn(q, idx, pos, out), lambda: host.update_landmarks(lm, ints([64, 64]))):
        with pytest.raises(dd.DDError):
            call()
