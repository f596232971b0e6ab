"""Every kernel that the selection of pages picks from, at the sizes that reach it and with ties that make its general forms run, against
the plain 64-bit definition; and what the lists of the attention mean however the work is split."""
import numpy as np
import pytest
import torch

from tests import _int4_ref as ref4
from tests._int4_ref import TYPES
from tests.test_gpu_int4 import dd, make  # noqa: F401  (dd is the fixture)
from tests.test_gpu_sparse import check_listed, ints, random_landmarks, run_listed, want_select

pytestmark = pytest.mark.gpu

PATHS = [  # requests, tokens of each, max_pages, H, G, d, type, k, first, recent, ties
    # many rows of short tables, one or two tokens a request: keys of a row in registers of eight warps
    (160, 1, 100, 8, 2, 128, "bf16", 8, 1, 2, False),
    (160, 1, 100, 8, 2, 64, "fp16", 9, 0, 1, True),
    (70, 2, 3000, 8, 1, 128, "bf16", 20, 1, 4, False),
    (70, 2, 3000, 8, 1, 128, "bf16", 20, 1, 4, True),
    # more pages to choose than the kernel of few rows ranks
    (2, 1, 2990, 2, 4, 128, "bf16", 300, 2, 8, False),
    (1, 1, 4096, 1, 4, 64, "bf16", 257, 0, 1, True),
    # few rows whose keys are all alike or nearly so: more candidates than are listed
    (1, 1, 3000, 1, 4, 128, "bf16", 50, 0, 1, True),
    (2, 2, 4096, 2, 1, 64, "fp16", 256, 1, 1, True),
    # tables too wide for one kernel: 8 tokens a block, several requests in a tile; 64 tokens a block with their codes made ahead
    (5, 3, 2100, 2, 4, 128, "bf16", 16, 1, 2, False),
    (3, 31, 2500, 3, 2, 64, "bf16", 33, 1, 2, True),
    (2, 45, 2500, 3, 2, 128, "bf16", 24, 1, 2, False),
    (3, 70, 2200, 2, 4, 128, "fp16", 12, 0, 3, True),
    (1, 200, 5000, 2, 1, 128, "bf16", 64, 1, 2, False),
    # wider still, and more entries than any list in shared memory
    (2, 1, 16384, 1, 2, 128, "bf16", 2500, 1, 4, False),
    (1, 2, 16385, 2, 2, 64, "bf16", 40, 1, 4, True),
    (1, 1, 20000, 1, 2, 64, "bf16", 2500, 1, 4, True),
    # tables that one kernel takes: the longest lists, all keys alike, tiles of several requests; few rows and many
    (1, 320, 2048, 1, 2, 128, "bf16", 300, 1, 2, True),
    (20, 12, 900, 8, 1, 64, "bf16", 40, 1, 2, True),
    (20, 12, 900, 8, 2, 128, "fp16", 256, 2, 1, False),
    (40, 5, 300, 8, 1, 128, "bf16", 17, 0, 2, False),
    (1, 40, 2048, 2, 2, 128, "bf16", 300, 1, 2, True),
    (7, 5, 900, 2, 2, 64, "fp16", 70, 1, 2, False),
    (7, 5, 900, 2, 2, 128, "bf16", 256, 0, 1, True),
]


@pytest.mark.parametrize("B,per,max_pages,H,G,d,kind,k,first,recent,ties", PATHS)
def test_every_kernel_of_the_selection(dd, B, per, max_pages, H, G, d, kind, k, first, recent, ties):
    gen = torch.Generator().manual_seed(max_pages + k + per)
    T, blocks = 16, 4096                                              # blocks appear many times: ties of their own
    table = torch.randint(0, blocks, (B, max_pages), generator=gen).to(torch.int32)
    lm = random_landmarks(gen, blocks, H, d, ties)
    if ties:
        lm[...] = lm[:1]                                              # all alike
        lm[::97, :, :d] = 0
    pool = torch.zeros(blocks, H, ref4.page_bytes("int4", T, d), dtype=torch.uint8, device="cuda")
    cache = dd.PagedCache(pool, table.cuda(), cache_format=dd.DD_CACHE_INT4, head_dim=d, page_tokens=T)
    n = B * per
    positions = torch.randint(0, max_pages * T, (n,), generator=gen).to(torch.int32)
    positions[::3] = max_pages * T - 1 - positions[::3] % (2 * T)     # a third at the far end
    if per > 2:
        positions[1::7] = -1
    q = torch.randn(n, H * G, d, generator=gen).to(TYPES[kind]).cuda()
    idx = torch.full((n, H, k), 77, dtype=torch.int32, device="cuda")
    cache.select(q, lm.cuda(), positions.cuda(), idx, first_pages=first, recent_pages=recent)
    torch.cuda.synchronize()
    want = want_select(q, lm, table, np.repeat(np.arange(B), per), positions.numpy(), k, first, recent, T)
    got = idx.cpu().numpy()
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]
    assert cache.device_error() == (0, 0)


LISTS = [[-1, 0, -1, -1], [0, 0, -1, -1], [0, -1, 0, 0], [-1, -1, -1, 0], [1, 0, 1, 0], [3, -1, 2, 2]]


@pytest.mark.parametrize("fmt", ["int4", "bf16", "e4m3"])
@pytest.mark.parametrize("copies,H", [(1, 1), (30, 2), (120, 8)])      # a cluster a unit, the flat list, two tokens to a unit
def test_entries_in_front_count_however_the_work_is_split(dd, fmt, copies, H):
    """As many entries are looked at as there are pages up to the token's own, holes and repeats among them: early in a context a
    list has to have its pages in front. The same for every split of the work."""
    gen = torch.Generator().manual_seed(copies)
    G, d, T = 4, 128, 16
    cache, raw, table = make(dd, gen, [200], H, d, T, fmt)
    lists, places = [np.array(l, dtype=np.int32) for l in LISTS], [3, 15, 17, 31, 150]
    positions = [p for p in places for _ in lists] * copies
    idx = np.stack([l for _ in places for l in lists] * copies)[:, None].repeat(H, 1)
    q = torch.randn(len(positions), H * G, d, generator=gen).to(torch.bfloat16).cuda()
    out, lse = run_listed(cache, q, idx, positions, [0] * len(positions))
    assert cache.device_error() == (0, 0)
    check_listed(out, lse, q, raw, table, [0] * len(positions), positions, idx, fmt, "bf16", T)
    nothing = np.array([not any(0 <= e <= p // T for e in l[:p // T + 1]) for p, l in zip(positions, idx[:, 0])])
    assert nothing.any() and not nothing.all()
    assert bool((out[torch.from_numpy(nothing)] == 0).all()) and bool(torch.isneginf(lse[torch.from_numpy(nothing)]).all())
    assert bool(torch.isfinite(lse[torch.from_numpy(~nothing)]).all())
