"""The 4-bit cache at the ends of what its calls allow: pages that are missing, keys that are turned beyond 32 bits, rows of zeros."""
import numpy as np
import pytest
import torch

from tests import _cache_ref as ref
from tests import _int4_ref as ref4
from tests._cache_ref import f64
from tests._int4_ref import TYPES
from tests.test_gpu_cache import dd, pool_of, rope_of  # noqa: F401  (dd is the fixture)
from tests.test_gpu_int4 import format_code, random_pages

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,out,T,d,pinned", [("int4", "bf16", 16, 128, False), ("int4", "fp16", 64, 64, False), ("int4", "fp16", 16, 128, True),
                                                ("e4m3", "bf16", 16, 128, False), ("e4m3", "fp16", 32, 64, True), ("bf16", "bf16", 16, 64, False)])
def test_missing_pages_read_as_zeros_without_a_sign(dd, fmt, out, T, d, pinned):
    """Every way in which a page can be missing: the bits are those of +0, as in every other format."""
    gen = torch.Generator().manual_seed(T + d)
    H, M = 2, 6
    _, pool = pool_of(random_pages(gen, M, H, fmt, T, d), 16, pinned)
    table = torch.arange(M, dtype=torch.int32).view(1, M)
    table[0, 2], table[0, 3] = -1, M
    cache = dd.PagedCache(pool, table.cuda(), cache_format=format_code(dd, fmt), head_dim=d, page_tokens=T)
    idx = torch.tensor([0, -1, 2, M, 3, 5, -7], dtype=torch.int32).expand(1, H, 7).contiguous().cuda()
    got = torch.full((1, H, 2, 7 * T, d), 7.0, dtype=TYPES[out], device="cuda")
    cache.read(idx, got)
    torch.cuda.synchronize()
    bits = got.view(torch.int16).view(H, 2, 7, T, d)
    assert bool((bits[:, :, [1, 2, 3, 4, 6]] == 0).all())
    assert bool((bits[:, :, [0, 5]] != 0).any())
    assert cache.device_error()[0] == dd.DD_ERR_INDEX_RANGE


def appended(dd, k, v, pos, rope, d, T=16):
    """Bytes of a cache of one request after an append of N tokens: parts of every row by the definition's places."""
    N, H = k.shape[:2]
    blocks = N // T
    raw = np.zeros((blocks, H, ref4.page_bytes("int4", T, d)), dtype=np.uint8)
    whole, pool = pool_of(raw)
    cache = dd.PagedCache(pool, torch.arange(blocks, dtype=torch.int32).view(1, blocks).cuda(), cache_format=dd.DD_CACHE_INT4, head_dim=d, page_tokens=T)
    cache.append(k.cuda(), v.cuda(), pos.cuda(), torch.zeros(N, dtype=torch.int32, device="cuda"), rope=rope)
    torch.cuda.synchronize()
    assert cache.device_error() == (0, 0)
    return whole.cpu().numpy()


def check_rows(got, rows, kv, pos, d, T=16):
    """The bytes of rows [N, H, d] (64 bits) are those of the definition."""
    code, shift, scale, ex = ref4.places(T, d)
    c, s, e = ref4.quantise(rows)
    n, off = np.arange(len(pos))[:, None], pos.numpy() % T
    for h in range(rows.shape[1]):
        page = got[pos.numpy() // T, h]
        assert np.array_equal(page[n, ex[kv, off, :1]][:, 0], e[:, h])
        assert np.array_equal(page[n, scale[kv, off, ::16]], s[:, h])
        assert np.array_equal(page[n, code[kv, off]] >> shift[kv, off] & 15, c[:, h])


@pytest.mark.parametrize("kind,d,rot,layout,amplitude", [("bf16", 128, 128, "half", 2.0 ** 60), ("bf16", 64, 32, "interleaved", 2.0 ** 100),
                                                         ("bf16", 128, 48, "half", 3.4e38), ("fp16", 64, 64, "half", 2.0 ** 115)])
def test_keys_turned_beyond_32_bits_count_as_infinite(dd, kind, d, rot, layout, amplitude):
    """Rows whose magnitudes end well below, around and far above what 32 bits hold: the groups beyond it are the NaN code, as they
    are the NaN code of an e4m3 page, and the others keep their values and an exponent that its byte holds."""
    gen = torch.Generator().manual_seed(d + rot)
    N, H = 512, 2
    lo, hi = (60, 110) if kind == "bf16" else (-10, 15)
    if amplitude > 2.0 ** 120:
        lo, hi = -40, 8
    x = torch.randn(N, 2 * H, d, generator=gen) * torch.exp2(torch.randint(lo, hi, (N, 2 * H, d // 16), generator=gen).float()).repeat_interleave(16, -1)
    x = x.to(TYPES[kind])
    if kind == "fp16":
        x = x.clamp(-65504, 65504)
    k, v = x[:, :H], x[:, H:]
    r, turns = rope_of(dd, d, rot, layout, "none", amplitude)
    pos = torch.randperm(N, generator=gen).to(torch.int32)
    got = appended(dd, k, v, pos, r, d)
    want = ref.rotate(f64(k), pos.numpy(), turns, layout, float(np.float32(amplitude)))
    top = float(np.finfo(np.float32).max)
    beyond = np.abs(want) > top
    assert beyond.any() and not beyond.all() and np.isfinite(want).all()
    want[beyond] = np.inf
    check_rows(got, want, 0, pos, d)
    check_rows(got, f64(v), 1, pos, d)


@pytest.mark.parametrize("d,rot,layout,amplitude", [(128, 128, "half", 2.0 ** -133), (64, 32, "interleaved", 2.0 ** -140), (64, 64, "half", 2.0 ** -101),
                                                    (128, 48, "half", 0.0)])
def test_keys_turned_with_the_smallest_amplitudes(dd, d, rot, layout, amplitude):
    """An amplitude that 32 bits hold as a subnormal times rows near the largest of their type: ordinary keys."""
    gen = torch.Generator().manual_seed(d + rot)
    N, H = 512, 2
    x = torch.randn(N, 2 * H, d, generator=gen)
    x[:, :H, :rot] *= 2.0 ** 124
    x = x.to(torch.bfloat16)
    k, v = x[:, :H], x[:, H:]
    r, turns = rope_of(dd, d, rot, layout, "none", amplitude)
    pos = torch.randperm(N, generator=gen).to(torch.int32)
    got = appended(dd, k, v, pos, r, d)
    check_rows(got, ref.rotate(f64(k), pos.numpy(), turns, layout, amplitude), 0, pos, d)
    check_rows(got, f64(v), 1, pos, d)


@pytest.mark.parametrize("kind,d,rot,layout", [("bf16", 128, 128, "half"), ("fp16", 64, 32, "interleaved"), ("bf16", 128, 48, "half"), ("bf16", 64, 0, "half")])
def test_rows_of_zeros(dd, kind, d, rot, layout):
    """Whole rows of zeros of either sign among others, turned and as they are; rows that vanish in 32 bits."""
    gen = torch.Generator().manual_seed(rot + d)
    N, H = 256, 2
    x = torch.randn(N, 2 * H, d, generator=gen)
    x[::3] = 0.0
    x[1::6] = -0.0
    x[2::9, :, 16:] = 0.0
    if kind == "bf16":
        x[4::12] *= 2.0 ** -133
    x = x.to(TYPES[kind])
    k, v = x[:, :H], x[:, H:]
    r, turns = rope_of(dd, d, rot, layout, "none", 1.1) if rot else (None, None)
    pos = torch.randperm(N, generator=gen).to(torch.int32)
    got = appended(dd, k, v, pos, r, d)
    check_rows(got, ref.rotate(f64(k), pos.numpy(), turns, layout, float(np.float32(1.1))) if rot else f64(k), 0, pos, d)
    check_rows(got, f64(v), 1, pos, d)
