"""The 4-bit cache at the ends of what its calls allow."""
import pytest
import torch

from tests._int4_ref import TYPES
from tests.test_gpu_cache import dd, pool_of  # noqa: F401  (dd is the fixture)
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
