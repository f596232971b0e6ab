"""Attention over the cache with many query rows per KV head: several row tiles, up to the limits of the call."""
import pytest
import torch

from tests.test_gpu_cache import check_attn, dd, make_attn, run_attn  # noqa: F401  (dd is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,H,G,d,T,fmt,kind,Tq,window", [
    ([70, 5, 200, 0], 1, 5, 128, 16, "bf16", "bf16", 64, 0),          # more query tokens than some requests have
    ([70, 5, 200, 0], 2, 1, 64, 32, "e4m3", "fp16", 64, 33),
    ([500, 3], 1, 8, 128, 16, "e4m3", "bf16", 3, 0),                  # 24 rows: a full and a half-empty row tile
    ([33, 1], 1, 1024, 64, 16, "fp16", "fp16", 1, 0),
    ([150], 2, 130, 128, 16, "bf16", "bf16", 2, 100),
    ([40], 1, 1024, 128, 16, "e4m3", "bf16", 2, 0),
    ([900] * 20, 2, 40, 64, 16, "e4m3", "bf16", 1, 0),                # long enough to be cut, several row tiles each
])
def test_many_query_rows(dd, lens, H, G, d, T, fmt, kind, Tq, window):
    gen = torch.Generator().manual_seed(sum(lens) + G + Tq)
    cache, raw, table, q = make_attn(dd, gen, lens, H, G, d, T, fmt, kind, Tq)
    out, lse = run_attn(cache, q, lens, window)
    assert cache.device_error() == (0, 0)
    check_attn(out, lse, q, raw, table, lens, fmt, kind, T, window)


def test_more_rows_than_the_call_takes_are_refused(dd):
    gen = torch.Generator().manual_seed(31)
    cache, raw, table, q = make_attn(dd, gen, [40], 1, 1025, 64, 16, "bf16", "bf16", 1)
    out, lens = torch.full_like(q, 7.0), torch.tensor([40], dtype=torch.int32).cuda()
    with pytest.raises(dd.DDError) as e:
        cache.decode_attn(q, lens, out)
    assert "1024" in str(e.value)
    cache, raw, table, q = make_attn(dd, gen, [40], 1, 1, 64, 16, "bf16", "bf16", 65)
    with pytest.raises(dd.DDError) as e:
        cache.decode_attn(q, lens, torch.empty_like(q))
    assert "64" in str(e.value)
