"""What the Python side of the paged cache refuses by itself, without a GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def dd():
    from paper_2607_26475_b200 import binding
    return binding


def refused(dd, call, text):
    with pytest.raises(dd.DDError) as e:
        call()
    assert e.value.code == dd.DD_ERR_INVALID_ARG and text in str(e.value)


def test_a_workspace_that_is_not_dense_is_refused(dd):
    """Its size says nothing about the memory behind it: an expanded one has a single byte."""
    c = dd.PagedCache(torch.zeros(4, 2, 8192, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.int32))
    q, lens = torch.zeros(2, 1, 4, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    for workspace in (torch.zeros(1, dtype=torch.uint8).expand(1 << 30), torch.zeros(64, 2, dtype=torch.uint8)[:, 0]):
        refused(dd, lambda: c.decode_attn(q, lens, q, workspace=workspace), "workspace must be dense")


def test_empty_pools_and_missing_sizes_are_refused(dd):
    table = torch.zeros(1, 1, dtype=torch.int32)
    for shape in ((0, 2, 8192), (2, 0, 8192)):
        refused(dd, lambda: dd.PagedCache(torch.zeros(shape, dtype=torch.uint8), table), "empty")
    for shape in ((0, 1, 1, 8192), (1, 0, 1, 8192), (1, 1, 0, 8192)):
        refused(dd, lambda: dd.PagedCache.of_store(torch.zeros(shape, dtype=torch.uint8), device="cpu"), "empty")
    flat = torch.zeros(2 * 8192, dtype=torch.uint8)
    sizes = dict(n_blocks=2, block_stride=8192, head_stride=8192, n_kv_heads=1)
    assert dd.PagedCache(flat, table, **sizes).c.n_blocks == 2
    for missing in ("block_stride", "head_stride", "n_kv_heads"):
        refused(dd, lambda: dd.PagedCache(flat, table, **{k: v for k, v in sizes.items() if k != missing}), "go together")
    for zero in ("n_blocks", "n_kv_heads"):
        refused(dd, lambda: dd.PagedCache(flat, table, **{**sizes, zero: 0}), "empty")
