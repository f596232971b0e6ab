"""The 4-bit cache and the calls on listed pages without a GPU: sizes, the definitions that the kernels are held to, and everything
that is refused before a device is asked for."""
import numpy as np
import pytest
import torch

from tests import _cache_ref as ref
from tests import _int4_ref as ref4
from tests.test_cache_ops import BAD_CACHES, _cache, _rows, dd  # noqa: F401  (dd is the fixture)


def test_sizes(dd):
    size = dd.lib.dd_cache_page_bytes
    for T in (16, 32, 64, 128, 256):
        for d in (64, 128):
            assert size(dd.DD_CACHE_INT4, T, d) == ref4.page_bytes("int4", T, d) == T // 16 * (18 * d + 32)
    assert size(dd.DD_CACHE_INT4, 16, 96) == 0 and size(dd.DD_CACHE_INT4, 8, 128) == 0
    assert dd.lib.dd_cache_landmark_bytes(128) == 144 and dd.lib.dd_cache_landmark_bytes(64) == 80 and dd.lib.dd_cache_landmark_bytes(96) == 0
    work = dd.lib.dd_cache_select_workspace
    assert work(1, 8, 2048) == 8 * (2048 * 4 + 128) and work(3, 1, 1) == 3 * (32 * 4 + 128)
    assert work(1 << 20, 8, 2048) == (64 << 20) + 1024 * 8 * 128 and work(1 << 20, 8, 1 << 20) == 64 * 8 * ((1 << 22) + 128)
    for bad in [(0, 8, 16), (1, 0, 16), (1, 8, 0), (-1, 8, 16)]:
        assert work(*bad) == 0
    one = dd.lib.dd_cache_decode_attn_workspace(32, 8, 128, 1)
    assert dd.lib.dd_cache_sparse_attn_workspace(8, 32, 8, 128, 64) == one > 0
    # many tokens of up to four heads: room for the pairs' lists and their lengths
    assert dd.lib.dd_cache_sparse_attn_workspace(2001, 32, 8, 128, 64) == one + 1001 * 8 * 128 * 4 + 4016
    assert dd.lib.dd_cache_sparse_attn_workspace(2001, 40, 8, 128, 64) == dd.lib.dd_cache_decode_attn_workspace(40, 8, 128, 1)
    for bad in [(8, 32, 5, 128, 1), (8, 32, 8, 96, 1), (8, 0, 8, 128, 1), (8, 4096, 1, 128, 1), (0, 32, 8, 128, 1), (8, 32, 8, 128, 0)]:
        assert dd.lib.dd_cache_sparse_attn_workspace(*bad) == 0


@pytest.mark.parametrize("T,d", [(16, 64), (32, 128), (256, 64)])
def test_every_byte_of_a_page_has_one_owner(T, d):
    code, shift, scale, ex = ref4.places(T, d)
    used = np.concatenate([np.unique(code * 2 + shift // 4) // 2, np.unique(scale), np.unique(ex)])
    assert len(np.unique(code * 2 + shift // 4)) == 2 * T * d
    counts = np.bincount(used, minlength=ref4.page_bytes("int4", T, d))
    assert counts.max() == 2 and counts.min() == 1 and (counts == 2).sum() == T * d and len(used) == 2 * T * d + 2 * T * d // 16 + 2 * T


def test_quantised_rows_are_as_near_as_they_say():
    rng = np.random.RandomState(0)
    x = torch.from_numpy(rng.randn(300, 128) * np.exp2(rng.randint(-30, 30, (300, 1)))).to(torch.bfloat16).double().numpy()
    codes, scales, ex = ref4.quantise(x)
    assert codes.min() >= 1 and codes.max() <= 15 and scales.min() >= 0x18
    step = ref.CODES[scales].repeat(16, -1) * np.exp2(ex.astype(np.float64) - 127)[:, None]
    back = (codes.astype(np.float64) - 8) * step
    # half a step, and what the scale's own rounding (2^-4 of it) cuts off the seventh
    assert np.all(np.abs(back - x) <= step * (0.5 + 7 * 2.0 ** -4))
    assert np.all((ref.CODES[scales].max(-1) >= 224) & (ref.CODES[scales].max(-1) <= 448))
    assert np.array_equal(torch.from_numpy(back).to(torch.bfloat16).double().numpy(), back)      # 7 significant bits
    pages = ref4.encode_pages(np.stack([x[:160].reshape(10, 16, 128), x[140:].reshape(10, 16, 128)], 1), "int4")
    v = ref4.decode_pages(pages, "int4", 16, 128)
    assert np.array_equal(v[:, 0].reshape(160, 128), back[:160]) and np.array_equal(v[:, 1].reshape(160, 128), back[140:])


def test_reference_attention_over_listed_pages_is_that_over_all_of_them():
    rng = np.random.RandomState(1)
    v = rng.randn(5, 2, 2, 16, 64)
    raw = ref4.encode_pages(v, "int4")
    table, q = np.array([[3, 0, 4, 1]]), rng.randn(1, 1, 6, 64)
    all_, lse, _, _ = ref4.attention(q, raw, table, [50], "int4", 16)
    got, got_lse, _, _ = ref4.listed_attention(q[0], raw, table, [0], [49], np.tile(np.array([2, 0, 3, 1], dtype=np.int32), (1, 2, 1)), "int4", 16)
    assert np.allclose(all_[0], got, rtol=0, atol=1e-13) and np.allclose(lse[0], got_lse, rtol=0, atol=1e-13)


def test_selection_of_one_head_is_top_k_of_dot_products():
    rng = np.random.RandomState(2)
    keys, q = rng.randint(-127, 128, (40, 16, 64)).astype(np.float64), rng.randint(-127, 128, (1, 64)).astype(np.float64)
    keys[:] = keys.mean(1, keepdims=True).round()                    # means that are their own landmarks
    lm = np.stack([ref4.landmark(k) for k in keys])
    z = keys.mean(1) @ q[0]
    got = ref4.select(q, lm, 9, 0, 1, 39)
    want = set(np.argsort(-z[:39], kind="stable")[:8]) | {39}
    assert set(got) == want and list(got) == sorted(got)


@pytest.mark.parametrize("kw,text", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(dd, kw, text):
    """The pointers are invented: each call has to stop at the named argument before it asks about them."""
    c, k = _cache(dd, **kw), _rows(dd)
    calls = [lambda: dd.lib.dd_cache_landmarks(c, 1 << 23, 0, 1 << 24, None),
             lambda: dd.lib.dd_cache_select(c, 2, 1 << 23, None, k, 1 << 24, 1, 0, 1, 1 << 25, 1 << 26, 1 << 30, None),
             lambda: dd.lib.dd_cache_sparse_attn(c, 2, 1 << 23, None, k, 1 << 24, 1, k, None, 0.0, 1 << 26, 1 << 30, None)]
    for call in calls:
        assert call() == dd.DD_ERR_INVALID_ARG
        assert text in dd.lib.dd_last_error_message(None).decode()


def test_bad_arguments_are_refused(dd):
    lib, bad = dd.lib, dd.DD_ERR_INVALID_ARG
    c, r, p = _cache(dd), _rows(dd), 1 << 23

    def refuses(rc, text):
        assert rc == bad and text in lib.dd_last_error_message(None).decode(), lib.dd_last_error_message(None)

    refuses(lib.dd_cache_landmarks(c, p, -1, p, None), "n_last")
    refuses(lib.dd_cache_landmarks(None, p, 0, p, None), "cache is NULL")

    def select(n=2, requests=None, q=r, k=3, first=0, recent=1):
        return lib.dd_cache_select(c, n, p, requests, q, p, k, first, recent, p, p, 1 << 30, None)
    refuses(select(n=-1), "negative")
    refuses(select(n=3), "multiple of batch")
    refuses(select(recent=0), "recent_pages >= 1")
    refuses(select(first=-1), "first_pages >= 0")
    refuses(select(k=0), "k_pages")
    refuses(select(first=2, recent=2), "must hold")
    refuses(select(first=2 ** 31 - 1, recent=2 ** 31 - 1), "must hold")
    refuses(select(q=None), "q is NULL")
    refuses(select(q=_rows(dd, n_heads=3)), "multiple of n_kv_heads")
    refuses(select(q=_rows(dd, dtype=7)), "unknown dtype")
    assert select(n=0) == dd.DD_OK

    def attend(n=2, requests=None, q=r, out=r, k=3, scale=0.0, cache=c):
        return lib.dd_cache_sparse_attn(cache, n, p, requests, q, p, k, out, None, scale, p, 1 << 30, None)
    refuses(attend(n=-1), "negative")
    refuses(attend(n=3), "multiple of batch")
    refuses(attend(k=0), "k_pages")
    for scale in (-1.0, float("nan"), float("inf")):
        refuses(attend(scale=scale), "scale")
    refuses(attend(q=None), "q is NULL")
    refuses(attend(q=_rows(dd, n_heads=3), out=_rows(dd, n_heads=3, token_stride=384)), "multiple of n_kv_heads")
    refuses(attend(out=_rows(dd, n_heads=4, token_stride=512)), "differ in heads")
    refuses(attend(out=_rows(dd, dtype=dd.DD_FP16)), "differ in heads or type")
    refuses(attend(out=_rows(dd, token_stride=128)), "overlap")
    refuses(attend(cache=_cache(dd, format=dd.DD_CACHE_FP16, head_stride=8192, block_stride=16384)), "own type")
    assert attend(n=0) == dd.DD_OK


def test_python_side_refuses_wrong_shapes_and_types(dd):
    c = dd.PagedCache(torch.zeros(4, 2, 2336, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.int32), cache_format=dd.DD_CACHE_INT4)
    with pytest.raises(dd.DDError):
        dd.PagedCache(torch.zeros(4, 2, 2335, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.int32), cache_format=dd.DD_CACHE_INT4)
    lm, pos, q = c.new_landmarks(), torch.zeros(6, dtype=torch.int32), torch.zeros(6, 4, 128, dtype=torch.bfloat16)
    idx, ws = torch.zeros(6, 2, 3, dtype=torch.int32), torch.zeros(16, dtype=torch.uint8)
    assert lm.shape == (4, 2, 144)
    bad = [lambda: c.update_landmarks(lm[:3], pos[:2]), lambda: c.update_landmarks(lm.int(), pos[:2]), lambda: c.update_landmarks(lm, pos),
           lambda: c.update_landmarks(lm, pos[:2], n_last=-1), lambda: c.update_landmarks(lm, pos[:2], n_last=1 << 31)]
    for x in (dict(q=q[:5]), dict(q=q.float()), dict(q=q[..., :64]), dict(positions=pos.long()), dict(positions=pos[:5]), dict(positions=pos.view(2, 3)),
              dict(idx=idx[:5]), dict(idx=idx.long()), dict(idx=idx[:, :1]), dict(idx=idx[..., 0]), dict(idx=idx[..., :0]), dict(idx=idx.transpose(0, 1)),
              dict(requests=pos[:5]), dict(requests=pos.float()), dict(workspace=ws.expand(2, 16))):
        a = dict(q=q, positions=pos, idx=idx, requests=pos, workspace=ws) | x
        bad.append(lambda a=a: c.select(a["q"], lm, a["positions"], a["idx"], a["requests"], workspace=a["workspace"]))
        bad.append(lambda a=a: c.sparse_attn(a["q"], a["idx"], a["positions"], torch.empty_like(a["q"]), None, a["requests"], workspace=a["workspace"]))
    bad += [lambda: c.select(q, lm[:, :1], pos, idx, workspace=ws), lambda: c.sparse_attn(q, idx, pos, q[:, :2], workspace=ws),
            lambda: c.sparse_attn(q, idx, pos, q.half(), workspace=ws, stream=0), lambda: c.sparse_attn(q, idx, pos, q, torch.zeros(6, 3), workspace=ws),
            lambda: c.sparse_attn(q, idx, pos, q, torch.zeros(6, 4, dtype=torch.float64), workspace=ws)]
    for call in bad:
        with pytest.raises(dd.DDError) as e:
            call()
        assert e.value.code == dd.DD_ERR_INVALID_ARG


def test_calls_without_tokens_do_nothing(dd):
    c = dd.PagedCache(torch.zeros(4, 2, 2336, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.int32), cache_format=dd.DD_CACHE_INT4)
    q, pos, idx = torch.zeros(0, 4, 128, dtype=torch.bfloat16), torch.zeros(0, dtype=torch.int32), torch.zeros(0, 2, 3, dtype=torch.int32)
    ws = torch.zeros(16, dtype=torch.uint8)
    c.select(q, c.new_landmarks(), pos, idx, workspace=ws, stream=0)
    c.sparse_attn(q, idx, pos, torch.empty_like(q), workspace=ws, stream=0)
    c.append(q[:, :2], q[:, :2], pos, pos, stream=0)


def test_numbers_beyond_31_bits_are_refused(dd):
    c = dd.PagedCache(torch.zeros(4, 2, 2336, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.int32), cache_format=dd.DD_CACHE_INT4)
    q, pos, idx = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2, 3, dtype=torch.int32)
    ws = torch.zeros(4096, dtype=torch.uint8)
    for more in (dict(first_pages=1 << 32), dict(recent_pages=(1 << 32) + 1), dict(first_pages=-1), dict(recent_pages=0)):
        with pytest.raises(dd.DDError) as e:
            c.select(q, c.new_landmarks(), pos, idx, workspace=ws, stream=0, **more)
        assert e.value.code == dd.DD_ERR_INVALID_ARG
    assert dd.lib.dd_cache_select_workspace(1, 1, (1 << 31) - 1) == 0
    assert dd.lib.dd_cache_select_workspace(1, 70000, 16) == 0
