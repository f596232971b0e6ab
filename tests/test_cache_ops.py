"""The paged-cache calls without a GPU: sizes, rotary frequencies against their formula, and everything that is refused
before a device is asked for."""
import ctypes

import numpy as np
import pytest
import torch

from tests import _cache_ref as ref


@pytest.fixture(scope="module")
def dd():
    from paper_2607_26475_b200 import binding
    return binding


def test_page_sizes(dd):
    size = dd.lib.dd_cache_page_bytes
    assert size(dd.DD_CACHE_BF16, 16, 128) == 8192 and size(dd.DD_CACHE_FP16, 64, 64) == 16384
    assert size(dd.DD_CACHE_E4M3, 16, 128) == 4096 + 32 and size(dd.DD_CACHE_E4M3, 256, 64) == 32768 + 512
    for bad in [(0, 16, 96), (0, 24, 128), (0, 8, 128), (0, 512, 128), (3, 16, 128), (-1, 16, 128), (0, 0, 128)]:
        assert size(*bad) == 0
    assert dd.lib.dd_cache_decode_attn_workspace(32, 8, 128, 1) > 0
    for bad in [(32, 5, 128, 1), (32, 8, 96, 1), (32, 8, 128, 0), (32, 8, 128, 65), (0, 8, 128, 1), (4096, 1, 128, 1)]:
        assert dd.lib.dd_cache_decode_attn_workspace(*bad) == 0


@pytest.mark.parametrize("rot,base,scaling,kw", [
    (128, 10000.0, "none", {}), (64, 500000.0, "linear", dict(factor=4.0)), (16, 10000.0, "ntk", dict(factor=8.0)),
    (128, 500000.0, "parts", dict(factor=8.0, original_len=8192.0, low=1.0, high=4.0)),
    (64, 10000.0, "parts", dict(factor=40.0, original_len=4096.0, low=1.0, high=32.0))])
def test_rotary_frequencies(dd, rot, base, scaling, kw):
    modes = dict(none=dd.DD_ROPE_NONE, linear=dd.DD_ROPE_LINEAR, ntk=dd.DD_ROPE_NTK, parts=dd.DD_ROPE_BY_PARTS)
    args = dict(kw)
    if "low" in args:
        args["low_turns"], args["high_turns"] = args.pop("low"), args.pop("high")
    r = dd.Rope(head_dim=128, rot_dim=rot, base=base, scaling=modes[scaling], device="cpu", **args)
    want = ref.turns_of(rot, base, scaling, **kw)
    # a few operations and one power in 64 bits on either side
    np.testing.assert_allclose(r.turns.numpy(), want, rtol=64 * 2.0 ** -53)
    if scaling == "parts":                       # both ends of the ramp are met
        plain = ref.turns_of(rot, base)
        assert r.turns[0] == plain[0] and np.isclose(r.turns[-1], plain[-1] / kw["factor"], rtol=1e-14)


@pytest.mark.parametrize("kw", [dict(rot_dim=24), dict(rot_dim=0), dict(rot_dim=144), dict(base=1.0), dict(base=float("nan")),
                                dict(scaling=7), dict(scaling=1, factor=0.0), dict(scaling=1, factor=float("inf")),
                                dict(scaling=3, factor=8.0), dict(scaling=3, factor=8.0, original_len=100.0, low_turns=4.0, high_turns=4.0)])
def test_rotary_frequencies_refused(dd, kw):
    with pytest.raises(dd.DDError) as e:
        dd.Rope(head_dim=128, device="cpu", **kw)
    assert e.value.code == dd.DD_ERR_INVALID_ARG and "dd_rope_turns" in str(e.value)


def _cache(dd, **kw):
    c = dict(data=1 << 20, format=dd.DD_CACHE_E4M3, n_kv_heads=2, head_dim=128, page_tokens=16, n_blocks=4,
             block_stride=2 * 4128, head_stride=4128, block_table=1 << 21, batch=2, max_pages=2, table_stride=2, status=None)
    c.update(kw)
    return dd.DDCache(*c.values())


def _rows(dd, **kw):
    r = dict(data=1 << 22, dtype=dd.DD_BF16, n_heads=2, token_stride=256, head_stride=128)
    r.update(kw)
    return dd.DDRows(*r.values())


BAD_CACHES = [(dict(data=None), "data is NULL"), (dict(data=(1 << 20) + 8), "not 16-byte aligned"), (dict(format=5), "not supported"),
              (dict(head_dim=96), "not supported"), (dict(page_tokens=20), "not supported"), (dict(n_kv_heads=0), "positive"),
              (dict(n_blocks=0), "positive"), (dict(batch=0), "positive"), (dict(max_pages=0), "positive"),
              (dict(max_pages=1 << 27, table_stride=1 << 27), "31 bits"), (dict(table_stride=1), "table_stride"),
              (dict(block_stride=4096 + 8), "multiples of 16"), (dict(block_stride=-8256), "non-negative"),
              (dict(head_stride=4112), "overlap"), (dict(block_stride=4112), "overlap"), (dict(block_table=None), "block_table is NULL")]


@pytest.mark.parametrize("kw,text", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(dd, kw, text):
    """The pointers are invented: each call has to stop at the named argument before it asks about them."""
    c, k = _cache(dd, **kw), _rows(dd)
    calls = [lambda: dd.lib.dd_cache_append(c, 2, 1 << 23, None, k, k, None, None, None, None),
             lambda: dd.lib.dd_cache_read(c, 1 << 23, 1, 1 << 24, dd.DD_BF16, None),
             lambda: dd.lib.dd_cache_decode_attn(c, 1, k, 1 << 23, k, None, 0, 0.0, 1 << 24, 1 << 30, None)]
    for call in calls:
        assert call() == dd.DD_ERR_INVALID_ARG
        assert text in dd.lib.dd_last_error_message(None).decode()


def test_bad_arguments_are_refused(dd):
    lib, bad = dd.lib, dd.DD_ERR_INVALID_ARG
    c, k, p = _cache(dd), _rows(dd), 1 << 23
    rope = dd.DDRope(1 << 24, 128, dd.DD_ROPE_HALF, 1.0)

    def refuses(rc, text):
        assert rc == bad and text in lib.dd_last_error_message(None).decode(), lib.dd_last_error_message(None)

    for kw, text in [(dict(dtype=9), "unknown dtype"), (dict(n_heads=0), "no heads"), (dict(token_stride=12), "multiples of 8"),
                     (dict(head_stride=-128), "non-negative"), (dict(data=None), "k is NULL"), (dict(n_heads=3), "2 heads"),
                     (dict(dtype=dd.DD_FP16), "differ in type")]:
        refuses(lib.dd_cache_append(c, 2, p, None, _rows(dd, **kw), k, None, None, None, None), text)
    refuses(lib.dd_cache_append(c, 3, p, None, k, k, None, None, None, None), "multiple of batch")
    refuses(lib.dd_cache_append(c, -1, p, None, k, k, None, None, None, None), "negative")
    refuses(lib.dd_cache_append(c, 2, p, None, k, k, None, k, k, None), "rope, which is NULL")
    refuses(lib.dd_cache_append(c, 2, p, None, k, k, rope, k, None, None), "go together")
    refuses(lib.dd_cache_append(c, 2, p, None, k, k, rope, k, _rows(dd, head_stride=64), None), "overlap")
    refuses(lib.dd_cache_append(c, 2, p, None, k, None, None, None, None, None), "v is NULL")
    refuses(lib.dd_cache_append(_cache(dd, format=dd.DD_CACHE_FP16, head_stride=8192, block_stride=16384), 2, p, None, k, k, None, None, None, None), "own type")
    assert lib.dd_cache_append(c, 0, None, None, None, None, None, None, None, None) == dd.DD_OK
    for r, text in [(dd.DDRope(1 << 24, 24, 0, 1.0), "rot_dim"), (dd.DDRope(1 << 24, 128, 2, 1.0), "layout"),
                    (dd.DDRope(1 << 24, 128, 0, float("inf")), "amplitude"), (dd.DDRope(None, 128, 0, 1.0), "turns is NULL")]:
        refuses(lib.dd_rope_apply(r, 128, 2, p, k, None, k, None, 0, None), text)
        refuses(lib.dd_cache_append(c, 2, p, None, k, k, r, None, None, None), text)
    refuses(lib.dd_rope_apply(rope, 64, 2, p, k, None, k, None, 0, None), "rot_dim")
    refuses(lib.dd_rope_apply(rope, 96, 2, p, k, None, k, None, 0, None), "head_dim")
    refuses(lib.dd_rope_apply(rope, 128, 2, p, None, None, None, None, 0, None), "neither")
    refuses(lib.dd_rope_apply(rope, 128, 2, p, k, None, None, None, 0, None), "go together")
    refuses(lib.dd_rope_apply(rope, 128, 2, p, k, None, k, None, 2, None), "backward")
    refuses(lib.dd_rope_apply(rope, 128, 2, p, k, _rows(dd, dtype=dd.DD_FP16), k, _rows(dd, dtype=dd.DD_FP16), 0, None), "differ in type")
    refuses(lib.dd_rope_apply(None, 128, 2, p, k, None, k, None, 0, None), "rope is NULL")
    assert lib.dd_rope_apply(rope, 128, 0, None, k, None, k, None, 0, None) == dd.DD_OK
    refuses(lib.dd_cache_read(c, p, -1, p, dd.DD_BF16, None), "negative")
    refuses(lib.dd_cache_read(c, p, 1, p, 4, None), "out_dtype")
    refuses(lib.dd_cache_read(_cache(dd, format=dd.DD_CACHE_BF16, head_stride=8192, block_stride=16384), p, 1, p, dd.DD_FP16, None), "own type")
    refuses(lib.dd_cache_read(None, p, 1, p, dd.DD_BF16, None), "cache is NULL")
    assert lib.dd_cache_read(c, None, 0, None, dd.DD_BF16, None) == dd.DD_OK

    def attn(cache=c, tq=1, q=k, out=k, window=0, scale=0.0):
        return lib.dd_cache_decode_attn(cache, tq, q, p, out, None, window, scale, p, 1 << 30, None)
    refuses(attn(tq=0), "n_q_tokens")
    refuses(attn(tq=65), "n_q_tokens")
    refuses(attn(q=_rows(dd, n_heads=3)), "multiple of n_kv_heads")
    refuses(attn(out=_rows(dd, n_heads=4, token_stride=512)), "differ in heads")
    refuses(attn(out=_rows(dd, token_stride=64)), "overlap")
    refuses(attn(out=_rows(dd, token_stride=128, head_stride=128)), "overlap")          # token 1 of head 0 is token 0 of head 1
    refuses(attn(out=_rows(dd, token_stride=128, head_stride=128), tq=2), "overlap")
    assert attn(out=_rows(dd, token_stride=128, head_stride=256)) == bad                # head-major is fine: the next check refuses
    assert "overlap" not in lib.dd_last_error_message(None).decode()
    refuses(attn(window=-1), "window")
    refuses(attn(scale=-1.0), "scale")
    refuses(attn(scale=float("nan")), "scale")
    refuses(attn(scale=float("inf")), "scale")
    refuses(attn(q=None), "q is NULL")


def test_python_side_refuses_wrong_shapes_and_types(dd):
    data = torch.zeros(4, 2, 4128, dtype=torch.uint8)
    table = torch.zeros(2, 2, dtype=torch.int32)
    for d, t, kw in [(data[:, :, :4096], table, {}), (data, table.long(), {}), (data, table[0], {}), (data, table.t()[:, ::2], dict(page_tokens=32)),
                     (data, table, dict(head_dim=96)), (data, table[:0], {}), (data[0], table, {})]:
        with pytest.raises(dd.DDError):
            dd.PagedCache(d, t, cache_format=dd.DD_CACHE_E4M3, **kw)
    with pytest.raises(dd.DDError) as e:
        dd.PagedCache(data, table, cache_format=dd.DD_CACHE_E4M3, n_blocks=4, block_stride=2 * 4128, head_stride=4144, n_kv_heads=2)
    assert "behind the end" in str(e.value)
    c = dd.PagedCache(data, table, cache_format=dd.DD_CACHE_E4M3)
    k, pos = torch.zeros(2, 2, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    for args in [(k.float(), k, pos), (k[:, :, :64], k, pos), (k, k[:1], pos), (k.transpose(0, 2).contiguous().transpose(0, 2), k, pos),
                 (k, k, pos.long()), (k, k, pos, pos[:1])]:
        with pytest.raises(dd.DDError) as e:
            c.append(*args)
        assert e.value.code == dd.DD_ERR_INVALID_ARG
    q = torch.zeros(2, 1, 4, 128, dtype=torch.bfloat16)
    for args in [(q[:1], pos, q[:1]), (q, pos[:1], q), (q, pos, q.float()), (q, pos, q, torch.zeros(2, 1, 4, dtype=torch.float64)),
                 (q, pos, q, torch.zeros(2, 4))]:
        with pytest.raises(dd.DDError):
            c.decode_attn(*args, workspace=torch.zeros(16))
    wide = torch.zeros(2, 4, 4, 128, dtype=torch.bfloat16)[:, :2]      # two tokens of each request, a gap between requests
    with pytest.raises(dd.DDError):
        c.decode_attn(wide, pos, wide, workspace=torch.zeros(16))
    for idx, out in [(torch.zeros(2, 2, 1, dtype=torch.int32), torch.zeros(2, 2, 2, 16, 128)), (torch.zeros(1, 2, 1, dtype=torch.int32), torch.zeros(2, 2, 2, 16, 128, dtype=torch.bfloat16)),
                     (torch.zeros(2, 2, 1, dtype=torch.int64), torch.zeros(2, 2, 2, 16, 128, dtype=torch.bfloat16)),
                     (torch.zeros(2, 2, 2, dtype=torch.int32), torch.zeros(2, 2, 2, 16, 128, dtype=torch.bfloat16))]:
        with pytest.raises(dd.DDError):
            c.read(idx, out)


def test_reference_quantiser_against_torch():
    """The definition the kernels are held to agrees with torch's e4m3 cast where both are defined."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(200, 64, generator=g).to(torch.bfloat16) * torch.exp2(torch.randint(-20, 20, (200, 1), generator=g).float()).to(torch.bfloat16)
    code, ex = ref.quantise(x.double().numpy())
    back = torch.from_numpy(ref.CODES[code])
    y = torch.ldexp(x.double(), torch.from_numpy(127 - ex.astype(np.int64)).unsqueeze(-1).int())
    assert torch.equal(y.float().to(torch.float8_e4m3fn).double(), back)
    top = y.abs().amax(-1)
    assert bool((top <= 448).all()) and bool((top > 224).all())


def test_store_format_of_a_context(dd):
    """A quantised store is taken with the zero-copy gather only; other formats and engines are refused before a device is
    asked for."""
    cfg = dd.DDConfig(n_layers=2, batch=2, n_q_heads=32, n_kv_heads=8, head_dim=128, page_tokens=16, max_pages=64, k_pages=8,
                      n_q_tokens=2, ring_depth=2, store_format=dd.DD_CACHE_E4M3)
    assert dd.lib.dd_slot_bytes(cfg) == 2 * 8 * 8 * 8192                      # slots stay bf16
    for kw in (dict(gather_mode=dd.DD_GATHER_BULK), dict(gather_mode=dd.DD_GATHER_STAGED), dict(store_format=dd.DD_CACHE_FP16),
               dict(store_format=-1)):
        bad = dd.DDConfig.from_buffer_copy(cfg)
        for k, v in kw.items():
            setattr(bad, k, v)
        assert dd.lib.dd_slot_bytes(bad) == 0
        h = ctypes.c_void_p()
        assert dd.lib.dd_create(bad, ctypes.byref(h)) == dd.DD_ERR_INVALID_ARG
        assert b"store" in dd.lib.dd_last_error_message(None)
