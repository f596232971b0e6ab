"""Error reports of the paged cache, and its calls, on streams other than the current one."""
import pytest
import torch

from tests.test_gpu_cache import dd, make_attn, rope_of, run_attn  # noqa: F401  (dd is the fixture)

pytestmark = pytest.mark.gpu

LATE = 100_000_000                 # clock cycles that keep a stream busy: 50 ms or more


def late_stream():
    """A stream that waits for everything enqueued so far and then for LATE cycles."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(LATE)
    return side


@pytest.mark.parametrize("call", ["append", "read", "decode_attn"])
def test_reports_of_calls_still_running_on_another_stream_are_seen(dd, call):
    gen = torch.Generator().manual_seed(21)
    cache, raw, table, q = make_attn(dd, gen, [40, 64], 1, 4, 128, 16, "bf16", "bf16", 1)
    M = table.shape[1]
    kv = torch.zeros(2, 1, 128, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([M * 16, -1], dtype=torch.int32).cuda()              # behind the table, padding
    idx = torch.full((2, 1, 1), -9, dtype=torch.int32, device="cuda")
    pages, out = torch.empty(2, 1, 2, 16, 128, dtype=torch.bfloat16, device="cuda"), torch.empty_like(q)
    lens = torch.tensor([40, -3], dtype=torch.int32).cuda()

    def run(**kw):
        if call == "append":
            cache.append(kv, kv, at, **kw)
        elif call == "read":
            cache.read(idx, pages, **kw)
        else:
            cache.decode_attn(q, lens, out, **kw)

    run()                                                                  # a kernel's first launch may wait for the device
    torch.cuda.synchronize()
    cache.device_error()
    for give in (lambda s: s, lambda s: s.cuda_stream, None):
        side = late_stream()
        with torch.cuda.stream(side if give is None else torch.cuda.current_stream()):
            run(**({} if give is None else dict(stream=give(side))))
        assert not side.query()                                            # the call has not run yet
        assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, {"append": M, "read": -9, "decode_attn": -3}[call])
        assert side.query() and cache.device_error() == (0, 0)


def test_a_cache_made_on_a_busy_stream_reports_calls_of_another(dd):
    """Setting the error word up belongs to the stream that the cache is made on; a call on another stream comes after it."""
    gen = torch.Generator().manual_seed(22)
    old, raw, table, q = make_attn(dd, gen, [40], 1, 4, 128, 16, "bf16", "bf16", 1)
    idx = torch.full((1, 1, 1), -9, dtype=torch.int32, device="cuda")
    pages = torch.empty(1, 1, 2, 16, 128, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    side = late_stream()
    with torch.cuda.stream(side):
        cache = dd.PagedCache(old.data, old.block_table, head_dim=128)
    assert not side.query()                                                # making one does not wait
    cache.read(idx, pages)
    torch.cuda.synchronize()
    assert cache.device_error() == (dd.DD_ERR_INDEX_RANGE, -9)
    assert cache.device_error() == (0, 0)


def test_calls_run_on_the_stream_they_are_given(dd):
    """What another stream writes before the call is there when the call runs: inputs arrive late on that stream."""
    gen = torch.Generator().manual_seed(23)
    B, H, G, d, T = 2, 2, 4, 128, 16
    cache, raw, table, q = make_attn(dd, gen, [40, 64], H, G, d, T, "bf16", "bf16", 1, poison=False)
    r, _ = rope_of(dd, d, 128)
    x = torch.randn(B, H * G, d, generator=gen).to(torch.bfloat16).cuda()
    kv = torch.randn(B, H, d, generator=gen).to(torch.bfloat16).cuda()
    pos = torch.tensor([39, 63], dtype=torch.int32).cuda()
    idx = torch.tensor([2, 3], dtype=torch.int32).view(B, 1, 1).expand(B, H, 1).contiguous().cuda()

    def steps(x, kv, **kw):
        turned, pages = torch.empty_like(x), torch.empty(B, H, 2, T, d, dtype=torch.bfloat16, device="cuda")
        r.apply(pos, x, None, turned, None, **kw)
        cache.append(kv, kv, pos, **kw)
        cache.read(idx, pages, **kw)
        return turned, pages

    steps(torch.zeros_like(x), torch.zeros_like(kv))                       # a kernel's first launch may wait for the device
    late_x, late_kv = torch.zeros_like(x), torch.zeros_like(kv)
    torch.cuda.synchronize()
    side = late_stream()
    with torch.cuda.stream(side):
        late_x.copy_(x)
        late_kv.copy_(kv)
    got = steps(late_x, late_kv, stream=side)
    assert not side.query()
    side.synchronize()
    want = steps(x, kv)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and cache.device_error() == (0, 0)


def test_own_workspace_belongs_to_the_stream_of_the_call(dd, monkeypatch):
    """A workspace of the call's own comes from the allocator's pool of the very stream it is used on, the default one (0) among
    them: memory of another stream's pool could be handed out there while the call still runs."""
    gen = torch.Generator().manual_seed(24)
    cache, raw, table, q = make_attn(dd, gen, [40], 1, 4, 128, 16, "bf16", "bf16", 1)
    lens, out = torch.tensor([40], dtype=torch.int32).cuda(), torch.empty_like(q)
    taken_on, empty = [], torch.empty

    def watch(*args, **kw):
        taken_on.append(torch.cuda.current_stream().cuda_stream)
        return empty(*args, **kw)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    monkeypatch.setattr(dd.torch, "empty", watch)
    for current in (torch.cuda.default_stream(), side):
        for stream in (0, side.cuda_stream, side, torch.cuda.default_stream()):
            with torch.cuda.stream(current):
                cache.decode_attn(q, lens, out, stream=stream)
            torch.cuda.synchronize()
            assert taken_on.pop() == (stream if isinstance(stream, int) else stream.cuda_stream)
    assert not taken_on
