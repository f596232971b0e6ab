"""The sparse path over a quantised KV store: pages of 4128 bytes in page-locked memory instead of 8192. Everything behind
the store sees the bf16 values that the codes stand for, so every result is compared bit for bit with the same path over a
bf16 store of those values."""
import numpy as np
import pytest
import torch

from oracle import dd_oracle as orc
from paper_2607_26475_b200 import workloads as wl
from tests import _cache_ref as ref
from tests._util import f32, raw16

pytestmark = pytest.mark.gpu

HKV, D, T, PAGE = 8, 128, 16, 4128


@pytest.fixture(scope="module")
def dd():
    from paper_2607_26475_b200 import binding
    return binding


def quantised(kv):
    """bf16 pages [..., 2, T, d] -> (uint8 pages [..., 4128], the bf16 values they stand for)."""
    raw = ref.encode_pages(kv.double().numpy(), "e4m3")
    return torch.from_numpy(raw), torch.from_numpy(ref.decode_pages(raw, "e4m3", T, D)).to(torch.bfloat16)


def test_gather_and_landmarks_are_those_of_the_values(dd):
    B, P, k = 2, 40, 13
    g = torch.Generator().manual_seed(1)
    kv = torch.randn(B, HKV, P, 2, T, D, generator=g).to(torch.bfloat16) * torch.exp2(torch.randint(-9, 9, (B, HKV, P, 2, T, 1), generator=g).float()).to(torch.bfloat16)
    raw, values = quantised(kv)
    idx = torch.stack([torch.stack([torch.randperm(P, generator=g)[:k].sort().values for _ in range(HKV)]) for _ in range(B)]).to(torch.int32)
    ctx_len = torch.tensor([P * T, P * T - 7 * T - 5], dtype=torch.int32)
    for chunk in (0, 4):
        R = T // chunk if chunk else 1
        c = dd.Context(n_layers=1, batch=B, max_pages=P, k_pages=k, store_format=dd.DD_CACHE_E4M3, landmark_chunk_tokens=chunk)
        store = raw.pin_memory()
        c.gather_kv_from_host(store, idx.cuda(), None, 1)
        assert np.array_equal(raw16(c.slot_tensor(1)), orc.gather_kv(raw16(values), idx.numpy()))
        c.gather_kv_from_host(raw.cuda(), idx.cuda(), None, 0)                      # a store on the device
        assert torch.equal(c.slot_tensor(0).view(torch.int16), c.slot_tensor(1).view(torch.int16))
        lm = torch.empty((B, HKV, P * R, D), dtype=torch.bfloat16, device="cuda")
        for where in (store, raw.cuda()):
            lm.fill_(7.0)
            c.build_landmarks(where, ctx_len.cuda(), lm)
            want = orc.build_landmarks(f32(values[:, :, :, 0]), ctx_len.numpy(), chunk_tokens=chunk or None)
            assert np.array_equal(f32(lm), want.reshape(lm.shape))
        assert c.device_error() == (0, 0)
        bad = idx.clone()
        bad[1, 3, 2] = P + 5                                                        # clamped and reported, as ever
        c.gather_kv_from_host(store, bad.cuda(), None, 0)
        assert c.device_error() == (dd.DD_ERR_INDEX_RANGE, P + 5)
        bad[1, 3, 2] = P - 1
        assert np.array_equal(raw16(c.slot_tensor(0)), orc.gather_kv(raw16(values), bad.numpy()))
        with pytest.raises(dd.DDError) as e:
            c.gather_kv_from_host(raw, idx.cuda(), None, 0)
        assert e.value.code == dd.DD_ERR_NOT_PINNED
        c.close()


@pytest.mark.parametrize("correct,depth", [(False, 2), (True, 3)])
def test_pipeline_over_a_quantised_store(dd, correct, depth):
    w = wl.small(wl.CONFIGS[2], n_layers=3, batch=2, ctx=1024, budget=192, steps=3)
    S, L, B = 3, w.n_layers, w.batch
    pairs = [quantised(torch.stack([wl.kv_slab(w, l, b) for b in range(B)])) for l in range(L)]
    ctx_len = wl.ctx_lens(w, ragged=True)
    npg = ((ctx_len + T - 1) // T).to(torch.int32)
    q_init = torch.stack([wl.queries(w, -1, l)[:, 1] for l in range(L)]).cuda()
    q = torch.stack([torch.stack([wl.queries(w, t, l) for l in range(L)]) for t in range(S)]).cuda()
    seen = []
    for fmt, part in ((dd.DD_CACHE_E4M3, 0), (dd.DD_CACHE_BF16, 1)):
        store = [p[part].contiguous().pin_memory() for p in pairs]
        c = dd.Context(n_layers=L, batch=B, max_pages=w.n_pages, k_pages=w.k_pages, ring_depth=depth, miss_correction=correct, store_format=fmt)
        lms = []
        for l in range(L):
            lms.append(torch.empty((B, HKV, w.n_pages, D), dtype=torch.bfloat16, device="cuda"))
            c.build_landmarks(store[l], ctx_len.cuda(), lms[-1])
        c.bind(lms, store, npg.cuda(), ctx_len.cuda())
        c.prime(q_init)
        outs = torch.zeros_like(q)
        for t in range(S):
            for l in range(L):
                c.decode_layer_step(t, l, q[t, l], outs[t, l])
        c.sync()
        assert c.device_error() == (0, 0)
        seen.append((outs, [x.clone() for x in lms], c.get_indices(S & 1, 0)))
        if correct:
            assert c.miss_stats()[0] > 0                                # the repair ran too
        c.close()
    assert torch.equal(seen[0][0].view(torch.int16), seen[1][0].view(torch.int16))
    assert all(torch.equal(a, b) for a, b in zip(seen[0][1], seen[1][1])) and torch.equal(seen[0][2], seen[1][2])


def test_new_tokens_enter_the_store_and_are_gathered(dd):
    """A decode step's keys and values go into the page-locked store through the cache view of the layer; a gather behind it
    on the same stream brings them back."""
    B, P, k = 2, 12, 12
    g = torch.Generator().manual_seed(5)
    raw, _ = quantised(torch.randn(B, HKV, P, 2, T, D, generator=g).to(torch.bfloat16))
    store = raw.contiguous().pin_memory()
    cache = dd.PagedCache.of_store(store, cache_format=dd.DD_CACHE_E4M3)
    c = dd.Context(n_layers=1, batch=B, max_pages=P, k_pages=k, store_format=dd.DD_CACHE_E4M3)
    every = torch.arange(P, dtype=torch.int32).expand(B, HKV, P).contiguous().cuda()
    k_new, v_new = (torch.randn(B, HKV, D, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    pos = torch.tensor([100, P * T - 1], dtype=torch.int32).cuda()
    cache.append(k_new, v_new, pos)
    c.gather_kv_from_host(store, every, None, 0)
    slot = c.slot_tensor(0)
    want = ref.decode_pages(raw.numpy(), "e4m3", T, D)
    for b in range(B):
        p = int(pos[b])
        for h in range(HKV):
            for kv, row in ((0, k_new[b, h]), (1, v_new[b, h])):
                code, ex = ref.quantise(ref.f64(row))
                want[b, h, p // T, kv, p % T] = ref.CODES[code] * 2.0 ** (int(ex) - 127)
    want = torch.from_numpy(np.moveaxis(want, 3, 2).copy()).to(torch.bfloat16).reshape(slot.shape)
    assert torch.equal(slot.cpu(), want)
    assert c.device_error() == (0, 0) and cache.device_error() == (0, 0)
    c.close()


def test_store_builder_quantises_on_the_device(dd):
    from paper_2607_26475_b200 import store as st
    w = wl.small(wl.CONFIGS[2], n_layers=2, batch=2, ctx=500, budget=64, steps=1)
    c = dd.Context(n_layers=2, batch=2, max_pages=w.n_pages, k_pages=w.k_pages, store_format=dd.DD_CACHE_E4M3)
    s = st.HostStore(w, c)
    assert s.host_bytes == 2 * 2 * HKV * w.n_pages * PAGE
    raw, values = quantised(torch.stack([wl.kv_slab(w, 1, b, device="cuda").cpu() for b in range(2)]))
    assert torch.equal(s.kv[1], raw)
    want = orc.build_landmarks(f32(values[:, :, :, 0]), s.ctx_len.numpy())
    assert np.array_equal(f32(s.landmarks[1]), want)
    c.close()
