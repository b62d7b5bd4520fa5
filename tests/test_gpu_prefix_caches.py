"""Caches of every mode on either side of a shared prefix: positions taken inside the cache that the
prefix comes from, and the fixed window."""
import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, inputs
from tests._gpu_util import TOL_LSE, TOL_O, assert_close
from tests.test_gpu_cache import GpuCache
from tests.test_gpu_decode_rope import TOL_LSE_ROPE, TOL_O_ROPE
from tests.test_gpu_prefix import BF, _normal

pytestmark = pytest.mark.gpu


def _stream(seed, B, steps, Hkv, Hq, d):
    ids = inputs.decode_stream_ids(seed, B, steps, 0.3)
    k, v, q = (x.cuda() for x in inputs.decode_kv_pool(seed, steps, B, Hkv, Hq, d))
    return ids, torch.from_numpy(np.ascontiguousarray(ids.T)).cuda(), k, v, q


def _prefix(cache, Kc, P):
    d = cache.desc
    Kp, Vp = (torch.full((d.Hkv, P, d.d), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    plen = torch.zeros(3, dtype=torch.int32, device="cuda")
    api.sepllm_prefix_from_cache(d, cache.state, Kc, cache.Vc, P, Kp, Vp, plen)
    torch.cuda.synchronize()
    return Kp, Vp, plen


@pytest.mark.parametrize("d,Hq,Hkv,steps", [(64, 2, 2, 30), (128, 8, 2, 90)])
def test_own_tokens_continue_the_positions_of_a_rotated_cache(d, Hq, Hkv, steps):
    """Kr becomes the prefix, entries at positions 0 .. R-1; the caller turns its own tokens to R, R + 1,
    ... (compactions before: 90 tokens in a cache of 40)."""
    a, s, w, c, base, B, n = 2, 8, 6, 40, 10000.0, 3, 20
    one = GpuCache(1, Hkv, Hq, d, a, s, w, c)
    table = api.alloc_bytes(api.sepllm_rope_table_bytes(one.desc))
    api.sepllm_rope_table_build(one.desc, base, table)
    Kr = torch.zeros_like(one.Kc)
    ids, ids_d, k, v, _ = _stream(d, 1, steps, Hkv, Hq, d)
    for t in range(steps):
        api.sepllm_cache_update_rope(one.desc, one.state, one.Kc, one.Vc, Kr, table, ids_d[t], inputs.SEP_IDS, k[t], v[t])
    Kp, Vp, plen = _prefix(one, Kr, c)
    slots = one.slot_of_virtual(api.read_cache_state(one.state), 0)
    R = len(slots)
    assert plen.tolist() == [R] * 3 and torch.equal(Kp[:, :R], Kr.view(Hkv, one.slots, d)[:, slots])
    kept_k, kept_v = (x.view(Hkv, one.slots, d)[:, slots].double().cpu().numpy() for x in (one.Kc, one.Vc))
    # own tokens, all of which their caches keep
    own = GpuCache(B, Hkv, Hq, d, 0, 8, 6, 40)
    ids, ids_d, k, v, q = _stream(d + 1, B, n, Hkv, Hq, d)
    ws = api.alloc_bytes(api.sepllm_decode_prefix_workspace_bytes(own.desc, c))
    o, lse = torch.empty((B, Hq, d), dtype=BF, device="cuda"), torch.empty((B, Hq), device="cuda")
    for t in range(n):
        desc = api.RopeDesc(B, 1, Hq, Hkv, d, base=base, pos_first=R + t)
        qt, kt, vt = (x[t][:, :, None] for x in (q, k, v))
        qr, kr, vr = (torch.empty_like(x) for x in (qt, kt, vt))
        api.sepllm_rope_fwd(desc, None, qt, kt, vt, qr, kr, vr)
        own.update(ids_d[t], kr[:, :, 0].contiguous(), vr[:, :, 0].contiguous())
        api.sepllm_decode_prefix(own.desc, c, 0.0, qr[:, :, 0].contiguous(), own.state, own.Kc, own.Vc, Kp, Vp, plen, o,
                                 lse, ws)
        torch.cuda.synchronize()
        for b in range(B):
            for h in range(Hq):
                hk = h // (Hq // Hkv)
                kk, vv = (np.concatenate((x[hk], y[:t + 1, b, hk].double().cpu().numpy()))
                          for x, y in ((kept_k, k), (kept_v, v)))
                ref, lref = orc.decode_attention_rope(q[t, b, h].double().cpu().numpy(), kk, vv, base)
                assert_close(o[b, h].float().cpu().numpy(), ref, TOL_O_ROPE, f"t={t} b={b} h={h}")
                assert abs(float(lse[b, h]) - lref) <= TOL_LSE_ROPE


@pytest.mark.parametrize("P", [300, 30000])
@pytest.mark.parametrize("d,Hq,Hkv,a,n", [(64, 2, 2, 0, 5), (128, 8, 2, 4, 16)])
def test_fixed_window_caches_behind_a_prefix(d, Hq, Hkv, a, n, P):
    """Generation that keeps every separator, behind a prefix read with each sequence and once for all."""
    g = torch.Generator(device="cuda").manual_seed(P)
    B, steps, cap = 2, 90, 60
    ids, ids_d, k, v, q = _stream(d + n, B, steps, Hkv, Hq, d)
    f = np.isin(ids, inputs.SEP_IDS)
    own = GpuCache(B, Hkv, Hq, d, a, cap, n, a + cap + n + 3, api.CACHE_FIXED_WINDOW)
    oc = [orc.FundamentalCache(a, n) for _ in range(B)]
    Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    plen = torch.tensor([P, P // 3], dtype=torch.int32, device="cuda")
    ws = api.alloc_bytes(api.sepllm_decode_prefix_workspace_bytes(own.desc, P))
    o, lse = torch.empty((B, Hq, d), dtype=BF, device="cuda"), torch.empty((B, Hq), device="cuda")
    for t in range(steps):
        own.update(ids_d[t], k[t], v[t])
        for b in range(B):
            oc[b].update(bool(f[b, t]))
        if t % 11 and t != steps - 1:
            continue
        api.sepllm_decode_prefix(own.desc, P, 0.0, q[t], own.state, own.Kc, own.Vc, Kp, Vp, plen, o, lse, ws)
        torch.cuda.synchronize()
        assert api.sepllm_last_device_status(ws) == 0 and api.sepllm_last_device_status(own.state) == 0
        for b in range(B):
            kept = oc[b].retained()
            for h in range(Hq):
                hk, m = h // (Hq // Hkv), int(plen[b])
                kk, vv = (torch.cat((x[hk, :m], y[kept, b, hk])).double().cpu().numpy() for x, y in ((Kp, k), (Vp, v)))
                ref, lref = orc.decode_attention(q[t, b, h].double().cpu().numpy(), kk, vv)
                assert np.abs(o[b, h].double().cpu().numpy() - ref).max() <= TOL_O["max_abs"], (t, b, h)
                assert abs(float(lse[b, h]) - lref) <= TOL_LSE, (t, b, h)


def test_prefix_of_a_fixed_window_cache():
    """Its rows are the oracle's retained set in order, bit for bit."""
    a, n, cap, steps, Hkv, d = 4, 16, 60, 120, 2, 64
    ids, ids_d, k, v, _ = _stream(9, 1, steps, Hkv, Hkv, d)
    f = np.isin(ids[0], inputs.SEP_IDS)
    one = GpuCache(1, Hkv, Hkv, d, a, cap, n, a + cap + n + 3, api.CACHE_FIXED_WINDOW)
    oc = orc.FundamentalCache(a, n)
    for t in range(steps):
        one.update(ids_d[t], k[t], v[t])
        oc.update(bool(f[t]))
    kept, P = oc.retained(), one.desc.c + 5
    Kp, Vp, plen = _prefix(one, one.Kc, P)
    assert plen.tolist() == [len(kept)] * 3 and len(oc.sep) <= cap
    for x, y in ((Kp, k), (Vp, v)):
        assert torch.equal(x[:, :len(kept)], y[kept, 0].transpose(0, 1)) and torch.isnan(x[:, len(kept):].float()).all()
