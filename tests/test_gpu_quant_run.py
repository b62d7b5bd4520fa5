"""The operators as a program uses them together: a fused projection is normalised and rotated, the prompt is
pre-filled, its entries are kept in 4 bits, and tokens are generated from that cache."""
import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, inputs
from tests._gpu_util import TOL_O, assert_close, attn_fwd, build_index, flags_of
from tests.test_gpu_qknorm import check_fwd
from tests.test_gpu_quant_cache import QuantCache, check_cache
from tests.test_gpu_quant_decode import check_decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,Hq,Hkv,layout,flags", [(64, 4, 4, "half", 0), (128, 8, 2, "interleaved", 0),
                                                   (128, 8, 2, "half", api.CACHE_FIXED_WINDOW)])
def test_prompt_to_generated_tokens(d, Hq, Hkv, layout, flags):
    B, L, more, a, s, w, c, eps = 2, 230, 70, 3, 80, 24, 140, 1e-6
    ids = inputs.token_ids(500 + d, B, L + more, 0.15)
    f = flags_of(ids, inputs.SEP_IDS)
    idesc, index = build_index(np.ascontiguousarray(ids[:, :L]), inputs.SEP_IDS, a, w)
    g = torch.Generator(device="cuda").manual_seed(501 + d)
    wq, wk = (1 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in "qk")
    norm = api.QkNorm(wq, wk, eps=eps)
    qkv = torch.randn((B, L + more, Hq + 2 * Hkv, d), generator=g, device="cuda").to(torch.bfloat16)

    def project(first, n):
        """Q, K, V of tokens first .. first + n - 1, as the attention and cache calls take them."""
        desc = api.RopeDesc(B, n, Hq, Hkv, d, layout=layout, pos_first=first)
        x = qkv[:, first:first + n].transpose(1, 2).split((Hq, Hkv, Hkv), 1)
        out = [torch.empty((B, h, n, d), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv)]
        api.sepllm_qknorm_rope_fwd(desc, norm, None, *x, *out)
        freq, m = api.sepllm_rope_frequencies(desc)
        for i, wt in ((0, wq), (1, wk)):
            check_fwd(out[i], x[i], wt, eps, 0.0, first + np.arange(n), freq, layout, m)
        return out
    Q, K, V = project(0, L)
    O, _ = attn_fwd(Q, K, V, idesc, index)
    Oref, _ = orc.attn_fwd(*(t.double().cpu().numpy() for t in (Q, K, V)), f[:, :L], a, w)
    assert_close(O.float().cpu().numpy(), Oref, TOL_O, "O")
    qc = QuantCache(B, Hkv, Hq, d, a, s, w, c, flags)
    api.sepllm_cache_from_prompt_quant(qc.desc, idesc, index, None, K, V, qc.state, qc.Kc, qc.Vc)
    oc = []
    for b in range(B):
        o = orc.FundamentalCache(a, w) if flags else orc.StreamingCache(a, s, w, c)
        for t in range(L):
            o.update(bool(f[b, t]))
        oc.append(o)
    Ks, Vs = [K], [V]
    for t in range(L, L + more):
        q1, k1, v1 = project(t, 1)
        Ks.append(k1)
        Vs.append(v1)
        qc.update(torch.from_numpy(ids[:, t].copy()).cuda(), k1[:, :, 0].contiguous(), v1[:, :, 0].contiguous())
        for b in range(B):
            oc[b].update(bool(f[b, t]))
        if t % 9 == 0 or t == L + more - 1:
            check_decode(qc, q1[:, :, 0].contiguous())
    assert api.sepllm_last_device_status(qc.state) == 0
    check_cache(qc, oc, f, torch.cat(Ks, 2).cpu(), torch.cat(Vs, 2).cpu())
    # the generated cache becomes a prefix that a batch shares (entries of one sequence, in 16 bits)
    K1, V1, n = qc.entries()
    kept = oc[1].retained()
    assert n[1] == len(kept)
    P, cd = c, api.CacheDesc(3, Hkv, Hq, d, 0, 4, 3, 16)
    state = api.alloc_bytes(api.sepllm_cache_bytes(cd)[0])
    api.sepllm_cache_init(cd, state)
    Kc = torch.zeros((3, Hkv, 20, d), dtype=torch.bfloat16, device="cuda")
    K1[1, :, len(kept):] = 0
    V1[1, :, len(kept):] = 0
    q = torch.randn((3, Hq, d), generator=g, device="cuda").to(torch.bfloat16)
    o = torch.empty_like(q)
    plen = torch.full((3,), len(kept), dtype=torch.int32, device="cuda")
    ws = api.alloc_bytes(api.sepllm_decode_prefix_workspace_bytes(cd, P))
    api.sepllm_decode_prefix(cd, P, 0.0, q, state, Kc, Kc, K1[1].contiguous(), V1[1].contiguous(), plen, o, None, ws)
    torch.cuda.synchronize()
    G = Hq // Hkv
    for h in range(Hq):
        oref, _ = orc.decode_attention(q[2, h].double().cpu().numpy(), K1[1, h // G, : len(kept)].double().cpu().numpy(),
                                       V1[1, h // G, : len(kept)].double().cpu().numpy())
        assert_close(o[2, h].float().cpu().numpy(), oref, TOL_O, f"prefix h={h}")
