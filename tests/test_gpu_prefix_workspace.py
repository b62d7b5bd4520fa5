"""One workspace, sized for the longest prefix, serves shorter ones in every form that the calls take."""
import pytest
import torch

from paper_2412_12094_b200 import api, inputs
from tests.test_gpu_attn_prefix import _index, _run
from tests.test_gpu_prefix import BF, Cache, _decode, _normal

pytestmark = pytest.mark.gpu
GUARD = 1 << 16


def _guarded(n):
    """n bytes and behind them a strip that nothing may touch."""
    ws = api.alloc_bytes(n + GUARD)
    ws.fill_(0xa5)
    return ws, ws[n:]


@pytest.mark.parametrize("B,d,longest,shorter", [(4, 128, 4737, (4736, 4700, 2000, 1)), (1, 128, 37900, (37550, 30000, 500)),
                                                 (2, 128, 10700, (9600, 9400, 9000, 300)), (40, 64, 3000, (2999, 900, 128, 5))])
def test_decode(B, d, longest, shorter):
    g = torch.Generator(device="cuda").manual_seed(longest)
    Hkv, Hq = 8, 32
    cache = Cache(g, B, Hkv, Hq, d, 4, 4, 8, 300, [(37 * b) % 300 for b in range(B)])
    q, K, V = _normal(g, B, Hq, d), _normal(g, Hkv, longest, d), _normal(g, Hkv, longest, d)
    ws, strip = _guarded(api.sepllm_decode_prefix_workspace_bytes(cache.desc, longest))
    for P in (longest, *shorter):
        Kp, Vp = K[:, :P].contiguous(), V[:, :P].contiguous()
        want = _decode(cache, P, q, Kp, Vp, None)
        o, lse = torch.empty((B, Hq, d), dtype=BF, device="cuda"), torch.empty((B, Hq), device="cuda")
        api.sepllm_decode_prefix(cache.desc, P, 0.0, q, cache.state, cache.Kc, cache.Vc, Kp, Vp, None, o, lse, ws)
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1]) and (strip == 0xa5).all(), P


@pytest.mark.parametrize("B,L,d,longest,shorter", [(2, 300, 128, 9000, (5000, 2000, 500, 1)), (8, 100, 128, 8192, (1000, 129, 7)),
                                                   (4, 200, 80, 3000, (2000, 900, 100))])
def test_attention(B, L, d, longest, shorter):
    g = torch.Generator(device="cuda").manual_seed(longest)
    Hkv, Hq = 2, 8
    idesc, index = _index(inputs.token_ids(5, B, L, 0.1), 30)
    Q, K, V = _normal(g, B, Hq, L, d), _normal(g, B, Hkv, L, d), _normal(g, B, Hkv, L, d)
    Kl, Vl = _normal(g, Hkv, longest, d), _normal(g, Hkv, longest, d)
    desc = api.AttnDesc(B, Hq, Hkv, d, L, 0.0, 0)
    ws, strip = _guarded(api.sepllm_attn_prefix_workspace_bytes(desc, idesc, longest))
    for P in (longest, *shorter):
        Kp, Vp = Kl[:, :P].contiguous(), Vl[:, :P].contiguous()
        want = _run(Q, K, V, idesc, index, Kp, Vp, None)
        O, LSE = torch.empty_like(Q), torch.empty((B, Hq, L), device="cuda")
        api.sepllm_attn_prefix_fwd(desc, idesc, P, Q, K, V, index, Kp, Vp, None, O, LSE, ws)
        torch.cuda.synchronize()
        assert torch.equal(O, want[0]) and torch.equal(LSE, want[1]) and (strip == 0xa5).all(), P
