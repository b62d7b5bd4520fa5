"""The largest query elements that sepllm_decode_quant takes."""
import pytest
import torch

from paper_2412_12094_b200 import api, inputs
from tests._gpu_util import build_index
from tests.test_gpu_quant_cache import QuantCache
from tests.test_gpu_quant_decode import check_decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,Hq", [(64, 4), (128, 6), (128, 12)])
def test_either_side_of_the_limit(d, Hq):
    """Keys near 2^-99 and a scale of 2^-20 make scores of a few; the element below 1.75 * 2^118 gives the reference's
    result, the next one a row of NaN, and the other heads are not touched by it."""
    n, g = 150, torch.Generator(device="cuda").manual_seed(800 + d)
    ids = inputs.token_ids(800, 1, n, 0.1)
    idesc, index = build_index(ids, inputs.SEP_IDS, 0, 16)
    K = torch.zeros((1, 1, n, d), dtype=torch.bfloat16, device="cuda")
    K[..., 3] = (torch.rand((1, 1, n), generator=g, device="cuda") + 0.5) * 2.0 ** -99
    V = torch.randn((1, 1, n, d), generator=g, device="cuda").to(torch.bfloat16)
    qc = QuantCache(1, 1, Hq, d, 0, 20, 64, n + 50)
    api.sepllm_cache_from_prompt_quant(qc.desc, idesc, index, None, K, V, qc.state, qc.Kc, qc.Vc)
    limit = torch.tensor(1.75 * 2.0 ** 118, dtype=torch.bfloat16)
    below = (limit.view(torch.int16) - 1).view(torch.bfloat16)
    assert float(below) < float(limit) == 1.75 * 2.0 ** 118
    q = torch.zeros((1, Hq, d), dtype=torch.bfloat16, device="cuda")
    for h in range(Hq):
        q[0, h, 3] = float(below) * (1.0, -1.0, 2.0 ** -1, 2.0 ** -3)[h % 4]
    o, lse, _ = check_decode(qc, q, 2.0 ** -20)
    q[0, 1, 3] = -float(limit)
    q[0, Hq - 1, 3] = float("inf")
    o2, lse2 = qc.decode(q, 2.0 ** -20)
    bad = torch.zeros(Hq, dtype=torch.bool, device="cuda")
    bad[[1, Hq - 1]] = True
    assert torch.isnan(o2[0, bad]).all() and torch.isnan(lse2[0, bad]).all()
    assert torch.equal(o2[0, ~bad], o[0, ~bad]) and torch.equal(lse2[0, ~bad], lse[0, ~bad])
