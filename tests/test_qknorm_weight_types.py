"""Weights whose type changes between calls: a module's .bfloat16() and .float() change its parameters in place."""
import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api
from tests.test_abi_argtypes import binding, stub  # noqa: F401  (fixtures)

B, L, Hq, Hkv, d = 2, 5, 4, 2, 64
EPS = 1e-5


class Norms(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.q, self.k = (torch.nn.Parameter(1 + torch.arange(d) / 64.0 * s, requires_grad=False) for s in (1, -1))


def _calls(desc, norm, device):
    bf = torch.bfloat16
    q, k = torch.ones((B, Hq, L, d), dtype=bf, device=device), torch.ones((B, Hkv, L, d), dtype=bf, device=device)
    dw = torch.zeros(d, device=device)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device=device)
    return (lambda: api.sepllm_qknorm_rope_fwd(desc, norm, None, q, k, k, q, k, k),
            lambda: api.sepllm_qknorm_rope_bwd(desc, norm, None, q, k, q, k, k, q, k, k, dw, dw, ws))


def test_every_call_takes_the_type_of_now(binding):  # noqa: F811
    m, desc = Norms(), api.RopeDesc(B, L, Hq, Hkv, d)
    norm = api.QkNorm(m.q, m.k, eps=EPS)
    for call in _calls(desc, norm, "cpu"):
        for change, w_dtype in ((m.bfloat16, 0), (m.float, 1), (m.bfloat16, 0)):
            change()
            call()
            assert norm.w_dtype == w_dtype and (norm.wq, norm.wk) == (m.q.data_ptr(), m.k.data_ptr())


def test_types_that_became_unusable_are_refused(binding):  # noqa: F811
    m, desc = Norms(), api.RopeDesc(B, L, Hq, Hkv, d)
    for call in _calls(desc, api.QkNorm(m.q, m.k, eps=EPS), "cpu"):
        for change in (m.half, m.double):
            change()
            with pytest.raises(ValueError):
                call()
        m.float()
        m.k.data = m.k.data.bfloat16()             # two types
        with pytest.raises(ValueError):
            call()
        m.float()
        call()
    only_k = api.QkNorm(None, m.k, eps=EPS)
    m.bfloat16()
    _calls(desc, only_k, "cpu")[0]()
    assert only_k.w_dtype == 0 and only_k.wq is None


@pytest.mark.gpu
def test_results_after_a_change_of_type():
    """Half a step of bf16 and the kernel's 4e-6 (sums of 64 squares, a root, products) of the pairs' sizes."""
    m, desc = Norms().cuda(), api.RopeDesc(B, L, Hq, Hkv, d)
    norm = api.QkNorm(m.q, m.k, eps=EPS)
    freq, _ = api.sepllm_rope_frequencies(desc)
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k = (torch.randn((B, h, L, d), generator=g, device="cuda").to(torch.bfloat16) for h in (Hq, Hkv))
    for change in (m.float, m.bfloat16, m.float):
        change()
        y = [torch.empty_like(t) for t in (q, k)]
        api.sepllm_qknorm_rope_fwd(desc, norm, None, q, k, None, *y, None)
        torch.cuda.synchronize()
        for x, out, w in ((q, y[0], m.q), (k, y[1], m.k)):
            n = orc.head_norm(x.double().cpu().numpy(), w.detach().double().cpu().numpy(), EPS)
            ref = orc.rope_apply(n, np.arange(L), freq)
            pair = np.abs(n[..., :d // 2]) + np.abs(n[..., d // 2:])
            tol = 2.0 ** -8 * np.abs(ref) + 4e-6 * np.concatenate((pair, pair), -1)
            assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
