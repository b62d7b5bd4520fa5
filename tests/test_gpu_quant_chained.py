"""4-bit cache calls right behind the kernels that write what they read, with nothing between: each call's kernel
starts while the one before it ends, and reads only behind its end."""
import pytest
import torch

from paper_2412_12094_b200 import api, inputs
from tests._gpu_util import build_index
from tests.test_gpu_quant_cache import QuantCache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,c", [(64, 300), (128, 3000)])
@pytest.mark.parametrize("captured", [False, True])
def test_results_do_not_depend_on_what_ran_just_before(d, c, captured):
    """A generation step, norm and rotation -> update -> decode -> read-back, and a hand-off behind a norm: the bits are
    those of the same calls with the GPU waited for in between."""
    B, Hq, Hkv, L, a = 4, 8, 2, 250, 2
    g = torch.Generator(device="cuda").manual_seed(700 + d)
    norm = api.QkNorm(*(1 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in "qk"))
    ids = inputs.token_ids(700 + d, B, L, 0.2)
    idesc, index = build_index(ids, inputs.SEP_IDS, a, 16)
    bf = torch.bfloat16

    class Run:
        def __init__(self):
            self.qc = QuantCache(B, Hkv, Hq, d, a, 20, 32, c)
            self.x = torch.zeros((B, L, Hq + 2 * Hkv, d), dtype=bf, device="cuda")
            self.x1 = torch.zeros((B, 1, Hq + 2 * Hkv, d), dtype=bf, device="cuda")
            self.out = [torch.zeros((B, h, L, d), dtype=bf, device="cuda") for h in (Hq, Hkv, Hkv)]
            self.one = [torch.zeros((B, h, 1, d), dtype=bf, device="cuda") for h in (Hq, Hkv, Hkv)]
            self.tok = torch.full((B,), 60, dtype=torch.int32, device="cuda")
            self.o = torch.zeros((B, Hq, d), dtype=bf, device="cuda")
            self.lse = torch.zeros((B, Hq), device="cuda")
            self.K, self.V = (torch.zeros((B, Hkv, c, d), dtype=bf, device="cuda") for _ in "kv")
            self.n = torch.zeros(B, dtype=torch.int32, device="cuda")

        def steps(self):
            qc, split = self.qc, lambda x: x.transpose(1, 2).split((Hq, Hkv, Hkv), 1)
            return [
                lambda: api.sepllm_qknorm_rope_fwd(api.RopeDesc(B, L, Hq, Hkv, d), norm, None, *split(self.x), *self.out),
                lambda: api.sepllm_cache_from_prompt_quant(qc.desc, idesc, index, None, self.out[1], self.out[2], qc.state,
                                                           qc.Kc, qc.Vc),
                lambda: api.sepllm_qknorm_rope_fwd(api.RopeDesc(B, 1, Hq, Hkv, d, pos_first=L), norm, None,
                                                   *split(self.x1), *self.one),
                lambda: qc.update(self.tok, self.one[1][:, :, 0], self.one[2][:, :, 0]),
                lambda: api.sepllm_decode_quant(qc.desc, 0.0, self.one[0][:, :, 0], qc.state, qc.Kc, qc.Vc, self.o, self.lse,
                                                qc.ws),
                lambda: api.sepllm_cache_entries_quant(qc.desc, qc.state, qc.Kc, qc.Vc, c, self.K, self.V, self.n)]

    near, apart = Run(), Run()
    for f in near.steps():      # (kernels loaded before a capture)
        f()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    if captured:
        with torch.cuda.graph(graph):
            for f in near.steps():
                f()
    for t in range(20):
        x, x1 = (torch.randn(y.shape, generator=g, device="cuda").to(bf) for y in (near.x, near.x1))
        for r in (near, apart):
            r.x.copy_(x)
            r.x1.copy_(x1)
        torch.cuda.synchronize()
        if captured:
            graph.replay()
        else:
            for f in near.steps():
                f()
        torch.cuda.synchronize()
        for f in apart.steps():
            f()
            torch.cuda.synchronize()
        for p, q in zip((near.o, near.lse, near.K, near.V, near.n), (apart.o, apart.lse, apart.K, apart.V, apart.n)):
            assert torch.equal(p, q), t
        assert (near.n > 0).all() and torch.isfinite(near.o.float()).all()
