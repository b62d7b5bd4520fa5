"""sepllm_decode_quant over long caches that one CTA walks alone: the sums over the entries keep their 32 bits."""
import pytest
import torch

from paper_2412_12094_b200 import api

pytestmark = pytest.mark.gpu

CTAS = 3 * 148    # of the largest grid: as many units are not cut


def long_caches(B, Hkv, Hq, d, n, seed, lowest):
    """Caches of n entries, all units alike: keys of zeros (all weights are equal, and exact), codes of V from
    `lowest` to 7, steps that are powers of two between 2^-10 and 1 (a weight times a step
    is exact in 16 bits).  Returns the calls' buffers and the held values of V [n][d], 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    desc = api.CacheDesc(B, Hkv, Hq, d, 0, 4, 8, n + 20)
    slots, units = desc.c + desc.s, B * Hkv
    sb, kb = api.sepllm_cache_bytes_quant(desc)
    state, Kc, Vc = (api.alloc_bytes(x) for x in (sb, kb, kb))
    api.sepllm_cache_init(desc, state)
    head = api.CacheHeader.from_buffer_copy(bytes(state[:256].tolist()))
    state[head.off_seq:head.off_seq + 64 * B].view(torch.int32).view(B, 16)[:, 4] = n      # neighbours alone
    code = torch.randint(lowest, 8, (slots, d), generator=g, device="cuda")
    step = -torch.exp2(torch.randint(-10, 1, (slots, d // 32), generator=g, device="cuda").double())
    e = torch.arange(d, device="cuda")
    place = ((e % 32 // 4) * (d // 32) + e // 32) * 4 + e % 4
    held = torch.empty((slots, d), dtype=torch.uint8, device="cuda")
    held[:, place] = (code + 8).to(torch.uint8)
    rows = units * slots
    at = (rows * d // 2 + 255) // 256 * 256
    Kc.zero_()                                                                             # (steps of 0)
    Vc[:rows * d // 2].view(units, -1).copy_((held[:, 0::2] | held[:, 1::2] << 4).flatten())
    Vc[at:at + rows * d // 16].view(units, -1).copy_(step.to(torch.bfloat16).view(torch.uint8).flatten())
    values = (code.double() * step.repeat_interleave(32, 1))[desc.s:desc.s + n]
    return desc, state, Kc, Vc, values


@pytest.mark.parametrize("d,G", [(128, 1), (128, 8), (128, 16), (64, 4), (64, 6), (64, 12)])
@pytest.mark.parametrize("lowest", [-7, 1])       # values of both signs, which cancel, and of one
def test_sums_over_100_000_entries(d, G, lowest):
    """The output is rounded once (2^-8).  Products are exact.  A warp adds up the tiles of 32 entries w, w + 4, ..,
    sixteen products at a time; these and what they are added to may be cut off, each of the seventeen at one unit
    in the last of 24 bits of the largest, which is no more than the largest sum on the way plus sixteen products
    of 7: 17 * 2^-23 of that, n / 64 times for each of four warps, and 2^-22 of it for the merge; over n."""
    n, B, Hkv = 100_000, CTAS // 4, 4
    desc, state, Kc, Vc, values = long_caches(B, Hkv, Hkv * G, d, n, 500 + d + G, lowest)
    q = torch.randn((B, Hkv * G, d), device="cuda").to(torch.bfloat16)
    o, lse = torch.empty_like(q), torch.empty((B, Hkv * G), device="cuda")
    ws = api.alloc_bytes(api.sepllm_decode_quant_workspace_bytes(desc))
    api.sepllm_decode_quant(desc, 0.0, q, state, Kc, Vc, o, lse, ws)
    torch.cuda.synchronize()
    ref = values.mean(0)
    warp = torch.arange(n, device="cuda") // 32 % 4
    way = torch.stack([values[warp == w].cumsum(0).abs().amax(0) for w in range(4)]).amax(0)
    tol = 2.0 ** -8 * ref.abs() + (17 * n / 16 * 2.0 ** -23 + 2.0 ** -22) * (way + 16 * 7) / n
    worst = float(((o.double() - ref).abs() / tol).max())
    assert worst <= 1, worst
    assert ((lse.double() - torch.log(torch.tensor(float(n), dtype=torch.float64))).abs() <= 1e-5).all()
