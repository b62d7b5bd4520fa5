"""Shared-prefix decode where a CTA of the prefix kernel walks many short segments one after the other:
pairs of row tiles that see a key tile or two of a long block."""
import numpy as np
import pytest
import torch

from tests.test_gpu_prefix import BF, Cache, _check_decode, _decode, _normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,far", [(64, 1), (64, 128), (128, 128), (64, 300), (128, 300)])
def test_runs_of_one_or_few_shared_key_tiles(d, far):
    """512 pairs of row tiles, more than three to a CTA, each with ceil(far / 128) key tiles: the two
    slots pass their turn at the exponentials on from segment to segment.  The result is the oracle's
    and the same at every call."""
    g = torch.Generator(device="cuda").manual_seed(d + far)
    rng = np.random.default_rng(far)
    B, Hkv, Hq, P = 2040, 4, 64, 4096
    runs, plen = rng.integers(0, 16, B), rng.integers(0, far + 1, B)
    plen[::3] = far
    cache = Cache(g, B, Hkv, Hq, d, 1, 4, 3, 16, runs.tolist())
    q = (torch.randn((B, Hq, d), generator=g, device="cuda") * 2).to(BF)
    Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    pl = torch.from_numpy(plen.astype(np.int32)).cuda()
    o, lse = _decode(cache, P, q, Kp, Vp, pl)
    some = [(int(b), int(h)) for b, h in zip(rng.integers(0, B, 300), rng.integers(0, Hq, 300))]
    _check_decode(cache, q, Kp, Vp, plen, o, lse, rows=some)
    for _ in range(5):
        o2, lse2 = _decode(cache, P, q, Kp, Vp, pl)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("far", [100, 200, 300])
def test_rows_behind_the_prefix_in_runs_of_uneven_pairs(d, far):
    """Pairs of row tiles in which the first, the second or both see the end of the block, in any order
    over a CTA's run; behind it stand values that are not finite, and nothing may depend on them."""
    g = torch.Generator(device="cuda").manual_seed(d * far)
    rng = np.random.default_rng(far)
    B, Hkv, Hq, P = 2040, 4, 64, 4096     # a row tile: 8 sequences
    runs = rng.integers(0, 16, B)
    tile = np.repeat(rng.choice([0, 60, far - 70, far, far], B // 8), 8)
    plen = np.minimum(tile, rng.integers(0, far + 1, B))
    plen[::8] = tile[::8]                 # the tile's longest
    cache = Cache(g, B, Hkv, Hq, d, 1, 4, 3, 16, runs.tolist())
    q = (torch.randn((B, Hq, d), generator=g, device="cuda") * 2).to(BF)
    Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    pl = torch.from_numpy(plen.astype(np.int32)).cuda()
    o, lse = _decode(cache, P, q, Kp, Vp, pl)
    some = [(int(b), int(h)) for b, h in zip(rng.integers(0, B, 300), rng.integers(0, Hq, 300))]
    _check_decode(cache, q, Kp, Vp, plen, o, lse, rows=some)
    Kp[:, far:], Vp[:, far:] = float("nan"), float("inf")
    for _ in range(5):
        o2, lse2 = _decode(cache, P, q, Kp, Vp, pl)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
