"""A workspace sized for a prefix of P rows serves every shorter one (no GPU: the size queries)."""
import ctypes as C

import numpy as np
import pytest

from paper_2412_12094_b200 import api, build


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()


LENGTHS = sorted({1, 2, 127, 128, 129, 4736, 4737, 37550, 37900, 1 << 20, 50_000_000, 1 << 27, 1 << 30,
                  *(int(p) for p in np.geomspace(1, 200_000, 400)), *range(8500, 11500, 37)})


@pytest.mark.parametrize("B,Hkv,Hq,d,c,flags", [(4, 8, 32, 128, 300, 0), (1, 8, 32, 128, 200, 0), (2, 8, 32, 128, 200, 0),
                                                (256, 8, 32, 128, 760, 0), (5, 12, 12, 64, 300, 0), (1, 1, 1, 64, 20, 0),
                                                (3000, 1, 16, 64, 40, 0), (32, 8, 32, 128, 3332, 0), (7, 400, 400, 64, 20, 0),
                                                (4, 8, 32, 128, 300, 1)])
def test_decode(B, Hkv, Hq, d, c, flags):
    desc = api.CacheDesc(B, Hkv, Hq, d, 4, 4, 8, c, flags)
    if flags:
        desc = api.CacheDesc(B, Hkv, Hq, d, 4, c - 13, 8, c, flags)
    lengths = [P for P in LENGTHS if P * Hkv <= 1 << 36]     # (longer ones are refused)
    n = [api.sepllm_decode_prefix_workspace_bytes(desc, P) for P in lengths]
    assert all(a <= b for a, b in zip(n, n[1:])), [(P, a, b) for P, a, b in zip(lengths, n, n[1:]) if a > b][:5]


@pytest.mark.parametrize("B,Hq,Hkv,d,L,w", [(8, 32, 8, 128, 100, 64), (2, 32, 8, 128, 1024, 256), (1, 32, 8, 128, 16, 16),
                                            (16, 32, 8, 128, 64, 64), (1, 32, 8, 128, 8192, 256), (8, 12, 12, 64, 1024, 64),
                                            (300, 2, 1, 64, 130, 20), (3, 130, 2, 80, 128, 30), (1, 400, 400, 64, 2, 3)])
def test_attention(B, Hq, Hkv, d, L, w):
    desc, idesc = api.AttnDesc(B, Hq, Hkv, d, L, 0.0, 0), api.IndexDesc(B, L, 0, w, 1, 128, 128, L)
    P = [p for p in LENGTHS if p <= 1 << 20]
    n = [api.sepllm_attn_prefix_workspace_bytes(desc, idesc, p) for p in P]
    assert all(a <= b for a, b in zip(n, n[1:])), [(p, a, b) for p, a, b in zip(P, n, n[1:]) if a > b][:5]


@pytest.mark.parametrize("B,Hq,L,fits", [(64, 64, 1 << 19, False), (64, 64, (1 << 19) - 1, True), (3000, 64, 1 << 15, False),
                                         # 65 536 query tiles, one more than the attention calls take
                                         (2, 32, 1 << 23, False), (2, 32, (1 << 23) - 128, True)])
def test_batches_of_too_many_rows_are_refused_before_anything_is_launched(B, Hq, L, fits):
    """2^31 query rows and more, or too many tiles: by the size query and by the call (whose addresses are not used)."""
    desc, idesc = api.AttnDesc(B, Hq, 8, 64, L, 0.0, 0), api.IndexDesc(B, L, 0, 8, 1, 128, 128, L)
    n = C.c_size_t(0)
    got = api.lib().sepllm_attn_prefix_workspace_bytes(C.byref(desc), C.byref(idesc), C.c_int32(60000), C.byref(n))
    assert got == (api.OK if fits else api.UNSUPPORTED)
    if not fits:
        a = 1 << 20
        assert api.lib().sepllm_attn_prefix_fwd(C.byref(desc), C.byref(idesc), 60000, a, a, a, a, a, a, None, a, a, a,
                                                None) == api.UNSUPPORTED
