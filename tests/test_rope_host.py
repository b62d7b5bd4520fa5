"""Rotary positions, host side: the oracle's rotation against the definition, the frequencies the
library computes against the oracle's, and the calls the entry points refuse (no GPU)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, build


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_oracle_rotation_is_the_pairwise_definition(layout):
    g = np.random.default_rng(1)
    r, d, L = 6, 10, 4
    x, pos, m = g.normal(size=(2, L, d)), np.array([0, 3, -7, 1000]), 1.25
    f = orc.rope_frequencies(r, 100.0)
    y = orc.rope_apply(x, pos, f, layout, m)
    for b in range(2):
        for l in range(L):
            for i in range(r // 2):
                p, q = (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)
                a = pos[l] * 100.0 ** (-2 * i / r)
                assert abs(y[b, l, p] - m * (x[b, l, p] * math.cos(a) - x[b, l, q] * math.sin(a))) < 1e-12
                assert abs(y[b, l, q] - m * (x[b, l, q] * math.cos(a) + x[b, l, p] * math.sin(a))) < 1e-12
            assert (y[b, l, r:] == x[b, l, r:]).all()
    # the gradient's map is the transposed one: <y', R x> = <R^T y', x>, and against differences
    dy = g.normal(size=x.shape)
    dx = orc.rope_apply(dy, pos, f, layout, 1.0, inverse=True)
    dx[..., :r] *= m
    full = lambda z: float((dy * orc.rope_apply(z, pos, f, layout, m)).sum())  # noqa: E731
    assert abs((dx * x).sum() - full(x)) < 1e-9
    for idx in [(0, 1, 0), (1, 2, 3), (0, 3, 5), (1, 0, 9)]:
        e = np.zeros_like(x)
        e[idx] = 1e-4
        assert abs((full(x + e) - full(x - e)) / 2e-4 - dx[idx]) < 1e-7


def test_oracle_rotation_agrees_with_the_rotation_inside_the_cache():
    x = np.random.default_rng(2).normal(size=(5, 64))
    pos = np.arange(5) * 37
    a = orc.rope_apply(x, pos, orc.rope_frequencies(64, 10000.0))
    assert np.allclose(a, orc.rope_rotate(x, pos, 10000.0), atol=1e-12)


SCALINGS = [("none", {}), ("linear", dict(factor=2.5)), ("ntk", dict(factor=4.0)),
            ("yarn", dict(factor=4.0, low=1.0, high=32.0, orig_len=4096.0)),
            ("yarn", dict(factor=16.0, low=1.0, high=32.0, orig_len=32768.0)),
            ("llama3", dict(factor=8.0, low=1.0, high=4.0, orig_len=8192.0)),
            ("llama3", dict(factor=32.0, low=1.0, high=4.0, orig_len=100.0))]


@pytest.mark.parametrize("scaling,kw", SCALINGS)
@pytest.mark.parametrize("r,base", [(128, 500000.0), (64, 10000.0), (20, 10000.0), (4, 1e6)])
def test_frequencies_match_the_oracle(scaling, kw, r, base):
    desc = api.RopeDesc(1, 1, 1, 1, 128, rot_dim=r, scaling=scaling, base=base, **kw)
    f, m = api.sepllm_rope_frequencies(desc)
    ref = orc.rope_frequencies(r, base, scaling, **kw)
    assert f.shape == ref.shape and np.allclose(f, ref, rtol=1e-13, atol=0)
    assert m == pytest.approx(0.1 * math.log(kw["factor"]) + 1 if scaling == "yarn" else 1.0, rel=1e-15)


def test_frequencies_of_the_stretched_forms_have_the_ends_they_should():
    """Pairs that turn often keep their frequency, slow pairs are stretched by the whole factor."""
    kw = dict(factor=8.0, orig_len=8192.0)
    plain = orc.rope_frequencies(128, 500000.0)
    for scaling, low, high in (("llama3", 1.0, 4.0), ("yarn", 1.0, 32.0)):
        f, _ = api.sepllm_rope_frequencies(api.RopeDesc(1, 1, 1, 1, 128, scaling=scaling, base=500000.0, low=low,
                                                        high=high, **kw))
        assert np.allclose(f[0], 1.0) and np.allclose(f[-1], plain[-1] / 8.0) and (np.diff(f) < 0).all()
        assert ((f <= plain * (1 + 1e-12)) & (f >= plain / 8.0 * (1 - 1e-12))).all()
    # ntk: the slowest pair is stretched by the factor, the fastest is left alone
    f, _ = api.sepllm_rope_frequencies(api.RopeDesc(1, 1, 1, 1, 128, scaling="ntk", base=500000.0, factor=8.0))
    assert f[0] == 1.0 and np.isclose(f[-1], plain[-1] / 8.0)
    fac = np.linspace(1.0, 5.0, 64)
    f, m = api.sepllm_rope_frequencies(api.RopeDesc(1, 1, 1, 1, 128, scaling="factors", base=500000.0,
                                                    freq_factors=fac, attn_factor=1.19))
    assert np.allclose(f, plain / fac, rtol=1e-13) and m == 1.19


BAD_DESC = [dict(B=0), dict(L=0), dict(Hq=0), dict(Hkv=-1), dict(rot_dim=3), dict(rot_dim=130), dict(rot_dim=-2),
            dict(layout=2), dict(scaling=6), dict(scaling=-1), dict(base=1.0), dict(base=math.inf),
            dict(base=math.nan), dict(scaling="linear", factor=0.0), dict(scaling="linear", factor=math.inf),
            dict(scaling="ntk", rot_dim=2, factor=2.0), dict(scaling="yarn", factor=2.0, low=4.0, high=4.0),
            dict(scaling="llama3", factor=2.0, orig_len=0.0), dict(scaling="llama3", factor=-1.0),
            dict(scaling="factors"), dict(scaling="factors", rot_dim=4, freq_factors=[1.0, 0.0]),
            dict(attn_factor=-1.0), dict(attn_factor=math.nan), dict(pos_stride=-1)]


@pytest.mark.parametrize("bad", BAD_DESC, ids=str)
def test_descriptors_that_are_refused(bad):
    kw = dict(dict(B=1, L=4, Hq=2, Hkv=1, d=64), **bad)
    with pytest.raises(api.SepllmError) as e:
        api.sepllm_rope_frequencies(api.RopeDesc(**kw))
    assert e.value.code == api.INVALID_ARG


@pytest.mark.parametrize("d", [16, 72, 144, 256])
def test_head_sizes_outside_the_attention_calls_are_unsupported(d):
    with pytest.raises(api.SepllmError) as e:
        api.sepllm_rope_frequencies(api.RopeDesc(1, 4, 2, 1, d))
    assert e.value.code == api.UNSUPPORTED


class View(C.Structure):
    _fields_ = [("data", C.c_void_p), ("sb", C.c_int64), ("sh", C.c_int64), ("sl", C.c_int64),
                ("dtype", C.c_int32), ("reserved", C.c_int32)]


@pytest.mark.parametrize("fn", ["sepllm_rope_fwd", "sepllm_rope_bwd"])
def test_views_that_are_refused(fn):
    """Found on the host before anything is launched (the addresses are never used)."""
    desc = api.RopeDesc(2, 4, 2, 1, 64)
    A, Z = 1 << 20, 1 << 24

    def view(data=A, sb=512, sh=256, sl=64, dtype=0):
        return View(data, sb, sh, sl, dtype, 0)

    def call(ins, outs, d=desc, pos=None):
        ins = (View * 3)(*ins) if ins else None
        outs = (View * 3)(*outs) if outs else None
        return getattr(api.lib(), fn)(C.byref(d) if d else None, pos, ins, outs, None)

    none = View()
    good, out = [view(), view(sb=256), none], [view(Z), view(Z + (1 << 16), sb=256), none]
    bad = [
        (None, out), (good, None), ([none] * 3, [none] * 3),
        ([view(), none, none], [none] * 3), ([none] * 3, [view(Z), none, none]),
        ([view(dtype=2), none, none], [view(Z), none, none]),
        ([view(), view(A + 4096, sb=256, dtype=1), none], out),              # two input types
        (good, [view(Z), view(Z + (1 << 16), sb=256, dtype=1), none]),       # two output types
        ([view(A + 1), none, none], [view(Z), none, none]),                  # no bf16 address
        ([view(dtype=1, data=A + 2), none, none], [view(Z), none, none]),    # no fp32 address
        ([view(sl=-64), none, none], [view(Z), none, none]),
        ([view(), none, none], [view(Z, sl=0), none, none]),                 # rows of the output share memory
        ([view(), none, none], [view(Z, sl=63), none, none]),
        ([view(), none, none], [view(Z, sh=128), none, none]),               # heads overlap
        ([view(), none, none], [view(Z, sb=448), none, none]),               # sequences overlap
        ([view(), none, none], [view(A, sh=64, sl=128), none, none]),        # in place with other strides
        ([view(dtype=1), none, none], [view(A, dtype=0), none, none]),       # in place with another type
    ]
    for ins, outs in bad:
        assert call(ins, outs) == api.INVALID_ARG
    assert call(good, out, d=None) == api.INVALID_ARG
    assert call(good, out, pos=C.c_void_p(4)) == api.INVALID_ARG
    assert call(good, out, d=api.RopeDesc(2, 4, 2, 1, 72)) == api.UNSUPPORTED


def test_binding_refuses_what_the_descriptor_does_not_say():
    desc = api.RopeDesc(1, 4, 2, 1, 64)
    with pytest.raises(ValueError):
        api._rope_views(desc, (torch.zeros(1, 2, 5, 64, dtype=torch.bfloat16), None, None), "x")
    with pytest.raises(ValueError):
        api._rope_views(desc, (torch.zeros(1, 2, 4, 64, dtype=torch.float16), None, None), "x")
    with pytest.raises(ValueError):
        api._rope_views(desc, (torch.zeros(1, 2, 64, 4, dtype=torch.bfloat16).transpose(2, 3), None, None), "x")
    with pytest.raises(ValueError):
        api.RopeDesc(1, 4, 2, 1, 64, scaling="factors", freq_factors=[1.0] * 31)
