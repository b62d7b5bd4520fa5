"""Head norms with rotary positions, host side: the oracle's gradient against differences, refusals and
argument widths (no GPU; the addresses are never used)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, build
from tests.test_abi_argtypes import STREAM, binding, stub  # noqa: F401  (fixtures)
from tests.test_rope_host import BAD_DESC, View


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()


@pytest.mark.parametrize("offset,weights", [(0.0, True), (1.0, True), (0.0, False)])
def test_oracle_norm_and_gradient_against_differences(offset, weights):
    g = np.random.default_rng(3)
    x, dy, eps = g.normal(size=(2, 3, 6)), g.normal(size=(2, 3, 6)), 0.1
    w = g.normal(size=6) if weights else None
    y = orc.head_norm(x, w, eps, offset)
    for i in np.ndindex(2, 3):
        r = 1.0 / math.sqrt(sum(v * v for v in x[i]) / 6 + eps)
        assert np.allclose(y[i], [v * r * ((offset + w[e]) if weights else 1.0) for e, v in enumerate(x[i])], rtol=1e-13)
    dx, dw = orc.head_norm_bwd(x, w, dy, eps, offset)
    f = lambda a, b: float((dy * orc.head_norm(a, b, eps, offset)).sum())  # noqa: E731
    for i in [(0, 0, 0), (1, 2, 5), (0, 1, 3)]:
        e = np.zeros_like(x)
        e[i] = 1e-5
        assert abs((f(x + e, w) - f(x - e, w)) / 2e-5 - dx[i]) < 1e-8
    if weights:
        for k in range(6):
            e = np.zeros(6)
            e[k] = 1e-5
            assert abs((f(x, w + e) - f(x, w - e)) / 2e-5 - dw[k]) < 1e-8


A, Z, X = 1 << 20, 1 << 24, 1 << 28
NONE = View()
P = C.c_void_p


def view(data=A, sb=512, sh=256, sl=64, dtype=0):
    return View(data, sb, sh, sl, dtype, 0)


def _norm(wq=1 << 16, wk=1 << 17, w_dtype=0, eps=1e-6, offset=0.0):
    n = api.QkNorm(eps=eps, offset=offset)
    n.wq, n.wk, n.w_dtype = wq, wk, w_dtype
    return n


def fwd(ins=None, outs=None, desc=None, norm=None, pos=None, no_norm=False):
    desc = api.RopeDesc(2, 4, 2, 1, 64) if desc is None else desc
    ins = (View * 3)(*(ins or [view(), view(sb=256), NONE]))
    outs = (View * 3)(*(outs or [view(Z), view(Z + (1 << 16), sb=256), NONE]))
    return api.lib().sepllm_qknorm_rope_fwd(C.byref(desc), None if no_norm else C.byref(norm or _norm()), pos, ins, outs,
                                            None)


def bwd(xs=None, ins=None, outs=None, desc=None, norm=None, dwq=P(1 << 18), dwk=P(1 << 19), ws=P(1 << 21), no_x=False):
    desc = api.RopeDesc(2, 4, 2, 1, 64) if desc is None else desc
    xs = None if no_x else (View * 3)(*(xs or [view(X), view(X + (1 << 16), sb=256), NONE]))
    ins = (View * 3)(*(ins or [view(), view(sb=256), NONE]))
    outs = (View * 3)(*(outs or [view(Z), view(Z + (1 << 16), sb=256), NONE]))
    return api.lib().sepllm_qknorm_rope_bwd(C.byref(desc), C.byref(norm or _norm()), None, xs, ins, outs, dwq, dwk, ws,
                                            None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_norms_that_are_refused(call):
    for bad in (dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(offset=math.nan),
                dict(w_dtype=2), dict(w_dtype=-1), dict(wq=(1 << 16) + 1), dict(wk=(1 << 16) + 2, w_dtype=1)):
        assert call(norm=_norm(**bad)) == api.INVALID_ARG, bad
    assert fwd(no_norm=True) == api.INVALID_ARG


@pytest.mark.parametrize("call", [fwd, bwd])
def test_views_that_are_refused(call):
    good = [view(), view(sb=256), NONE]
    out = [view(Z), view(Z + (1 << 16), sb=256), NONE]
    for ins, outs in [([NONE] * 3, [NONE] * 3), ([view(), NONE, NONE], out), (good, [view(Z), NONE, NONE]),
                      ([view(dtype=2), NONE, NONE], [view(Z), NONE, NONE]),
                      (good, [view(Z), view(Z + (1 << 16), sb=256, dtype=1), NONE]),
                      ([view(A + 1), NONE, NONE], [view(Z), NONE, NONE]),
                      (good, [view(Z, sl=32), view(Z + (1 << 16), sb=256), NONE])]:
        assert call(ins=ins, outs=outs) == api.INVALID_ARG
    assert call(desc=api.RopeDesc(2, 4, 2, 1, 72)) == api.UNSUPPORTED
    for bad in BAD_DESC:
        assert call(desc=api.RopeDesc(**dict(dict(B=1, L=4, Hq=2, Hkv=1, d=64), **bad))) == api.INVALID_ARG


def test_inputs_of_the_gradient_that_are_refused():
    x = [view(X), view(X + (1 << 16), sb=256), NONE]
    for xs in ([NONE, x[1], NONE], [x[0], NONE, NONE],                    # there in the gradients only
               [view(X, dtype=1), x[1], NONE], [view(X + 1), x[1], NONE], [view(X, sl=-64), x[1], NONE],
               [view(Z, sh=64, sl=128), x[1], NONE]):                     # in place with other strides
        assert bwd(xs=xs) == api.INVALID_ARG
    assert bwd(xs=[x[0], NONE, NONE], ins=[view(), NONE, NONE], outs=[view(Z, dtype=1), NONE, NONE]) == api.INVALID_ARG
    assert bwd(no_x=True) == api.INVALID_ARG
    assert bwd(ws=None) == api.INVALID_ARG and bwd(ws=P((1 << 21) + 128)) == api.INVALID_ARG
    assert bwd(dwq=P((1 << 18) + 2)) == api.INVALID_ARG and bwd(dwk=P((1 << 18) + 2)) == api.INVALID_ARG
    assert bwd(norm=_norm(wq=None)) == api.INVALID_ARG      # the gradient of weights that are not there
    assert bwd(norm=_norm(wk=None)) == api.INVALID_ARG


def test_workspace_size():
    n = {d: api.sepllm_qknorm_rope_bwd_workspace_bytes(api.RopeDesc(2, 4, 2, 1, d)) for d in (64, 80, 128)}
    assert all(v % 256 == 0 and v >= 2 * d * 4 for d, v in n.items())
    with pytest.raises(api.SepllmError) as e:
        api.sepllm_qknorm_rope_bwd_workspace_bytes(api.RopeDesc(2, 4, 2, 1, 72))
    assert e.value.code == api.UNSUPPORTED


def test_binding(binding):  # noqa: F811
    bf, f32 = torch.bfloat16, torch.float32
    B, L, Hq, Hkv, d = 2, 5, 4, 2, 64
    desc = api.RopeDesc(B, L, Hq, Hkv, d)
    q, k = torch.zeros((B, Hq, L, d), dtype=bf), torch.zeros((B, Hkv, L, d), dtype=bf)
    pos, w, dw, ws = torch.zeros((B, L), dtype=torch.int64), torch.zeros(d), torch.zeros(d), torch.zeros(8, dtype=torch.uint8)
    norm = api.QkNorm(w, w, eps=1e-5, offset=1.0)
    api.sepllm_qknorm_rope_fwd(desc, norm, pos, q, k, k, q, k, k)
    got = binding()
    assert got[2] == pos.data_ptr() and got[5] == STREAM and len(got) == 6 and norm.wq == w.data_ptr() and norm.w_dtype == 1
    api.sepllm_qknorm_rope_bwd(desc, norm, None, q, k, q, k, k, q, k, k, dw, None, ws)
    got = binding()
    assert got[2] == 0 and got[6:] == [dw.data_ptr(), 0, ws.data_ptr(), STREAM]
    with pytest.raises(ValueError):
        api.QkNorm(w, w.to(bf))
    with pytest.raises(ValueError):
        api.QkNorm(w.double())
    with pytest.raises(ValueError):
        api.sepllm_qknorm_rope_fwd(desc, api.QkNorm(torch.zeros(d + 1)), None, q, k, k, q, k, k)
    with pytest.raises(ValueError):
        api.sepllm_qknorm_rope_fwd(desc, api.QkNorm(torch.zeros(2 * d)[::2]), None, q, k, k, q, k, k)
    with pytest.raises(ValueError):
        api.sepllm_qknorm_rope_bwd(desc, norm, None, q, k, q, k, k, q, k, k, dw.to(bf), None, ws)
    with pytest.raises(ValueError):
        api.sepllm_qknorm_rope_bwd(desc, norm, None, q[:, :3], k, q, k, k, q, k, k, dw, dw, ws)
    with pytest.raises(ValueError):
        api.sepllm_qknorm_rope_bwd(desc, norm, None, q, k, q, k, k, q, k, k, dw, dw, torch.zeros(8, dtype=f32)[::2])
