"""Shared-prefix calls, host side: sizes and refusals (no GPU; the addresses are never used)."""
import ctypes as C

import pytest
import torch

from paper_2412_12094_b200 import api, build

A = C.c_void_p(1 << 20)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()


def _desc(**kw):
    return api.CacheDesc(**dict(dict(B=3, Hkv=2, Hq=8, d=64, a=2, s=8, w=8, c=32, flags=0), **kw))


def test_decode_workspace_holds_both_parts():
    d = _desc()
    own = api.sepllm_decode_workspace_bytes(d)
    for P in (1, 127, 128, 129, 100000, 10 ** 7):
        n = api.sepllm_decode_prefix_workspace_bytes(d, P)
        assert n % 256 == 0 and n >= own
    big = _desc(B=200, Hkv=8, Hq=32, d=128)      # a prefix read by many: parts of the shared kernel as well
    assert api.sepllm_decode_prefix_workspace_bytes(big, 40000) >= api.sepllm_decode_workspace_bytes(big) + (1 << 20)
    with pytest.raises(api.SepllmError) as e:
        api.sepllm_decode_prefix_workspace_bytes(d, 0)
    assert e.value.code == api.INVALID_ARG
    with pytest.raises(api.SepllmError) as e:
        api.sepllm_decode_prefix_workspace_bytes(_desc(d=80), 5)
    assert e.value.code == api.UNSUPPORTED


def _decode(desc=None, P=100, **over):
    names = ("q", "state", "Kc", "Vc", "Kp", "Vp", "prefix_len", "o", "lse", "workspace")
    v = dict({n: A for n in names}, **over)
    desc = _desc() if desc is None else desc
    return api.lib().sepllm_decode_prefix(C.byref(desc), C.c_int32(P), C.c_float(0.0), v["q"], v["state"], v["Kc"],
                                          v["Vc"], v["Kp"], v["Vp"], v["prefix_len"], v["o"], v["lse"],
                                          v["workspace"], None)


def test_decode_refusals():
    for name in ("q", "state", "Kc", "Vc", "Kp", "Vp", "o", "workspace"):
        assert _decode(**{name: None}) == api.INVALID_ARG
        assert _decode(**{name: C.c_void_p((1 << 20) + 8)}) == api.INVALID_ARG
    for name in ("prefix_len", "lse"):
        assert _decode(**{name: C.c_void_p((1 << 20) + 2)}) == api.INVALID_ARG
    assert _decode(P=0) == api.INVALID_ARG and _decode(P=-5) == api.INVALID_ARG
    assert _decode(_desc(B=0)) == api.INVALID_ARG and _decode(_desc(w=0)) == api.INVALID_ARG
    assert _decode(_desc(Hq=7)) == api.INVALID_ARG
    assert _decode(_desc(d=80)) == api.UNSUPPORTED and _decode(_desc(Hq=34)) == api.UNSUPPORTED
    assert _decode(_desc(B=65536)) == api.UNSUPPORTED


def _copy(desc=None, P=32, n=3, **over):
    v = dict({k: A for k in ("state", "Kc", "Vc", "Kp", "Vp", "prefix_len")}, **over)
    desc = _desc(B=1) if desc is None else desc
    return api.lib().sepllm_prefix_from_cache(C.byref(desc), v["state"], v["Kc"], v["Vc"], C.c_int32(P), v["Kp"],
                                              v["Vp"], v["prefix_len"], C.c_int32(n), None)


def test_prefix_from_cache_refusals():
    for name in ("state", "Kc", "Vc", "Kp", "Vp"):
        assert _copy(**{name: None}) == api.INVALID_ARG
        assert _copy(**{name: C.c_void_p((1 << 20) + 8)}) == api.INVALID_ARG
    assert _copy(prefix_len=None) == api.INVALID_ARG
    assert _copy(prefix_len=C.c_void_p((1 << 20) + 2)) == api.INVALID_ARG
    assert _copy(n=-1) == api.INVALID_ARG and _copy(P=0) == api.INVALID_ARG
    assert _copy(_desc(B=2)) == api.INVALID_ARG
    assert _copy(P=31) == api.BUFFER_TOO_SMALL


def _attn(P=100, L=50, Hq=4, d=64, idesc=None, **over):
    names = ("Q", "K", "V", "index", "Kp", "Vp", "prefix_len", "O", "LSE", "workspace")
    v = dict({n: A for n in names}, **over)
    desc = api.AttnDesc(2, Hq, 2, d, L, 0.0, 0)
    idesc = idesc or api.IndexDesc(2, L, 0, 8, 1, 128, 128, L)
    return api.lib().sepllm_attn_prefix_fwd(C.byref(desc), C.byref(idesc), C.c_int32(P), v["Q"], v["K"], v["V"],
                                            v["index"], v["Kp"], v["Vp"], v["prefix_len"], v["O"], v["LSE"],
                                            v["workspace"], None)


def test_attention_refusals_and_workspace():
    for name in ("Q", "K", "V", "index", "Kp", "Vp", "O", "LSE", "workspace"):
        assert _attn(**{name: None}) == api.INVALID_ARG
        assert _attn(**{name: C.c_void_p((1 << 20) + 2)}) == api.INVALID_ARG
    assert _attn(prefix_len=C.c_void_p((1 << 20) + 2)) == api.INVALID_ARG
    assert _attn(P=0) == api.INVALID_ARG and _attn(Hq=3) == api.INVALID_ARG and _attn(L=0) == api.INVALID_ARG
    assert _attn(d=72) == api.UNSUPPORTED
    assert _attn(idesc=api.IndexDesc(2, 51, 0, 8, 1, 128, 128, 51)) == api.INVALID_ARG
    assert _attn(idesc=api.IndexDesc(2, 50, 0, 8, 1, 64, 128, 50)) == api.UNSUPPORTED
    desc, idesc = api.AttnDesc(2, 4, 2, 80, 50, 0.0, 0), api.IndexDesc(2, 50, 0, 8, 1, 128, 128, 50)
    # K and V rows of prefix and side list, or the forward's own, its output in 32 bits and the parts
    assert api.sepllm_attn_prefix_workspace_bytes(desc, idesc, 300) >= 2 * 2 * 2 * 350 * 128 * 2
    fwd, _ = api.sepllm_attn_workspace_bytes(desc, idesc)
    assert api.sepllm_attn_prefix_workspace_bytes(desc, idesc, 30000) >= fwd + 2 * 4 * 50 * (128 + 1) * 4
    with pytest.raises(api.SepllmError):
        api.sepllm_attn_prefix_workspace_bytes(desc, idesc, 0)


def test_binding_refuses_other_shapes_and_types():
    with pytest.raises(ValueError):
        api._expect("x", ("q", torch.zeros(2, 3), (2, 4), torch.float32))
    with pytest.raises(ValueError):
        api._expect("x", ("q", torch.zeros(2, 4), (2, 4), torch.bfloat16))
    api._expect("x", ("q", None, (2, 4), torch.float32), ("k", torch.zeros(2, 4), (2, 4), torch.float32))


def test_binding_refuses_other_devices_and_strided_buffers(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError):
        api._addresses("x", (torch.zeros(2),))           # host memory
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)   # a CPU tensor's device number
    assert api._addresses("x", (None, torch.zeros(0))) == [0, 0]
    with pytest.raises(ValueError):
        api._addresses("x", (torch.zeros(2, 4).t(),))
    with pytest.raises(ValueError):
        api._rope_views(api.RopeDesc(1, 4, 2, 1, 64), (torch.zeros(1, 2, 4, 64), None, None), "x", 0)
