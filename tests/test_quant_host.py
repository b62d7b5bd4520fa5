"""The cache in 4 bits, host side: the oracle's format against its definition, sizes, refusals and argument
widths (no GPU; the addresses are never used)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, build
from tests.test_abi_argtypes import STREAM, binding, stub  # noqa: F401  (fixtures)

A = C.c_void_p(1 << 20)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()


def _bf16(x):
    return torch.tensor(x, dtype=torch.float32).to(torch.bfloat16).double().numpy()


def test_oracle_codes_are_the_nearest_multiples():
    g = np.random.default_rng(1)
    x = _bf16(g.normal(size=(200, 64)) * np.exp(g.normal(size=(200, 1)) * 4))
    x[:20] = _bf16(g.integers(-16, 17, size=(20, 64)) / 8.0)       # many ties
    code, step = orc.quantise_rows(x)
    assert code.min() == -8 and code.max() == 7
    s = np.repeat(step, 32, -1)
    for n in range(-8, 8):      # no code is nearer, and of two as near the even one is taken
        mine, other = np.abs(x - code * s), np.abs(x - n * s)
        assert (mine <= other).all()
        assert ((mine < other) | (n == code) | (code % 2 == 0)).all()
    # the element of largest magnitude is held exactly; the others to half a step, or a whole one at 7
    v = orc.quant_values(code, step)
    y = x.reshape(200, 2, 32)
    top = np.where(y.max(-1) >= -y.min(-1), y.max(-1), y.min(-1))[..., None]     # (the positive one of two)
    assert (v.reshape(y.shape)[y == top] == y[y == top]).all()
    assert (np.abs(x - v) <= np.where(code == 7, 1.0, 0.5) * np.abs(s)).all()
    # steps are bf16 numbers
    assert (_bf16(step) == step).all()


def test_oracle_codes_at_the_edges():
    x = np.zeros((6, 32))
    x[1, 3], x[1, 4] = 2.0, -2.0            # two of one size: the positive one sets the step
    x[2, 0] = 2.0 ** -101                   # too small to be held
    x[3, 5], x[3, 6] = -1.0, 1.0 - 2 ** -8  # the other sign beyond 7.5 steps
    x[4, 0] = np.inf
    x[5, 0] = np.nan
    code, step = orc.quantise_rows(x)
    assert step[0] == 0 and (code[0] == 0).all() and step[2] == 0
    assert step[1] == -0.25 and code[1, 3] == -8 and code[1, 4] == 7
    assert step[3] == 0.125 and code[3, 5] == -8 and code[3, 6] == 7
    assert np.isnan(step[4]) and np.isnan(step[5])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m", [4, 8])
def test_places_are_a_permutation_and_unpack_inverts_it(d, m):
    p = orc.quant_places(d, m)
    assert sorted(p.tolist()) == list(range(d))
    g = np.random.default_rng(2)
    rows = 5
    code = g.integers(-8, 8, size=(rows, d))
    held = np.zeros((rows, d), dtype=np.uint8)
    held[:, p] = code + 8
    buf = np.zeros((rows * d // 2 + 255) // 256 * 256 + rows * d // 16, dtype=np.uint8)
    buf[: rows * d // 2] = (held[:, 0::2] | held[:, 1::2] << 4).reshape(-1)
    steps = g.integers(0, 1 << 16, size=(rows, d // 32)).astype(np.uint16)
    buf[-rows * d // 16:] = steps.reshape(-1).view(np.uint8)
    got, st = orc.quant_unpack(buf, rows, d, m)
    assert (got == code).all() and (st == steps).all()


def _desc(**kw):
    return api.CacheDesc(**dict(dict(B=3, Hkv=2, Hq=8, d=64, a=2, s=8, w=8, c=32, flags=0), **kw))


def test_sizes():
    state, kv = api.sepllm_cache_bytes_quant(_desc())
    assert state == api.sepllm_cache_bytes(_desc())[0]
    assert kv == 3 * 2 * 40 * 32 + 3 * 2 * 40 * 4 + (-3 * 2 * 40 * 4) % 256
    full = api.CacheDesc(32, 8, 32, 128, 4, 1024, 256, 3332)
    assert api.sepllm_cache_bytes(full)[1] / api.sepllm_cache_bytes_quant(full)[1] > 3.5
    for d in (_desc(), full, _desc(Hq=32, d=128), _desc(B=1, Hkv=1, Hq=1), _desc(c=2 ** 31 - 100, B=1)):
        n = api.sepllm_decode_quant_workspace_bytes(d)
        assert n % 256 == 0 and 0 < n < 1 << 26
    for fn in (api.sepllm_cache_bytes_quant, api.sepllm_decode_quant_workspace_bytes):
        for bad, code in ((dict(d=80), api.UNSUPPORTED), (dict(w=0), api.INVALID_ARG), (dict(c=18), api.INVALID_ARG),
                          (dict(Hq=34), api.UNSUPPORTED), (dict(Hq=7), api.INVALID_ARG)):
            with pytest.raises(api.SepllmError) as e:
                fn(_desc(**bad))
            assert e.value.code == code


def _call(fn, names, desc, order, no_desc=False, **over):
    v = dict({n: A for n in names}, **over)
    desc = _desc() if desc is None else desc
    return getattr(api.lib(), fn)(None if no_desc else C.byref(desc), *[v[n] if isinstance(n, str) else n for n in order], None)


SEPS = (C.c_int32 * 65)()


def _decode(desc=None, **over):
    names = ("q", "state", "Kc", "Vc", "o", "lse", "workspace")
    return _call("sepllm_decode_quant", names, desc, (C.c_float(0.0), *names), **over)


def _update(desc=None, n_sep=1, sep=SEPS, **over):
    names = ("state", "Kc", "Vc", "ids", "k", "v")
    return _call("sepllm_cache_update_quant", names, desc, ("state", "Kc", "Vc", "ids", sep, C.c_int32(n_sep), "k", "v"),
                 **over)


def _prompt(desc=None, idesc=None, **over):
    names = ("index", "prompt_len", "K", "V", "state", "Kc", "Vc")
    idesc = idesc or api.IndexDesc(3, 50, 2, 8, 0, 128, 128, 50)
    return _call("sepllm_cache_from_prompt_quant", names, desc, (C.byref(idesc), *names), **over)


def _entries(desc=None, n=32, **over):
    names = ("state", "Kc", "Vc", "K", "V", "length")
    return _call("sepllm_cache_entries_quant", names, desc, ("state", "Kc", "Vc", C.c_int32(n), "K", "V", "length"), **over)


@pytest.mark.parametrize("fn,needed,optional", [
    (_decode, {"q": 16, "state": 256, "Kc": 256, "Vc": 256, "o": 2, "workspace": 256}, {"lse": 4}),
    (_update, {"state": 256, "Kc": 256, "Vc": 256, "ids": 4, "k": 16, "v": 16}, {}),
    (_prompt, {"index": 256, "K": 16, "V": 16, "state": 256, "Kc": 256, "Vc": 256}, {"prompt_len": 4}),
    (_entries, {"state": 256, "Kc": 256, "Vc": 256, "K": 16, "V": 16}, {"length": 4})])
def test_addresses_that_are_refused(fn, needed, optional):
    for name, a in {**needed, **optional}.items():
        assert fn(**{name: C.c_void_p((1 << 20) + a // 2)}) == api.INVALID_ARG, name
    for name in needed:
        assert fn(**{name: None}) == api.INVALID_ARG, name
    for bad, code in ((dict(B=0), api.INVALID_ARG), (dict(w=0), api.INVALID_ARG), (dict(d=80), api.UNSUPPORTED),
                      (dict(Hq=7), api.INVALID_ARG), (dict(Hq=34), api.UNSUPPORTED), (dict(flags=2), api.INVALID_ARG)):
        assert fn(_desc(**bad)) == code
    assert fn(None, no_desc=True) == api.INVALID_ARG


def test_other_refusals():
    assert _update(n_sep=-1) == api.INVALID_ARG and _update(n_sep=65) == api.UNSUPPORTED
    assert _update(sep=None) == api.INVALID_ARG
    assert _update(_desc(c=40000)) == api.UNSUPPORTED                   # a compaction of more entries than fit
    assert _update(_desc(Hkv=65536, Hq=65536)) == api.UNSUPPORTED
    for fn in (_decode, _prompt, _entries):
        assert fn(_desc(B=65536)) in (api.UNSUPPORTED, api.INVALID_ARG)
    assert _decode(_desc(B=65536)) == api.UNSUPPORTED and _entries(_desc(B=65536)) == api.UNSUPPORTED
    assert _entries(n=31) == api.BUFFER_TOO_SMALL and _entries(n=0) == api.INVALID_ARG
    assert _prompt(idesc=api.IndexDesc(2, 50, 2, 8, 0, 128, 128, 50)) == api.INVALID_ARG
    assert _prompt(idesc=api.IndexDesc(3, 50, 3, 8, 0, 128, 128, 50)) == api.INVALID_ARG


@pytest.mark.parametrize("fn", [_decode, _update, _prompt])
def test_caches_of_more_slots_than_32_bits_can_wrap_are_refused(fn):
    assert fn(_desc(B=3, s=2 ** 30 - 40, c=2 ** 30, flags=1)) == api.UNSUPPORTED
    assert _entries(_desc(s=0, c=2 ** 30 + 1), n=2 ** 30 + 1) == api.UNSUPPORTED
    # more rows than 32 bits number
    assert _decode(_desc(B=65535, Hkv=64, Hq=64, s=0, c=1025)) == api.UNSUPPORTED


def test_the_size_query_refuses_what_the_calls_refuse():
    with pytest.raises(api.SepllmError) as e:
        api.sepllm_cache_bytes_quant(_desc(s=2 ** 30 - 40, c=2 ** 30, flags=1))
    assert e.value.code == api.UNSUPPORTED
    assert api.sepllm_cache_bytes_quant(_desc(s=0, c=2 ** 30))[1] > 2 ** 30


def test_arguments_arrive_whole(binding):  # noqa: F811
    bf = torch.bfloat16
    d = _desc()
    _, kv = 0, 3 * 2 * 40 * 32 + 3 * 2 * 40 * 4 + (-3 * 2 * 40 * 4) % 256
    state, kc, vc, buf = (torch.zeros(n, dtype=torch.uint8) for n in (1 << 13, kv, kv, 64))
    ids, k1 = torch.zeros(3, dtype=torch.int32), torch.zeros((3, 2, 64), dtype=bf)
    api.sepllm_cache_update_quant(d, state, kc, vc, ids, [5, 6, 7], k1, k1)
    got = binding()
    assert got[1:5] == [t.data_ptr() for t in (state, kc, vc, ids)] and got[6] == 3
    assert got[7:] == [k1.data_ptr(), k1.data_ptr(), STREAM]
    K = torch.zeros((3, 2, 50, 64), dtype=bf)
    api.sepllm_cache_from_prompt_quant(d, api.IndexDesc(3, 50, 2, 8, 0, 128, 128, 50), buf, ids, K, K, state, kc, vc)
    assert binding()[2:] == [t.data_ptr() for t in (buf, ids, K, K, state, kc, vc)] + [STREAM]
    E = torch.zeros((3, 2, 33, 64), dtype=bf)
    api.sepllm_cache_entries_quant(d, state, kc, vc, 33, E, E, None)
    assert binding()[1:] == [state.data_ptr(), kc.data_ptr(), vc.data_ptr(), 33, E.data_ptr(), E.data_ptr(), 0, STREAM]
    q, lse = torch.zeros((3, 8, 64), dtype=bf), torch.zeros((3, 8))
    api.sepllm_decode_quant(d, 0.5, q, state, kc, vc, q, lse, buf)
    got = binding()
    assert got[2:] == [t.data_ptr() for t in (q, state, kc, vc, q, lse, buf)] + [STREAM]
    assert np.array([got[1]], dtype=np.uint64).view(np.float32)[0] == 0.5


def test_binding_refuses_other_shapes_types_and_short_buffers(binding):  # noqa: F811
    bf = torch.bfloat16
    d = _desc()
    kv = 3 * 2 * 40 * 32 + 3 * 2 * 40 * 4 + (-3 * 2 * 40 * 4) % 256
    state, kc = torch.zeros(1 << 13, dtype=torch.uint8), torch.zeros(kv, dtype=torch.uint8)
    ids, k1 = torch.zeros(3, dtype=torch.int32), torch.zeros((3, 2, 64), dtype=bf)
    q = torch.zeros((3, 8, 64), dtype=bf)
    E = torch.zeros((3, 2, 33, 64), dtype=bf)
    with pytest.raises(ValueError):
        api.sepllm_cache_update_quant(d, state, kc, kc, ids.long(), [5], k1, k1)
    with pytest.raises(ValueError):
        api.sepllm_cache_update_quant(d, state, kc, kc, ids, [5], k1.float(), k1)
    with pytest.raises(ValueError):
        api.sepllm_cache_update_quant(d, state, kc[:-1], kc, ids, [5], k1, k1)
    with pytest.raises(ValueError):
        api.sepllm_decode_quant(d, 0.0, q[:, :4], state, kc, kc, q, None, state)
    with pytest.raises(ValueError):
        api.sepllm_decode_quant(d, 0.0, q, state, kc, kc[:256], q, None, state)
    with pytest.raises(ValueError):
        api.sepllm_cache_entries_quant(d, state, kc, kc, 32, E, E)
    with pytest.raises(ValueError):
        api.sepllm_cache_entries_quant(d, state, kc[:256], kc, 33, E, E)
    with pytest.raises(ValueError):
        api.sepllm_cache_from_prompt_quant(d, api.IndexDesc(3, 50, 2, 8, 0, 128, 128, 50), state, None, E, E, state, kc, kc)
