"""Buffers that are too short for the descriptor are refused before a call (it would write, or read, past their end)."""
import pytest
import torch

from paper_2412_12094_b200 import api, build

BF = torch.bfloat16


@pytest.fixture
def sizes_only(monkeypatch):
    """The library for sizes; every other call keeps its name in the list and does nothing.  CPU tensors."""
    build.build()
    real, calls = api.lib(), []

    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes") or "_bytes_" in name or name == "sepllm_status_string":
                return getattr(real, name)
            return lambda *a: calls.append(name) or api.OK
    monkeypatch.setattr(api, "_lib", Library())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    return calls


def _bytes(n):
    return torch.zeros(n, dtype=torch.uint8)


@pytest.mark.parametrize("B,c,s", [(3, 32, 8), (1, 2000, 0), (5, 700, 77)])
def test_state_and_cache_buffers(sizes_only, B, c, s):
    desc = api.CacheDesc(B, 2, 8, 64, 2, s, 8, c)
    idesc = api.IndexDesc(B, 50, 2, 8, 0, 128, 128, 50)
    n_state, n_kv = api.sepllm_cache_bytes_quant(desc)
    ids, row, q = torch.zeros(B, dtype=torch.int32), torch.zeros((B, 2, 64), dtype=BF), torch.zeros((B, 8, 64), dtype=BF)
    K, E = (torch.zeros((B, 2, n, 64), dtype=BF) for n in (50, c))
    index, ws = _bytes(api.sepllm_index_bytes(idesc)[0]), _bytes(api.sepllm_decode_quant_workspace_bytes(desc))

    def run(state=n_state, kc=n_kv, vc=n_kv):
        st, k, v = _bytes(state), _bytes(kc), _bytes(vc)
        return [lambda: api.sepllm_cache_update_quant(desc, st, k, v, ids, [5], row, row),
                lambda: api.sepllm_cache_from_prompt_quant(desc, idesc, index, None, K, K, st, k, v),
                lambda: api.sepllm_cache_entries_quant(desc, st, k, v, c, E, E),
                lambda: api.sepllm_decode_quant(desc, 0.0, q, st, k, v, q, None, ws)]
    for call in run():
        call()
    for call in run(state=n_state + 256):
        call()
    assert len(sizes_only) == 8
    for short in (dict(state=n_state - 1), dict(state=256), dict(kc=n_kv - 1), dict(vc=n_kv - 1)):
        for call in run(**short):
            with pytest.raises(ValueError):
                call()
    assert len(sizes_only) == 8


def test_decode_workspaces(sizes_only):
    """The workspace of a short cache is 256 bytes, that of a longer one megabytes: neither stands for the other."""
    short, long = (api.CacheDesc(2, 2, 8, 64, 2, 8, 8, c) for c in (300, 3000))
    need = api.sepllm_decode_quant_workspace_bytes(long)
    assert need > 256 == api.sepllm_decode_quant_workspace_bytes(short)
    q = torch.zeros((2, 8, 64), dtype=BF)
    for desc, n, ok in ((short, 256, True), (short, 255, False), (long, 256, False), (long, need - 1, False),
                        (long, need, True), (short, need, True)):
        sb, kb = api.sepllm_cache_bytes_quant(desc)
        args = (desc, 0.0, q, _bytes(sb), _bytes(kb), _bytes(kb), q, None, _bytes(n))
        if ok:
            api.sepllm_decode_quant(*args)
        else:
            with pytest.raises(ValueError):
                api.sepllm_decode_quant(*args)
    assert sizes_only.count("sepllm_decode_quant") == 3


@pytest.mark.parametrize("d", [64, 80, 128])
def test_workspace_of_the_norms_gradient(sizes_only, d):
    desc = api.RopeDesc(2, 5, 4, 2, d)
    norm, dw = api.QkNorm(torch.zeros(d), torch.zeros(d)), torch.zeros(d)
    q, k = torch.zeros((2, 4, 5, d), dtype=BF), torch.zeros((2, 2, 5, d), dtype=BF)
    need = api.sepllm_qknorm_rope_bwd_workspace_bytes(desc)
    api.sepllm_qknorm_rope_bwd(desc, norm, None, q, k, q, k, k, q, k, k, dw, dw, _bytes(need))
    for n in (8, need - 1):
        with pytest.raises(ValueError):
            api.sepllm_qknorm_rope_bwd(desc, norm, None, q, k, q, k, k, q, k, k, dw, dw, _bytes(n))
    assert sizes_only == ["sepllm_qknorm_rope_bwd"]
