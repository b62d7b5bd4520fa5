"""The binding hands every argument over in the width that the header declares (no GPU): the table of
ctypes types against sepllm.h, and calls through the binding into a stand-in library, generated from the
header, that keeps what it was given."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from paper_2412_12094_b200 import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STREAM = 0x7F0012345678    # a handle that does not fit 32 bits, as drivers hand them out


def _prototypes():
    """Parameters of every call that returns a status, as (C type, name)."""
    text = open(os.path.join(ROOT, "include", "sepllm.h")).read()
    text = re.sub(r"/\*.*?\*/", " ", text, flags=re.S)
    out = {}
    for name, args in re.findall(r"\bsepllm_status\s+(sepllm_\w+)\s*\(([^)]*)\)\s*;", text):
        out[name] = [re.match(r"\s*(.*?)(\w+)\s*$", a, re.S).groups() for a in args.split(",")]
    return out


def _ctype(c):
    return C.c_void_p if "*" in c else {"int32_t": C.c_int32, "float": C.c_float}[c.strip()]


def test_argument_types_are_those_of_the_header():
    protos = _prototypes()
    assert len(protos) == len(api.EXPORTS) - 1     # (sepllm_status_string returns text)
    for name, types in api._ARGTYPES.items():
        assert types == [_ctype(c) for c, _ in protos[name]], name


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    d = tmp_path_factory.mktemp("stub")
    body = ["#include <string.h>", '#include "sepllm.h"', "unsigned long long got[16];", "int n_got;"]
    for name, args in _prototypes().items():
        # (a parameter is 8 bytes of `got`, its low ones)
        keep = " ".join(f"got[{i}] = 0; memcpy(&got[{i}], &{a}, sizeof {a});" for i, (_, a) in enumerate(args))
        body.append(f"sepllm_status {name}({', '.join(c + ' ' + a for c, a in args)}) "
                    f"{{ {keep} n_got = {len(args)}; return 0; }}")
    src, so = d / "stub.c", d / "stub.so"
    src.write_text("\n".join(body))
    subprocess.run(["gcc", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"), "-o", str(so), str(src)], check=True)
    return C.CDLL(str(so))


@pytest.fixture
def binding(stub, monkeypatch):
    """The binding over the stand-in library, with tensors in host memory and STREAM as the current one."""
    for name, types in api._ARGTYPES.items():
        getattr(stub, name).argtypes = types
    monkeypatch.setattr(api, "_lib", stub)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)   # a CPU tensor's device number
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: STREAM, raising=False)
    n_got, got = C.c_int.in_dll(stub, "n_got"), (C.c_ulonglong * 16).in_dll(stub, "got")
    return lambda: list(got[:n_got.value])


def test_streams_and_addresses_arrive_whole(binding):
    bf = torch.bfloat16
    buf = torch.zeros(64, dtype=torch.uint8)
    B, L, Hq, Hkv, d, P = 2, 5, 4, 2, 64, 9
    q, k = torch.zeros((B, Hq, L, d), dtype=bf), torch.zeros((B, Hkv, L, d), dtype=bf)
    o, lse, plen = torch.zeros_like(q), torch.zeros((B, Hq, L)), torch.zeros(B, dtype=torch.int32)
    kp, vp = (torch.zeros((Hkv, P, d), dtype=bf) for _ in range(2))

    def ends(n_front, *tensors):
        got = binding()
        assert got[n_front:] == [t.data_ptr() for t in tensors] + [STREAM]

    api.sepllm_attn_prefix_fwd(api.AttnDesc(B, Hq, Hkv, d, L, 0.0, 0), api.IndexDesc(B, L, 0, 8, 1, 128, 128, L), P,
                               q, k, k, buf, kp, vp, plen, o, lse, buf)
    ends(3, q, k, k, buf, kp, vp, plen, o, lse, buf)
    cd = api.CacheDesc(B, Hkv, Hq, d, 0, 4, 3, 16)
    q1, o1, l1 = q[:, :, 0].contiguous(), o[:, :, 0].contiguous(), lse[:, :, 0].contiguous()
    api.sepllm_decode_prefix(cd, P, 0.5, q1, buf, k, k, kp, vp, plen, o1, l1, buf)
    ends(3, q1, buf, k, k, kp, vp, plen, o1, l1, buf)
    api.sepllm_prefix_from_cache(cd, buf, k, k, P, kp, vp, plen)
    got = binding()
    assert got[1:4] + got[5:8] == [t.data_ptr() for t in (buf, k, k, kp, vp, plen)]
    assert got[4] == P and got[8] == B and got[9] == STREAM
    pos = torch.zeros((B, L), dtype=torch.int64)
    for call in (api.sepllm_rope_fwd, api.sepllm_rope_bwd):
        call(api.RopeDesc(B, L, Hq, Hkv, d), pos, q, k, k, o, k, k)
        got = binding()
        assert got[1] == pos.data_ptr() and got[4] == STREAM and len(got) == 5
