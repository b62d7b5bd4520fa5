"""The cache in 4 bits on the GPU: update, hand-off and read-back against the oracle's state machine and
format, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, inputs
from tests._gpu_util import build_index

pytestmark = pytest.mark.gpu


class QuantCache:
    def __init__(self, B, Hkv, Hq, d, a, s, w, c, flags=0):
        self.desc = api.CacheDesc(B, Hkv, Hq, d, a, s, w, c, flags)
        sb, kb = api.sepllm_cache_bytes_quant(self.desc)
        self.state, self.Kc, self.Vc = api.alloc_bytes(sb), api.alloc_bytes(kb), api.alloc_bytes(kb)
        self.Kc.fill_(0xAB)
        self.Vc.fill_(0xAB)
        self.ws = api.alloc_bytes(api.sepllm_decode_quant_workspace_bytes(self.desc))
        self.ws.fill_(0xCD)
        api.sepllm_cache_init(self.desc, self.state)
        self.slots = c + s

    def update(self, ids, k, v):
        api.sepllm_cache_update_quant(self.desc, self.state, self.Kc, self.Vc, ids, inputs.SEP_IDS, k, v)

    def decode(self, q, scale=0.0):
        d = self.desc
        o = torch.full((d.B, d.Hq, d.d), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((d.B, d.Hq), 7.0, dtype=torch.float32, device="cuda")
        api.sepllm_decode_quant(d, scale, q, self.state, self.Kc, self.Vc, o, lse, self.ws)
        return o, lse

    def entries(self, extra=0):
        d = self.desc
        K, V = (torch.full((d.B, d.Hkv, d.c + extra, d.d), -7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        n = torch.full((d.B,), -1, dtype=torch.int32, device="cuda")
        api.sepllm_cache_entries_quant(d, self.state, self.Kc, self.Vc, d.c + extra, K, V, n)
        return K, V, n

    def held(self):
        """Codes [B][Hkv][slots][d] and step bits of K and of V, from the buffers."""
        d, out = self.desc, []
        for buf, m in ((self.Kc, 8), (self.Vc, 4)):
            c, s = orc.quant_unpack(buf.cpu().numpy(), d.B * d.Hkv * self.slots, d.d, m)
            out.append((c.reshape(d.B, d.Hkv, self.slots, d.d), s.reshape(d.B, d.Hkv, self.slots, d.d // 32)))
        return out


def regions(desc, st, b):
    """Slots of the three regions, in order."""
    ring = desc.c - desc.a
    return ([i for i in range(st["size_init"][b])],
            [desc.a + (st["sep_start"][b] + i) % max(desc.s, 1) for i in range(st["size_sep"][b])],
            [desc.a + desc.s + (st["win_start"][b] + i) % ring for i in range(st["size_win"][b])])


def step_bits(step):
    """bf16 bits of steps; NaN as the library writes it."""
    t = torch.from_numpy(np.ascontiguousarray(step, dtype=np.float32)).to(torch.bfloat16)
    bits = t.view(torch.int16).numpy().view(np.uint16).copy()
    bits[np.isnan(step)] = 0x7fc0
    bits[step == 0] = 0
    return bits


def check_cache(qc, oc, f, K, V):
    """Sizes, retained positions in order, counters; codes and steps of every retained row; and the entries
    read back.  K, V: bf16 CPU tensors [B][Hkv][T][d] of the text."""
    d = qc.desc
    st = api.read_cache_state(qc.state)
    (kcode, kstep), (vcode, vstep) = qc.held()
    Ke, Ve, n = (t.cpu() for t in qc.entries(extra=3))
    for b in range(d.B):
        reg = regions(d, st, b)
        assert [[int(st["slot_pos"][b][i]) for i in r] for r in reg] == [oc[b].init, oc[b].sep, oc[b].window], b
        assert st["next_pos"][b] == oc[b].next_pos and st["compactions"][b] == oc[b].compactions
        slots, kept = sum(reg, []), oc[b].retained()
        assert st["slot_is_sep"][b][slots].astype(bool).tolist()[len(reg[0]):] == [bool(f[b, p]) for p in kept][len(reg[0]):]
        assert n[b] == len(kept)
        for code, step, x, out in ((kcode, kstep, K, Ke), (vcode, vstep, V, Ve)):
            ref, s = orc.quantise_rows(x[b][:, kept].double().numpy())
            got = step[b][:, slots]
            got = np.where(got == 0x8000, 0, got)         # (a zero of either sign)
            assert np.array_equal(code[b][:, slots], ref) and np.array_equal(got, step_bits(s)), b
            # values: the product is exact in 32 bits, its rounding to bf16 is torch's
            val = torch.from_numpy(orc.quant_values(ref, s)).float().to(torch.bfloat16)
            assert torch.equal(out[b][:, : len(kept)].nan_to_num(9e9), val.nan_to_num(9e9))
            assert (out[b][:, len(kept):] == -7.0).all()
    return st


def _rows(seed, shape):
    """bf16 rows with groups of very different sizes, exact ties, zeros and equal largest elements."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(3 * torch.randn((*shape[:-1], 1), generator=g))
    grid = torch.randint(-16, 17, shape, generator=g) / 8.0           # codes at ties
    kind = torch.randint(0, 8, (*shape[:-1], 1), generator=g)
    x = torch.where(kind == 0, grid, torch.where(kind == 1, torch.zeros_like(x), x))
    return torch.where(kind == 2, x.abs(), x).to(torch.bfloat16)


def _drive(B, Hkv, Hq, d, a, s, w, c, steps, rho, seed, flags=0, check_every=1):
    ids = inputs.decode_stream_ids(seed, B, steps, rho)
    f = np.isin(ids, inputs.SEP_IDS)
    K, V = _rows(seed, (B, Hkv, steps, d)), _rows(seed + 1, (B, Hkv, steps, d))
    Kd, Vd = K.cuda(), V.cuda()
    ids_d = torch.from_numpy(np.ascontiguousarray(ids.T)).cuda()
    qc = QuantCache(B, Hkv, Hq, d, a, s, w, c, flags)
    oc = [orc.FundamentalCache(a, w) if flags else orc.StreamingCache(a, s, w, c) for _ in range(B)]
    for t in range(steps):
        qc.update(ids_d[t], Kd[:, :, t].contiguous(), Vd[:, :, t].contiguous())
        for b in range(B):
            oc[b].update(bool(f[b, t]))
        if (t + 1) % check_every == 0 or t == steps - 1:
            assert api.sepllm_last_device_status(qc.state) == 0
            check_cache(qc, oc, f, K, V)
    return qc, oc


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 2, 2), (128, 8, 2)])
def test_update_every_step(d, Hq, Hkv):
    _, oc = _drive(2, Hkv, Hq, d, a=2, s=5, w=4, c=20, steps=130, rho=0.3, seed=150 + d)
    assert min(x.compactions for x in oc) > 5


@pytest.mark.parametrize("a,s,w,c,rho", [(0, 3, 2, 9, 0.5), (3, 0, 5, 12, 0.5), (1, 4, 3, 30, 0.9), (0, 1, 1, 3, 1.0)])
def test_update_at_the_edges(a, s, w, c, rho):
    """No initial tokens, no separator ring, separators in bursts, the smallest cache."""
    _drive(2, 1, 1, 64, a, s, w, c, steps=90, rho=rho, seed=160 + c, check_every=4)


@pytest.mark.parametrize("d", [64, 128])
def test_update_in_the_fundamental_design(d):
    _drive(2, 2, 4, d, a=3, s=60, w=7, c=100, steps=150, rho=0.3, seed=170 + d, flags=api.CACHE_FIXED_WINDOW, check_every=5)


def test_update_many_past_entries():
    """A compaction of thousands of entries (more ranks in shared memory than the default allows)."""
    a, s, w, c = 1, 3000, 8, 22010
    B, Hkv, d, L = 1, 1, 64, 21990
    ids = inputs.token_ids(171, B, L + 30, 0.2)
    f = np.isin(ids, inputs.SEP_IDS)
    K, V = _rows(171, (B, Hkv, L + 30, d)), _rows(172, (B, Hkv, L + 30, d))
    qc = QuantCache(B, Hkv, 1, d, a, s, w, c)
    idesc, index = build_index(np.ascontiguousarray(ids[:, :L]), inputs.SEP_IDS, a, 16)
    api.sepllm_cache_from_prompt_quant(qc.desc, idesc, index, None, K[:, :, :L].contiguous().cuda(),
                                       V[:, :, :L].contiguous().cuda(), qc.state, qc.Kc, qc.Vc)
    oc = [orc.cache_after_prompt(f[0, :L], a, s, w, c)]
    for t in range(L, L + 30):
        qc.update(torch.from_numpy(ids[:, t].copy()).cuda(), K[:, :, t].contiguous().cuda(), V[:, :, t].contiguous().cuda())
        oc[0].update(bool(f[0, t]))
    assert oc[0].compactions == 1
    check_cache(qc, oc, f, K, V)


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 2, 2), (128, 8, 2)])
def test_hand_off_every_prompt_length(d, Hq, Hkv):
    a, s, w, c, B, L = 2, 5, 4, 20, 8, 64
    ids = inputs.token_ids(180 + d, B, L, 0.3)
    f = np.isin(ids, inputs.SEP_IDS)
    K, V = _rows(180 + d, (B, Hkv, L, d)), _rows(181 + d, (B, Hkv, L, d))
    idesc, index = build_index(ids, inputs.SEP_IDS, a, 16)
    for first in range(0, L + 1, B):
        lens = [min(L, first + b) for b in range(B)]
        qc = QuantCache(B, Hkv, Hq, d, a, s, w, c)
        api.sepllm_cache_from_prompt_quant(qc.desc, idesc, index, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                           K.cuda(), V.cuda(), qc.state, qc.Kc, qc.Vc)
        assert api.sepllm_last_device_status(qc.state) == 0
        check_cache(qc, [orc.cache_after_prompt(f[b, :lens[b]], a, s, w, c) for b in range(B)], f, K, V)


@pytest.mark.parametrize("flags", [0, api.CACHE_FIXED_WINDOW])
def test_hand_off_then_updates_equal_updates_alone(flags):
    B, Hkv, d, a, s, w, c, L, more = 3, 2, 128, 4, 40, 16, 100, 140, 60
    ids = inputs.token_ids(190, B, L + more, 0.2)
    f = np.isin(ids, inputs.SEP_IDS)
    K, V = _rows(190, (B, Hkv, L + more, d)), _rows(191, (B, Hkv, L + more, d))
    qc = QuantCache(B, Hkv, 4, d, a, s, w, c, flags)
    idesc, index = build_index(np.ascontiguousarray(ids[:, :L]), inputs.SEP_IDS, a, 16)
    api.sepllm_cache_from_prompt_quant(qc.desc, idesc, index, None, K[:, :, :L].contiguous().cuda(),
                                       V[:, :, :L].contiguous().cuda(), qc.state, qc.Kc, qc.Vc)
    oc = []
    for b in range(B):
        o = orc.FundamentalCache(a, w) if flags else orc.StreamingCache(a, s, w, c)
        for t in range(L):
            o.update(bool(f[b, t]))
        oc.append(o)
    check_cache(qc, oc, f, K, V)
    for t in range(L, L + more):
        qc.update(torch.from_numpy(ids[:, t].copy()).cuda(), K[:, :, t].contiguous().cuda(), V[:, :, t].contiguous().cuda())
        for b in range(B):
            oc[b].update(bool(f[b, t]))
    # (a fixed window's text that has more than s separators keeps the newest s, and says so)
    assert api.sepllm_last_device_status(qc.state) == (
        api.CAPACITY_EXCEEDED if flags and max(len(o.sep) for o in oc) > s else 0)
    for o in oc:
        o.sep = o.sep[-s:]
    check_cache(qc, oc, f, K, V)


def test_separators_beyond_a_fixed_windows_capacity_are_reported():
    B, a, s, w, c = 1, 1, 3, 2, 10
    qc = QuantCache(B, 1, 1, 64, a, s, w, c, api.CACHE_FIXED_WINDOW)
    x = torch.ones((B, 1, 64), dtype=torch.bfloat16, device="cuda")
    sep = torch.tensor([int(inputs.SEP_IDS[0])], dtype=torch.int32, device="cuda")
    for t in range(9):
        qc.update(sep, x, x)
    assert api.sepllm_last_device_status(qc.state) == api.CAPACITY_EXCEEDED
    st = api.read_cache_state(qc.state)
    assert (st["size_init"][0], st["size_sep"][0], st["size_win"][0]) == (1, 3, 2)


def test_numbers_that_are_not_finite_and_the_ends_of_the_range():
    """NaN and infinities make their group NaN and no other; the largest and smallest bf16 numbers."""
    B, Hkv, d = 1, 1, 128
    qc = QuantCache(B, Hkv, 1, d, 0, 0, 8, 16)
    rows = torch.zeros((8, d))
    rows[0] = torch.linspace(-3, 3, d)
    rows[0, 5], rows[1, 40], rows[1, 70], rows[1, 100] = float("nan"), float("inf"), -float("inf"), 2.5
    big = float(torch.finfo(torch.bfloat16).max)
    rows[2, 0], rows[2, 1], rows[2, 2] = big, -big, big / 2
    rows[2, 32], rows[2, 33] = -big, big / 16
    rows[3, 0], rows[3, 32], rows[3, 33] = 2.0 ** -100, 2.0 ** -101, -(2.0 ** -120)
    rows[4] = 2.0 ** -130                      # below the normal numbers
    rows[5, :32] = -1.0
    rows[6] = torch.arange(d) % 7 - 3.0
    rows = rows.to(torch.bfloat16)
    ids = torch.tensor([60], dtype=torch.int32, device="cuda")
    for t in range(8):
        qc.update(ids, rows[t].view(1, 1, d).cuda(), rows[7 - t].view(1, 1, d).cuda())
    (kc, ks), (vc, vs) = qc.held()
    for code, step, x in ((kc, ks, rows), (vc, vs, rows.flip(0))):
        ref, s = orc.quantise_rows(x.double().numpy())
        got = np.where(step[0, 0, :8] == 0x8000, 0, step[0, 0, :8])
        assert np.array_equal(code[0, 0, :8], ref) and np.array_equal(got, step_bits(s))
    K, V, n = qc.entries()
    val = torch.from_numpy(orc.quant_values(*orc.quantise_rows(rows.double().numpy()))).float().to(torch.bfloat16)
    assert torch.equal(K[0, 0, :8].cpu().nan_to_num(1.5), val.nan_to_num(1.5)) and n.item() == 8
    assert torch.equal(V[0, 0, :8].cpu().nan_to_num(1.5), val.flip(0).nan_to_num(1.5))
    assert (K[0, 0, 8:] == -7.0).all()


def test_prompt_lengths_out_of_range_and_another_index_leave_the_cache_empty():
    a, s, w, c, B, L = 2, 5, 4, 20, 3, 40
    ids = inputs.token_ids(200, B, L, 0.3)
    K = _rows(200, (B, 1, L, 64)).cuda()
    idesc, index = build_index(ids, inputs.SEP_IDS, a, 16)
    qc = QuantCache(B, 1, 1, 64, a, s, w, c)
    api.sepllm_cache_from_prompt_quant(qc.desc, idesc, index, torch.tensor([5, L + 1, -1], dtype=torch.int32, device="cuda"),
                                       K, K, qc.state, qc.Kc, qc.Vc)
    assert api.sepllm_last_device_status(qc.state) == api.INVALID_ARG
    assert qc.entries()[2].tolist() == [5, 0, 0]


def test_captured_updates_continue_and_streams():
    """A captured update and read-back, replayed with new tokens, on a stream of its own."""
    B, Hkv, d, a, s, w, c, steps = 2, 2, 64, 2, 5, 4, 20, 70
    ids = inputs.decode_stream_ids(210, B, steps, 0.3)
    f = np.isin(ids, inputs.SEP_IDS)
    K, V = _rows(210, (B, Hkv, steps, d)), _rows(211, (B, Hkv, steps, d))
    qc = QuantCache(B, Hkv, 2, d, a, s, w, c)
    k, v = (torch.zeros((B, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    tok = torch.zeros(B, dtype=torch.int32, device="cuda")
    oc = [orc.StreamingCache(a, s, w, c) for _ in range(B)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            qc.update(tok, k, v)
        for t in range(steps):
            tok.copy_(torch.from_numpy(ids[:, t].copy()))
            k.copy_(K[:, :, t])
            v.copy_(V[:, :, t])
            graph.replay()
            for b in range(B):
                oc[b].update(bool(f[b, t]))
        stream.synchronize()
        check_cache(qc, oc, f, K, V)
