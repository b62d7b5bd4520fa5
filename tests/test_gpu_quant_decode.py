"""sepllm_decode_quant against the oracle's attention over the held values in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, inputs
from tests._gpu_util import build_index
from tests.test_gpu_quant_cache import QuantCache, regions

pytestmark = pytest.mark.gpu


def reference(q, code, step, vcode, vstep, scale):
    """o [G][d], lse [G] of query rows q over held rows, and the bounds on the kernel's errors.

    Scores.  q is held as two numbers of four bits: exact where |q_e| is at least 2^-9 of the head's largest
    element m, else within 2^-17 m.  Products are exact; sums of 32 elements are 32 bits with the codes'
    offset in them (terms up to 23 |q_e| steps), and eight roundings are allowed for each group: 2^-24 * 8 * 23
    * sum |q_e| |step|.  The weight 2^x has 2^-22 of its own, of x up to a few hundred 2^-24 |x| more.
    Output.  P times the step is rounded to bf16 once (2^-8 at most); sums run with the offset 136 in them,
    128 roundings of 2^-24 allowed; the result is rounded to bf16.  LSE: 32 bits of the score's size."""
    G, d = q.shape
    k, v = orc.quant_values(code, step), orc.quant_values(vcode, vstep)
    lam = scale * q @ k.T
    m = np.abs(q).max(-1, keepdims=True)
    small = (np.abs(q) < 2.0 ** -9 * m) * 2.0 ** -17 * m
    group = np.abs(q).reshape(G, -1, 32).sum(-1)
    es = abs(scale) * (small @ np.abs(k).T + 2.0 ** -24 * 8 * 23 * group @ np.abs(step).T) + 2.0 ** -23 * np.abs(lam)
    lse = np.logaddexp.reduce(lam, -1)
    p = np.exp(lam - lse[:, None])
    ep = 2 * es.max(-1, keepdims=True) + 2.0 ** -22 + 2.0 ** -23 * np.abs(lam).max(-1, keepdims=True)   # relative, of p
    o = p @ v
    size, off = p @ np.abs(v), p @ np.repeat(np.abs(vstep), 32, -1)
    eo = (2.0 ** -8 + 2 * ep) * size + 128 * 136 * 2.0 ** -24 * off + 2.0 ** -8 * np.abs(o)
    return o, lse, eo, es.max(-1) + 2.0 ** -22 * (1 + np.abs(lse)) + ep[:, 0]


def check_decode(qc, q, scale=0.0):
    d = qc.desc
    o, lse = qc.decode(q, scale)
    torch.cuda.synchronize()
    assert api.sepllm_last_device_status(qc.ws) == 0
    st = api.read_cache_state(qc.state)
    (kc, ks), (vc, vs) = qc.held()

    def step(bits):
        return torch.from_numpy(bits.view(np.int16).copy()).view(torch.bfloat16).double().numpy()
    G = d.Hq // d.Hkv
    on, ln, qn = o.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
    worst = 0.0
    for b in range(d.B):
        slots = sum(regions(d, st, b), [])
        for h in range(d.Hkv):
            rows = slice(h * G, h * G + G)
            if not slots:
                assert (on[b, rows] == 0).all() and (ln[b, rows] == -np.inf).all()
                continue
            ref, lref, eo, el = reference(qn[b, rows], kc[b, h, slots], step(ks[b, h, slots]), vc[b, h, slots],
                                          step(vs[b, h, slots]), scale or d.d ** -0.5)
            assert (np.abs(on[b, rows] - ref) <= eo).all(), (b, h, float((np.abs(on[b, rows] - ref) / eo).max()))
            assert (np.abs(ln[b, rows] - lref) <= el).all(), (b, h, float(np.abs(ln[b, rows] - lref).max()), el.max())
            worst = max(worst, float((np.abs(on[b, rows] - ref) / eo).max()))
    return o, lse, worst


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def filled(B, Hkv, Hq, d, a, s, w, c, lens, seed, rho=0.2, flags=0, size=1.0):
    """Caches of prompts of the given lengths."""
    L = max(max(lens), 1)
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = inputs.token_ids(seed, B, L, rho)
    idesc, index = build_index(ids, inputs.SEP_IDS, a, 16)
    qc = QuantCache(B, Hkv, Hq, d, a, s, w, c, flags)
    api.sepllm_cache_from_prompt_quant(qc.desc, idesc, index, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                       _normal(g, B, Hkv, L, d) * size, _normal(g, B, Hkv, L, d) * size, qc.state,
                                       qc.Kc, qc.Vc)
    return qc, g


# lengths from none to a few tiles, one below, at and above a warp's tile and a CTA's step
LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (8, 2), (10, 2), (8, 1), (9, 1), (32, 2)])
def test_lengths_and_query_groups(d, Hq, Hkv):
    qc, g = filled(len(LENS), Hkv, Hq, d, 3, 100, 64, 310, LENS, 300 + Hq)
    check_decode(qc, _normal(g, len(LENS), Hq, d))


@pytest.mark.parametrize("d,Hq,Hkv,B,n", [(128, 4, 1, 1, 30000), (64, 2, 2, 1, 9001), (128, 16, 1, 2, 5000),
                                          (128, 32, 8, 40, 700), (64, 4, 4, 130, 200)])
def test_units_cut_over_many_ctas_and_many_units(d, Hq, Hkv, B, n):
    """A few long caches (each cut over many CTAs), and more units than CTAs; lengths differ."""
    g = np.random.default_rng(7)
    lens = [n] + [int(x) for x in g.integers(0, n + 1, size=B - 1)]
    qc, gen = filled(B, Hkv, Hq, d, 4, 64, 32, n + 200, lens, 400 + B)
    check_decode(qc, _normal(gen, B, Hq, d))


def test_rings_that_wrap_and_compacted_caches():
    """Updates past several compactions: entries start anywhere in the rings."""
    B, Hkv, Hq, d, a, s, w, c = 2, 2, 4, 128, 3, 37, 50, 150
    qc, g = filled(B, Hkv, Hq, d, a, s, w, c, [149, 90], 410)
    ids = torch.from_numpy(inputs.token_ids(411, 400, B, 0.3)).cuda()
    for t in range(400):
        qc.update(ids[t], _normal(g, B, Hkv, d), _normal(g, B, Hkv, d))
        if t % 57 == 0:
            check_decode(qc, _normal(g, B, Hq, d))
    assert min(api.read_cache_state(qc.state)["compactions"]) > 3


@pytest.mark.parametrize("scale", [0.0, 0.5, -0.1, 1e-4])
def test_scales_and_sharp_heads(scale):
    """Scores up to +-200, other scales, one of them negative."""
    qc, g = filled(2, 2, 8, 128, 4, 100, 64, 600, [599, 350], 420)
    q = _normal(g, 2, 8, 128) * torch.tensor([0.1, 1, 4, 16, 1, 2, 8, 0.01], device="cuda")[None, :, None]
    check_decode(qc, q.to(torch.bfloat16), scale)


def test_values_of_one_sign_and_of_very_different_sizes():
    """Values all positive (the offsets' sums do not cancel), groups from 2^-40 to 2^40, keys with large channels."""
    B, Hkv, Hq, d, n = 2, 1, 4, 128, 1000
    g = torch.Generator(device="cuda").manual_seed(430)
    ids = inputs.token_ids(430, B, n, 0.1)
    idesc, index = build_index(ids, inputs.SEP_IDS, 4, 16)
    K, V = _normal(g, B, Hkv, n, d), _normal(g, B, Hkv, n, d)
    K[..., 5] *= 20
    K[..., 77] += 10
    V[0] = V[0].abs()
    V[1, ..., 0:32] *= 2.0 ** 40
    V[1, ..., 64:96] *= 2.0 ** -40
    V[1, :, ::3, 32:64] *= 64
    qc = QuantCache(B, Hkv, Hq, d, 4, 64, 64, n + 100)
    api.sepllm_cache_from_prompt_quant(qc.desc, idesc, index, None, K, V, qc.state, qc.Kc, qc.Vc)
    check_decode(qc, _normal(g, B, Hq, d))


def test_query_sizes_from_tiny_to_huge():
    """The split of q follows its size: elements from 2^-60 to 2^60 of heads, one element far above the others,
    zero queries."""
    qc, g = filled(1, 1, 8, 64, 2, 10, 20, 200, [190], 440)
    q = _normal(g, 1, 8, 64).float()
    q[0, 1] *= 2.0 ** -60
    q[0, 2] *= 2.0 ** -126
    q[0, 3, 7] *= 2.0 ** 12
    q[0, 4] = 0
    q[0, 5] *= torch.exp(3 * torch.randn(64, generator=g, device="cuda"))
    check_decode(qc, q.to(torch.bfloat16))
    # so large that the scores are, too: one entry takes all the weight
    q[0] = 0
    q[0, :, 3] = 2.0 ** 100
    o, lse = qc.decode(q.to(torch.bfloat16))
    K, V, _ = qc.entries()
    i = int(K[0, 0, :190, 3].float().argmax())
    best = K[0, 0, :190, 3].float()
    if int((best == best[i]).sum()) == 1:
        # (V as it is held: one rounding of P times the step, one of the result)
        assert ((o[0, 0].float() - V[0, 0, i].float()).abs() <= 3 * 2.0 ** -8 * V[0, 0, i].float().abs() + 1e-4).all()


def test_not_finite_stays_where_it_is():
    """NaN or infinite keys and values make their kv head's outputs NaN (values: the group's elements only); a
    query element that is not finite its own row; other sequences and heads keep their results."""
    B, Hkv, Hq, d, n = 3, 2, 4, 128, 200
    g = torch.Generator(device="cuda").manual_seed(450)
    ids = inputs.token_ids(450, B, n, 0.1)
    idesc, index = build_index(ids, inputs.SEP_IDS, 0, 16)
    K, V = _normal(g, B, Hkv, n, d), _normal(g, B, Hkv, n, d)
    q = _normal(g, B, Hq, d)

    def run(K, V, q):
        qc = QuantCache(B, Hkv, Hq, d, 0, 20, 64, n + 1)
        api.sepllm_cache_from_prompt_quant(qc.desc, idesc, index, None, K, V, qc.state, qc.Kc, qc.Vc)
        return qc.decode(q)
    o, lse = run(K, V, q)
    K2, V2, q2 = K.clone(), V.clone(), q.clone()
    K2[0, 1, 150, 3] = float("nan")
    V2[1, 0, 199, 40] = float("inf")
    q2[2, 1, 0] = float("inf")
    q2[2, 2, 9] = float("nan")
    o2, lse2 = run(K2, V2, q2)
    bad_o, bad_l = torch.zeros_like(o, dtype=torch.bool), torch.zeros_like(lse, dtype=torch.bool)
    bad_o[0, 2:4] = True
    bad_l[0, 2:4] = True
    bad_o[1, 0:2, 32:64] = True
    bad_o[2, 1:3] = True
    bad_l[2, 1:3] = True
    assert torch.equal(torch.isnan(o2), bad_o) and torch.equal(torch.isnan(lse2), bad_l)
    assert torch.equal(o2[~bad_o], o[~bad_o]) and torch.equal(lse2[~bad_l], lse[~bad_l])


def test_same_result_every_time_without_lse_and_in_any_workspace():
    qc, g = filled(3, 2, 8, 128, 4, 64, 64, 5000, [4999, 17, 2500], 460)
    q = _normal(g, 3, 8, 128)
    o, lse = qc.decode(q)
    for fill in (0, 0xFF):
        qc.ws.fill_(fill)
        o2, lse2 = qc.decode(q)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    o3 = torch.empty_like(o)
    api.sepllm_decode_quant(qc.desc, 0.0, q, qc.state, qc.Kc, qc.Vc, o3, None, qc.ws)
    assert torch.equal(o, o3)


def test_captured_with_the_update_and_two_streams_at_once():
    """A generation step as a graph, replayed; two batches on two streams with a workspace each."""
    B, Hkv, Hq, d = 2, 2, 8, 64
    runs = []
    for k in range(2):
        qc, g = filled(B, Hkv, Hq, d, 2, 30, 40, 400, [399, 120], 470 + k)
        tok = torch.zeros(B, dtype=torch.int32, device="cuda")
        kn, vn, q = _normal(g, B, Hkv, d), _normal(g, B, Hkv, d), _normal(g, B, Hq, d)
        o, lse = torch.zeros((B, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((B, Hq), device="cuda")
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            qc.update(tok, kn, vn)
            api.sepllm_decode_quant(qc.desc, 0.0, q, qc.state, qc.Kc, qc.Vc, o, lse, qc.ws)
        runs.append((qc, g, tok, kn, vn, q, o, lse, stream, graph))
    for t in range(12):
        torch.cuda.synchronize()
        for qc, g, tok, kn, vn, q, *_ in runs:
            tok.fill_(int(inputs.SEP_IDS[t % 9]) if t % 3 else 60)
            for x in (kn, vn, q):
                x.copy_(_normal(g, *x.shape))
        torch.cuda.synchronize()
        for *_, stream, graph in runs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for qc, _, _, _, _, q, o, lse, *_ in runs:
            o2, lse2, _ = check_decode(qc, q)
            assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 4, 2), (128, 6, 1)])
@pytest.mark.parametrize("c", [511, 512, 513, 1025])
def test_capacities_about_the_change_from_one_cta_a_unit(d, Hq, Hkv, c):
    """Short caches are one CTA's each, longer ones are cut into equal runs: both, full and nearly empty."""
    qc, g = filled(3, Hkv, Hq, d, 2, 40, 30, c, [c - 1, 1, 300], 480 + c)
    check_decode(qc, _normal(g, 3, Hq, d))


def test_offsets_past_two_to_the_32():
    """The last sequence's rows start more than 2^32 bytes into the buffers: hand-off, updates, read-back, decode.
    (In the fundamental design: an update of the streaming one looks at no more than 24 576 entries.)"""
    B, Hkv, Hq, d, a, s, w, c, L = 36, 2, 4, 128, 2, 1000, 60, 10 ** 6, 300
    g = torch.Generator(device="cuda").manual_seed(490)
    ids = inputs.token_ids(490, B, L, 0.2)
    idesc, index = build_index(ids, inputs.SEP_IDS, a, 16)
    qc = QuantCache(B, Hkv, Hq, d, a, s, w, c, api.CACHE_FIXED_WINDOW)
    assert (B * Hkv - 1) * (c + s) * d // 2 > 2 ** 32
    K, V = (_normal(g, B, Hkv, L, d) for _ in "kv")
    lens = [0] * (B - 1) + [L]
    api.sepllm_cache_from_prompt_quant(qc.desc, idesc, index, torch.tensor(lens, dtype=torch.int32, device="cuda"), K, V,
                                       qc.state, qc.Kc, qc.Vc)
    k1, v1 = (_normal(g, B, Hkv, d) for _ in "kv")
    qc.update(torch.full((B,), 60, dtype=torch.int32, device="cuda"), k1, v1)
    q = _normal(g, B, Hq, d)
    o, lse = qc.decode(q)
    Ke, Ve = (torch.empty((B, Hkv, c, d), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    n = torch.empty(B, dtype=torch.int32, device="cuda")
    api.sepllm_cache_entries_quant(qc.desc, qc.state, qc.Kc, qc.Vc, c, Ke, Ve, n)
    assert api.sepllm_last_device_status(qc.state) == 0
    for b in (0, B - 1):
        oc = orc.FundamentalCache(a, w)
        for t in range(lens[b] + 1):
            oc.update(t < lens[b] and bool(np.isin(ids[b, t], inputs.SEP_IDS)))
        kept = oc.retained()
        assert n[b] == len(kept) and (b == 0 or len(oc.sep) > 20)
        rows = [torch.cat((x[b, :, : lens[b]], y[b][:, None]), 1)[:, kept].double().cpu().numpy()
                for x, y in ((K, k1), (V, v1))]
        for h in range(Hkv):
            (kc, ks), (vc, vs) = (orc.quantise_rows(x[h]) for x in rows)
            for out, code, step in ((Ke, kc, ks), (Ve, vc, vs)):
                val = torch.from_numpy(orc.quant_values(code, step)).float().to(torch.bfloat16)
                assert torch.equal(out[b, h, : len(kept)].cpu(), val)
            G = Hq // Hkv
            qn = q[b, h * G:h * G + G].double().cpu().numpy()
            ref, lref, eo, el = reference(qn, kc, ks, vc, vs, d ** -0.5)
            assert (np.abs(o[b, h * G:h * G + G].double().cpu().numpy() - ref) <= eo).all()
            assert (np.abs(lse[b, h * G:h * G + G].double().cpu().numpy() - lref) <= el).all()
