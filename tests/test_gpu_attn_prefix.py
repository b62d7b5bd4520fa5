"""sepllm_attn_prefix_fwd against the oracle's masked softmax over the joined keys, and a serving run
through the shared prefix from the prompt to generated tokens."""
import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, inputs
from tests._gpu_util import TOL_LSE, TOL_O, build_index
from tests.test_gpu_cache import GpuCache

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(BF)


def _index(ids, n, a=0, seq_len=None, doc_first=None):
    B, L = ids.shape
    if seq_len is None and doc_first is None:
        return build_index(ids, inputs.SEP_IDS, a, n)
    desc = api.IndexDesc(B, L, a, n, len(inputs.SEP_IDS), 128, 128, L)
    ib, sb = api.sepllm_index_bytes(desc)
    index, scratch = api.alloc_bytes(ib), api.alloc_bytes(sb)
    ids_d = torch.from_numpy(np.ascontiguousarray(ids)).cuda()
    len_d = None if seq_len is None else torch.tensor(seq_len, dtype=torch.int32, device="cuda")
    if doc_first is not None:
        api.sepllm_build_index_packed(desc, ids_d, torch.from_numpy(doc_first).cuda(), len_d, inputs.SEP_IDS, index)
    else:
        api.sepllm_build_index_varlen(desc, ids_d, len_d, inputs.SEP_IDS, index, scratch)
    return desc, index


def _run(Q, K, V, idesc, index, Kp, Vp, plen, scale=0.0, out=None):
    B, Hq, L, d = Q.shape
    P = Kp.shape[1]
    desc = api.AttnDesc(B, Hq, K.shape[1], d, L, scale, 0)
    ws = api.alloc_bytes(api.sepllm_attn_prefix_workspace_bytes(desc, idesc, P))
    ws.fill_(0xff)
    O, LSE = out or (torch.full_like(Q, 3.5), torch.full((B, Hq, L), -2.5, device="cuda"))
    api.sepllm_attn_prefix_fwd(desc, idesc, P, Q, K, V, index, Kp, Vp, plen, O, LSE, ws)
    torch.cuda.synchronize()
    assert api.sepllm_last_device_status(ws) == 0
    return O, LSE


def _check(Q, K, V, Kp, Vp, masks, plen, seq_len, O, LSE, scale=None, heads=None):
    """Beside the common bounds an entry gets what its terms cost: weights rounded to bf16 (2^-9 at
    most relative to the running reference, five deviations of the terms' root sum of squares) and
    half a step of the bf16 output."""
    B, Hq, L, d = Q.shape
    G = Hq // K.shape[1]
    num, den = 0.0, 0.0
    for b in range(B):
        n, m = seq_len[b], plen[b]
        M = np.concatenate((np.ones((n, m), bool), masks[b][:n, :n]), 1)
        for h in heads or range(Hq):
            q = Q[b, h, :n].double().cpu().numpy()
            k, v = (np.concatenate((x[h // G, :m].double().cpu().numpy(), y[b, h // G, :n].double().cpu().numpy()))
                    for x, y in ((Kp, K), (Vp, V)))
            ref, lref, A = orc.attn_fwd_rows(q, k, v, M, scale)
            rss = np.sqrt(A ** 2 @ v ** 2)
            err = np.abs(O[b, h, :n].double().cpu().numpy() - ref)
            tol = np.maximum(TOL_O["max_abs"], 5 * 2.0 ** -9 * rss + 2.0 ** -8 * np.abs(ref))
            assert (err <= tol).all(), (b, h, float((err / tol).max()))
            num, den = num + (err ** 2).sum(), den + (ref ** 2).sum()
            assert np.abs(LSE[b, h, :n].double().cpu().numpy() - lref).max(initial=0.0) <= TOL_LSE, (b, h)
            # rows behind the end are left as they were
            assert (O[b, h, n:] == 3.5).all() and (LSE[b, h, n:] == -2.5).all()
    assert np.sqrt(num / den) <= TOL_O["rel_fro"]


SHAPES = [
    # B, Hq, Hkv, d, L, P
    (1, 1, 1, 64, 1, 1), (2, 4, 1, 128, 1, 300), (3, 4, 2, 64, 5, 129), (1, 8, 2, 128, 16, 700), (2, 4, 1, 128, 32, 256),
    (3, 6, 2, 80, 43, 200), (2, 3, 1, 96, 50, 333), (2, 5, 5, 64, 130, 128), (1, 8, 2, 128, 257, 1000),
    (2, 4, 4, 112, 129, 64), (9, 8, 1, 64, 3, 500), (5, 8, 2, 128, 100, 640), (1, 2, 1, 64, 700, 2000),
    (40, 4, 4, 128, 140, 260),
    # prefixes long enough for the kernel that shares them
    (2, 4, 1, 128, 1, 9000), (1, 4, 1, 128, 5, 6001), (3, 4, 2, 64, 20, 12000), (1, 8, 2, 128, 16, 5000),
    (2, 6, 2, 80, 43, 8192), (2, 3, 1, 96, 50, 9000), (2, 5, 5, 64, 130, 7777), (1, 8, 2, 128, 257, 6000),
    (2, 4, 4, 112, 129, 5120), (9, 8, 1, 64, 3, 14000), (5, 8, 2, 128, 100, 4000), (1, 2, 1, 64, 700, 9001),
    (40, 4, 4, 128, 140, 2500),
]


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,d,L,P", SHAPES)
def test_forward(B, Hq, Hkv, d, L, P, ragged):
    g = torch.Generator(device="cuda").manual_seed(B * L + P)
    rng = np.random.default_rng(L)
    ids, n = inputs.token_ids(P, B, L, 0.15), max(1, L // 6)
    seq_len = [int(x) for x in rng.integers(0, L + 1, B)] if ragged else [L] * B
    if ragged and seq_len[0] == 0:
        seq_len[0] = L
    plen = [int(x) for x in rng.integers(0, P + 1, B)] if ragged else [P] * B
    idesc, index = _index(ids, n, 0, seq_len if ragged else None)
    Q, K, V = _normal(g, B, Hq, L, d), _normal(g, B, Hkv, L, d), _normal(g, B, Hkv, L, d)
    Q = (Q.float() * 2).to(BF)
    Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    far = max(plen)
    Kp[:, far:], Vp[:, far:] = float("nan"), float("inf")      # behind the longest prefix: anything
    pl = torch.tensor(plen, dtype=torch.int32, device="cuda") if ragged else None
    O, LSE = _run(Q, K, V, idesc, index, Kp, Vp, pl)
    f = np.isin(ids, inputs.SEP_IDS)
    masks = [orc.mask_matrix(f[b], 0, n) for b in range(B)]
    heads = None if B * Hq * L * (P + L) < 4e6 else [0, Hq - 1]
    if B == 40:    # the many-sequence form: a few sequences are enough
        sel = slice(0, 40, 13)
        Q, K, V, O, LSE, masks, plen, seq_len = (x[sel] for x in (Q, K, V, O, LSE, masks, plen, seq_len))
    _check(Q, K, V, Kp, Vp, masks, plen, seq_len, O, LSE, heads=heads)


def test_more_row_tiles_than_one_launch_takes():
    """Sequences and lengths whose row tiles go beyond one launch of the prefix kernel, with units cut
    between its CTAs and whole ones; sampled sequences against the oracle."""
    g = torch.Generator(device="cuda").manual_seed(12)
    B, Hq, Hkv, d, L, P = 300, 2, 1, 64, 130, 2100     # 300 sequences x 3 tiles = 450 pairs
    ids = inputs.token_ids(7, B, L, 0.1)
    lens = [int(x) for x in np.random.default_rng(7).integers(0, L + 1, B)]
    plen = [int(x) for x in np.random.default_rng(8).integers(0, P + 1, B)]
    lens[0], lens[-1], plen[-1], plen[1] = L, L, P, 0
    idesc, index = _index(ids, 20, 0, lens)
    Q, K, V = _normal(g, B, Hq, L, d), _normal(g, B, Hkv, L, d), _normal(g, B, Hkv, L, d)
    Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    O, LSE = _run(Q, K, V, idesc, index, Kp, Vp, torch.tensor(plen, dtype=torch.int32, device="cuda"))
    f = np.isin(ids, inputs.SEP_IDS)
    sel = sorted({0, 1, 2, B - 1, *range(5, B, 17)})
    _check(Q[sel], K[sel], V[sel], Kp, Vp, [orc.mask_matrix(f[b], 0, 20) for b in sel], [plen[b] for b in sel],
           [lens[b] for b in sel], O[sel], LSE[sel])


@pytest.mark.parametrize("P", [150, 9000])
def test_groups_wider_than_a_row_tile(P):
    """200 query heads on one kv head: a token's heads take two row tiles."""
    g = torch.Generator(device="cuda").manual_seed(13)
    B, Hq, d, L = 2, 200, 64, 3
    ids = inputs.token_ids(9, B, L, 0.2)
    idesc, index = _index(ids, 2, 0)
    Q, K, V = _normal(g, B, Hq, L, d), _normal(g, B, 1, L, d), _normal(g, B, 1, L, d)
    Kp, Vp = _normal(g, 1, P, d), _normal(g, 1, P, d)
    O, LSE = _run(Q, K, V, idesc, index, Kp, Vp, torch.tensor([P, 7], dtype=torch.int32, device="cuda"))
    f = np.isin(ids, inputs.SEP_IDS)
    _check(Q, K, V, Kp, Vp, [orc.mask_matrix(f[b], 0, 2) for b in range(B)], [P, 7], [L, L], O, LSE,
           heads=[0, 63, 127, 128, 199])


def test_many_kv_heads_and_a_short_prefix():
    """More (kv head, pair) units than SMs, each with a single key tile."""
    g = torch.Generator(device="cuda").manual_seed(14)
    for B, Hq, d, L, P in ((1, 400, 64, 2, 5), (3, 180, 128, 150, 128), (1, 400, 64, 2, 3000), (3, 180, 128, 150, 2900)):
        ids = inputs.token_ids(10, B, L, 0.2)
        idesc, index = _index(ids, 3, 0)
        Q, K, V = _normal(g, B, Hq, L, d), _normal(g, B, Hq, L, d), _normal(g, B, Hq, L, d)
        Kp, Vp = _normal(g, Hq, P, d), _normal(g, Hq, P, d)
        O, LSE = _run(Q, K, V, idesc, index, Kp, Vp, None)
        f = np.isin(ids, inputs.SEP_IDS)
        _check(Q, K, V, Kp, Vp, [orc.mask_matrix(f[b], 0, 3) for b in range(B)], [P] * B, [L] * B, O, LSE,
               heads=[0, 1, 77, Hq - 1])


@pytest.mark.parametrize("P", [900, 9000])
def test_repeated_calls_without_waiting_use_one_workspace(P):
    """Calls of different prefix lengths back to back on one workspace: each gives what it gives alone."""
    g = torch.Generator(device="cuda").manual_seed(15)
    B, Hq, Hkv, d, L = 2, 8, 2, 128, 300
    ids = inputs.token_ids(11, B, L, 0.1)
    idesc, index = _index(ids, 32, 0)
    Q, K, V = _normal(g, B, Hq, L, d), _normal(g, B, Hkv, L, d), _normal(g, B, Hkv, L, d)
    Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    plens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([P, 10], [0, 0], [333, P], [128, 129])]
    want = [_run(Q, K, V, idesc, index, Kp, Vp, p) for p in plens]
    desc = api.AttnDesc(B, Hq, Hkv, d, L, 0.0, 0)
    ws = api.alloc_bytes(api.sepllm_attn_prefix_workspace_bytes(desc, idesc, P))
    outs = [(torch.empty_like(Q), torch.empty((B, Hq, L), device="cuda")) for _ in plens]
    for _ in range(10):
        for p, (O, LSE) in zip(plens, outs):
            api.sepllm_attn_prefix_fwd(desc, idesc, P, Q, K, V, index, Kp, Vp, p, O, LSE, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) for a, b in zip(outs, want))


@pytest.mark.parametrize("P", [77, 9001])
def test_initial_tokens_of_their_own_and_a_scale(P):
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = inputs.token_ids(3, 2, 150, 0.1)
    idesc, index = _index(ids, 10, a=4)
    Q, K, V = _normal(g, 2, 4, 150, 64), _normal(g, 2, 2, 150, 64), _normal(g, 2, 2, 150, 64)
    Kp, Vp = _normal(g, 2, P, 64), _normal(g, 2, P, 64)
    O, LSE = _run(Q, K, V, idesc, index, Kp, Vp, None, 0.2)
    f = np.isin(ids, inputs.SEP_IDS)
    _check(Q, K, V, Kp, Vp, [orc.mask_matrix(f[b], 4, 10) for b in range(2)], [P, P], [150, 150], O, LSE,
           scale=float(np.float32(0.2)))


@pytest.mark.parametrize("P", [200, 9000])
def test_rows_that_pack_documents_all_continue_the_prefix(P):
    g = torch.Generator(device="cuda").manual_seed(2)
    B, L, n, a = 2, 300, 16, 2
    ids, df = inputs.token_ids(4, B, L, 0.1), inputs.doc_first(4, B, L, 70.0)
    idesc, index = _index(ids, n, a, doc_first=df)
    Q, K, V = _normal(g, B, 4, L, 128), _normal(g, B, 1, L, 128), _normal(g, B, 1, L, 128)
    Kp, Vp = _normal(g, 1, P, 128), _normal(g, 1, P, 128)
    O, LSE = _run(Q, K, V, idesc, index, Kp, Vp, torch.tensor([P, 50], dtype=torch.int32, device="cuda"))
    f = np.isin(ids, inputs.SEP_IDS)
    _check(Q, K, V, Kp, Vp, [orc.packed_mask_matrix(f[b], df[b], a, n) for b in range(B)], [P, 50], [L, L], O, LSE)


@pytest.mark.parametrize("P", [90, 20000])
def test_no_prefix_in_sight_is_the_plain_forward(P):
    g = torch.Generator(device="cuda").manual_seed(3)
    for B, Hq, Hkv, d, L in ((2, 4, 2, 64, 200), (1, 8, 2, 128, 300)):
        ids = inputs.token_ids(5, B, L, 0.1)
        idesc, index = _index(ids, 20, 3)
        Q, K, V = _normal(g, B, Hq, L, d), _normal(g, B, Hkv, L, d), _normal(g, B, Hkv, L, d)
        Kp = torch.full((Hkv, P, d), float("nan"), dtype=BF, device="cuda")
        O, LSE = _run(Q, K, V, idesc, index, Kp, Kp, torch.zeros(B, dtype=torch.int32, device="cuda"))
        desc = api.AttnDesc(B, Hq, Hkv, d, L, 0.0, 0)
        ws = api.alloc_bytes(api.sepllm_attn_workspace_bytes(desc, idesc)[0])
        O2, LSE2 = torch.empty_like(O), torch.empty_like(LSE)
        api.sepllm_attn_fwd(desc, idesc, Q, K, V, index, O2, LSE2, ws)
        torch.cuda.synchronize()
        # the same 32-bit result; the join scales it by a quotient of two equal numbers
        assert (O.float() - O2.float()).abs().max() <= 2.0 ** -7 * O2.float().abs().max()
        assert (LSE - LSE2).abs().max() <= 1e-5


@pytest.mark.parametrize("P", [400, 9000])
def test_graph_and_other_stream_and_ignored_side_flag(P):
    g = torch.Generator(device="cuda").manual_seed(4)
    B, Hq, Hkv, d, L = 2, 8, 2, 128, 150
    ids = inputs.token_ids(6, B, L, 0.1)
    idesc, index = _index(ids, 20, 0)
    Q, K, V = _normal(g, B, Hq, L, d), _normal(g, B, Hkv, L, d), _normal(g, B, Hkv, L, d)
    Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    want = _run(Q, K, V, idesc, index, Kp, Vp, None)
    desc = api.AttnDesc(B, Hq, Hkv, d, L, 0.0, 0)
    ws = api.alloc_bytes(api.sepllm_attn_prefix_workspace_bytes(desc, idesc, P))
    outs = [(torch.zeros_like(want[0]), torch.zeros_like(want[1])) for _ in range(3)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        api.sepllm_attn_prefix_fwd(desc, idesc, P, Q, K, V, index, Kp, Vp, None, *outs[0], ws)
    torch.cuda.current_stream().wait_stream(s)
    ws.fill_(0xff)
    desc.flags = api.SIDE_READY      # not looked at: the call gathers its side rows
    api.sepllm_attn_prefix_fwd(desc, idesc, P, Q, K, V, index, Kp, Vp, None, *outs[1], ws)
    desc.flags = 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.sepllm_attn_prefix_fwd(desc, idesc, P, Q, K, V, index, Kp, Vp, None, *outs[2], ws)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[0]) and torch.equal(l, want[1]) for o, l in outs)


@pytest.mark.parametrize("Hq,Hkv,d,rot,layout", [(4, 2, 64, 32, "interleaved"), (8, 2, 128, 128, "half")])
def test_a_serving_run_through_a_shared_prefix(Hq, Hkv, d, rot, layout):
    """Prompt -> rotation -> forward -> its retained entries become the shared prefix; every sequence's own
    turn is rotated to the positions behind the prompt, pre-filled behind the prefix and handed to its
    cache; then tokens are generated over prefix and cache.  Every step against the oracle, from the
    keys and values as the rotation left them."""
    g = torch.Generator(device="cuda").manual_seed(5)
    Lp, B, L, steps, a, s, w, c, n = 700, 3, 90, 12, 4, 200, 24, 260, 24
    sep = inputs.SEP_IDS

    def rotate(qkv, pos, first=0):
        b, l = qkv.shape[:2]
        desc = api.RopeDesc(b, l, Hq, Hkv, d, rot_dim=rot, layout=layout, scaling="llama3", base=500000.0,
                            factor=8.0, pos_first=first)
        out = [torch.empty((b, h, l, d), dtype=BF, device="cuda") for h in (Hq, Hkv, Hkv)]
        api.sepllm_rope_fwd(desc, pos, *qkv.transpose(1, 2).split((Hq, Hkv, Hkv), 1), *out)
        return out
    # the shared prompt
    pids = inputs.token_ids(40, 1, Lp, 0.12)
    Qs, Ks, Vs = rotate(_normal(g, 1, Lp, Hq + 2 * Hkv, d), None)
    idesc1, index1 = _index(pids, n, a)
    one = GpuCache(1, Hkv, Hq, d, a, s, w, c)
    api.sepllm_cache_from_prompt(one.desc, idesc1, index1, None, Ks, Vs, one.state, one.Kc, one.Vc)
    Kp, Vp = (torch.full((Hkv, c, d), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    plen = torch.zeros(B, dtype=torch.int32, device="cuda")
    api.sepllm_prefix_from_cache(one.desc, one.state, one.Kc, one.Vc, c, Kp, Vp, plen)
    kept = orc.cache_after_prompt(np.isin(pids[0], sep).tolist(), a, s, w, c).retained()
    R = len(kept)
    torch.cuda.synchronize()
    assert plen.tolist() == [R] * B
    for x, y in ((Kp, Ks), (Vp, Vs)):
        assert torch.equal(x[:, :R], y[0][:, kept])
    # the sequences' own turns, of unequal lengths
    ids = inputs.token_ids(41, B, L + steps, 0.12)
    f = np.isin(ids, sep)
    lens = [L, 37, 1]
    qkv = _normal(g, B, L + steps, Hq + 2 * Hkv, d)
    Q, K, V = rotate(qkv[:, :L].contiguous(), None, first=Lp)
    idesc, index = _index(ids[:, :L], n, 0, lens)
    O, LSE = _run(Q, K, V, idesc, index, Kp, Vp, plen)
    _check(Q, K, V, Kp, Vp, [orc.mask_matrix(f[b, :L], 0, n) for b in range(B)], [R] * B, lens, O, LSE)
    own = GpuCache(B, Hkv, Hq, d, 0, s, w, c)
    lens_d = torch.tensor(lens, dtype=torch.int32, device="cuda")
    api.sepllm_cache_from_prompt(own.desc, idesc, index, lens_d, K, V, own.state, own.Kc, own.Vc)
    # generation: sequence b's t-th token has position Lp + lens[b] + t
    ws = api.alloc_bytes(api.sepllm_decode_prefix_workspace_bytes(own.desc, c))
    hist = [([K[b, :, j] for j in range(lens[b])], [V[b, :, j] for j in range(lens[b])]) for b in range(B)]
    oc = [orc.cache_after_prompt(f[b, :lens[b]].tolist(), 0, s, w, c) for b in range(B)]
    o = torch.empty((B, Hq, d), dtype=BF, device="cuda")
    lse = torch.empty((B, Hq), dtype=torch.float32, device="cuda")
    rows = torch.arange(B, device="cuda")
    for t in range(steps):
        pos = (lens_d.long() + Lp + t)[:, None].contiguous()
        q, k, v = rotate(qkv[rows, lens_d.long() + t][:, None].contiguous(), pos)
        tok = torch.from_numpy(ids)[np.arange(B), np.array(lens) + t].to(torch.int32).cuda()
        api.sepllm_cache_update(own.desc, own.state, own.Kc, own.Vc, tok, sep, k[:, :, 0].contiguous(),
                                v[:, :, 0].contiguous())
        q0 = q[:, :, 0].contiguous()
        api.sepllm_decode_prefix(own.desc, c, 0.0, q0, own.state, own.Kc, own.Vc, Kp, Vp, plen, o, lse, ws)
        torch.cuda.synchronize()
        assert api.sepllm_last_device_status(ws) == 0
        for b in range(B):
            hist[b][0].append(k[b, :, 0])
            hist[b][1].append(v[b, :, 0])
            oc[b].update(bool(f[b, lens[b] + t]))
            kk, vv = (torch.cat((x[:, :R], torch.stack([hist[b][i][j] for j in oc[b].retained()], 1)), 1)
                      .double().cpu().numpy() for i, x in ((0, Kp), (1, Vp)))
            for h in range(Hq):
                ref, lref = orc.decode_attention(q0[b, h].double().cpu().numpy(), kk[h // (Hq // Hkv)],
                                                 vv[h // (Hq // Hkv)])
                assert np.abs(o[b, h].double().cpu().numpy() - ref).max() <= TOL_O["max_abs"], (t, b, h)
                assert abs(float(lse[b, h]) - lref) <= TOL_LSE


def test_packed_rows_with_many_documents_in_the_direct_form():
    """Side tiles of earlier documents lie between the prefix and a row's own side entries."""
    g = torch.Generator(device="cuda").manual_seed(16)
    for Hq, Hkv, d, L, P, mean in ((4, 1, 128, 900, 130, 120.0), (2, 2, 64, 1100, 256, 60.0), (3, 1, 80, 700, 1, 300.0)):
        ids, df = inputs.token_ids(17, 1, L, 0.5), inputs.doc_first(17, 1, L, mean)
        idesc, index = _index(ids, 16, 3, doc_first=df)
        Q, K, V = _normal(g, 1, Hq, L, d), _normal(g, 1, Hkv, L, d), _normal(g, 1, Hkv, L, d)
        Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
        O, LSE = _run(Q, K, V, idesc, index, Kp, Vp, None)
        f = np.isin(ids, inputs.SEP_IDS)
        _check(Q, K, V, Kp, Vp, [orc.packed_mask_matrix(f[0], df[0], 3, 16)], [P], [L], O, LSE)


def test_two_streams_at_once():
    """Pre-filling on one stream and decoding on another, each in its own workspace, both forms of each."""
    g = torch.Generator(device="cuda").manual_seed(18)
    Hq, Hkv, d, L, B = 8, 2, 128, 200, 3
    ids = inputs.token_ids(18, B, L, 0.1)
    idesc, index = _index(ids, 24, 0)
    Q, K, V = _normal(g, B, Hq, L, d), _normal(g, B, Hkv, L, d), _normal(g, B, Hkv, L, d)
    desc = api.AttnDesc(B, Hq, Hkv, d, L, 0.0, 0)
    cd = api.CacheDesc(48, Hkv, Hq, d, 0, 4, 3, 16)
    state = api.alloc_bytes(api.sepllm_cache_bytes(cd)[0])
    api.sepllm_cache_init(cd, state)
    Kc = torch.zeros((48, Hkv, 20, d), dtype=BF, device="cuda")
    q = _normal(g, 48, Hq, d)
    jobs = []
    for P in (200, 7000):
        Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
        for _ in range(2):
            wa = api.alloc_bytes(api.sepllm_attn_prefix_workspace_bytes(desc, idesc, P))
            wd = api.alloc_bytes(api.sepllm_decode_prefix_workspace_bytes(cd, P))
            out = (torch.empty_like(Q), torch.empty((B, Hq, L), device="cuda"), torch.empty_like(q),
                   torch.empty((48, Hq), device="cuda"))
            jobs.append((P, Kp, Vp, wa, wd, out))

    def attn(j):
        api.sepllm_attn_prefix_fwd(desc, idesc, j[0], Q, K, V, index, j[1], j[2], None, *j[5][:2], j[3])

    def dec(j):
        api.sepllm_decode_prefix(cd, j[0], 0.0, q, state, Kc, Kc, j[1], j[2], None, *j[5][2:], j[4])
    for j in jobs[::2]:      # one after the other
        attn(j), dec(j)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        with torch.cuda.stream(s1):
            for j in jobs[1::2]:
                attn(j)
        with torch.cuda.stream(s2):
            for j in jobs[1::2]:
                dec(j)
    torch.cuda.synchronize()
    for a, b in zip(jobs[::2], jobs[1::2]):
        assert all(torch.equal(x, y) for x, y in zip(a[5], b[5]))
        assert api.sepllm_last_device_status(b[3]) == 0 and api.sepllm_last_device_status(b[4]) == 0


@pytest.mark.parametrize("P", [200, 9000])
def test_events_between_the_launches(P):
    """The descriptor's events are recorded as by the plain forward; the results stay what they are."""
    g = torch.Generator(device="cuda").manual_seed(19)
    B, Hq, Hkv, d, L = 2, 4, 1, 128, 150
    ids = inputs.token_ids(19, B, L, 0.1)
    idesc, index = _index(ids, 24, 0)
    Q, K, V = _normal(g, B, Hq, L, d), _normal(g, B, Hkv, L, d), _normal(g, B, Hkv, L, d)
    Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    want = _run(Q, K, V, idesc, index, Kp, Vp, None)
    desc = api.AttnDesc(B, Hq, Hkv, d, L, 0.0, 0)
    events = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    for e in events:
        e.record()
    desc.set_events(events)
    ws = api.alloc_bytes(api.sepllm_attn_prefix_workspace_bytes(desc, idesc, P))
    O, LSE = torch.empty_like(Q), torch.empty((B, Hq, L), device="cuda")
    for _ in range(3):
        api.sepllm_attn_prefix_fwd(desc, idesc, P, Q, K, V, index, Kp, Vp, None, O, LSE, ws)
    torch.cuda.synchronize()
    assert torch.equal(O, want[0]) and torch.equal(LSE, want[1])
    assert events[0].elapsed_time(events[1]) > 0 and events[1].elapsed_time(events[2]) > 0


@pytest.mark.parametrize("P,B,L", [(300, 3, 200), (6000, 3, 200), (50, 2, 1)])
def test_a_batch_of_padding_alone_writes_nothing(P, B, L):
    g = torch.Generator(device="cuda").manual_seed(20)
    ids = inputs.token_ids(20, B, L, 0.1)
    idesc, index = _index(ids, 24, 0, [0] * B)
    Q, K, V = _normal(g, B, 4, L, 128), _normal(g, B, 1, L, 128), _normal(g, B, 1, L, 128)
    Kp, Vp = _normal(g, 1, P, 128), _normal(g, 1, P, 128)
    O, LSE = _run(Q, K, V, idesc, index, Kp, Vp, None)
    assert (O == 3.5).all() and (LSE == -2.5).all()
