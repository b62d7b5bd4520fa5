"""sepllm_prefix_from_cache / sepllm_decode_prefix against the oracle's softmax over the joined keys."""
import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, inputs
from tests._gpu_util import TOL_LSE, TOL_O

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(BF)


class Cache:
    """Caches of given sizes with ring starts anywhere, written straight into the state buffer."""

    def __init__(self, g, B, Hkv, Hq, d, a, s, w, c, runs):
        self.desc = api.CacheDesc(B, Hkv, Hq, d, a, s, w, c)
        sb, kv = api.sepllm_cache_bytes(self.desc)
        self.state = api.alloc_bytes(sb)
        api.sepllm_cache_init(self.desc, self.state)
        self.Kc, self.Vc = _normal(g, B, Hkv, c + s, d), _normal(g, B, Hkv, c + s, d)
        rng = np.random.default_rng(int(torch.randint(0, 1 << 30, (1,), generator=g, device="cuda")))
        seq = self.state[256:256 + 64 * B].view(torch.int32).view(B, 16)
        self.slots = []
        for b, run in enumerate(runs):
            i = min(run, a)
            q = min(s, (run - i) // 2) if run - i > w else 0
            n = run - i - q
            s0, w0 = int(rng.integers(0, max(s, 1))), int(rng.integers(0, c - a))
            seq[b, :5] = torch.tensor([i, s0, q, w0, n], dtype=torch.int32)
            self.slots.append(list(range(i)) + [a + (s0 + k) % s for k in range(q)]
                              + [a + s + (w0 + k) % (c - a) for k in range(n)])


def _check_decode(cache, q, Kp, Vp, plen, o, lse, scale=None, rows=None):
    """Every (sequence, head) against the 64-bit softmax.  Beside the common bounds of a bf16 output
    an entry gets what its terms cost: the weights are rounded to bf16 (2^-8 at most, 2^-9 / sqrt(3)
    at rms) before the second product, five deviations of the terms' root sum of squares."""
    d = cache.desc
    G = d.Hq // d.Hkv
    kp, vp = Kp.double().cpu().numpy(), Vp.double().cpu().numpy()
    kc, vc = cache.Kc.double().cpu().numpy(), cache.Vc.double().cpu().numpy()
    qn, on, ln = q.double().cpu().numpy(), o.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, h in (rows or [(b, h) for b in range(d.B) for h in range(d.Hq)]):
        hk, n = h // G, plen[b]
        k = np.concatenate((kp[hk, :n], kc[b, hk][cache.slots[b]]))
        v = np.concatenate((vp[hk, :n], vc[b, hk][cache.slots[b]]))
        if not len(k):
            assert (on[b, h] == 0).all() and ln[b, h] == -np.inf
            continue
        ref, lref = orc.decode_attention(qn[b, h], k, v, scale)
        s = k @ qn[b, h] * (scale or 1 / np.sqrt(d.d))
        rss = np.sqrt(((np.exp(s - lref)[:, None] * v) ** 2).sum(0))
        tol = np.maximum(TOL_O["max_abs"], 5 * 2.0 ** -9 * rss + 2.0 ** -8 * np.abs(ref))
        assert (np.abs(on[b, h] - ref) <= tol).all(), (b, h, np.abs(on[b, h] - ref).max())
        # relative: 2^-9 / sqrt(3) of the weights' rounding and as much of the output's, doubled
        assert np.linalg.norm(on[b, h] - ref) <= TOL_O["rel_fro"] * max(np.linalg.norm(ref), np.linalg.norm(rss)), (b, h)
        assert abs(ln[b, h] - lref) <= TOL_LSE, (b, h)


def _decode(cache, P, q, Kp, Vp, plen, scale=0.0):
    d = cache.desc
    o = torch.full((d.B, d.Hq, d.d), float("nan"), dtype=BF, device="cuda")
    lse = torch.full((d.B, d.Hq), float("nan"), dtype=torch.float32, device="cuda")
    ws = api.alloc_bytes(api.sepllm_decode_prefix_workspace_bytes(d, P))
    ws.fill_(0xff)   # whatever an earlier call left
    api.sepllm_decode_prefix(d, P, scale, q, cache.state, cache.Kc, cache.Vc, Kp, Vp, plen, o, lse, ws)
    torch.cuda.synchronize()
    assert api.sepllm_last_device_status(ws) == 0
    return o, lse


SHAPES = [
    # B, Hkv, Hq, d, P
    (1, 1, 1, 64, 1), (1, 1, 1, 128, 127), (2, 2, 4, 64, 128), (3, 1, 4, 128, 129), (5, 3, 3, 64, 1000),
    (1, 2, 32, 128, 257), (9, 2, 30, 64, 640), (33, 1, 4, 128, 300), (130, 1, 2, 64, 513), (1, 8, 32, 128, 5001),
    # a prefix long enough, or read by enough sequences, for the kernel that shares it
    (30, 1, 4, 128, 9000), (9, 2, 30, 64, 30000), (128, 1, 1, 64, 4001), (33, 1, 4, 128, 8191), (130, 1, 2, 64, 4100),
    (70, 2, 8, 128, 2050), (300, 1, 1, 64, 1920), (64, 2, 24, 128, 1999), (3, 12, 12, 64, 20011), (40, 4, 64, 128, 1500),
]


@pytest.mark.parametrize("B,Hkv,Hq,d,P", SHAPES)
def test_decode_of_ragged_batches(B, Hkv, Hq, d, P):
    """Prefix lengths from none to all, caches from empty to nearly full, sequences without any key."""
    g = torch.Generator(device="cuda").manual_seed(B + Hq + P)
    a, s, w, c = 2, 6, 5, 40
    rng = np.random.default_rng(B * P)
    runs = rng.integers(0, c, B)
    plen = rng.integers(0, P + 1, B)
    plen[0], runs[-1] = P, c - 1
    if B > 2:
        plen[1] = runs[1] = 0
        plen[2], runs[2] = 0, 3
    cache = Cache(g, B, Hkv, Hq, d, a, s, w, c, runs.tolist())
    q = (torch.randn((B, Hq, d), generator=g, device="cuda") * 2).to(BF)
    Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    # values outside [0, P] are clamped
    pl = torch.from_numpy(plen.astype(np.int32)).cuda()
    pl[0] = P + 1000
    if B > 2:
        pl[1] = -7
    o, lse = _decode(cache, P, q, Kp, Vp, pl)
    some = [(b, h) for b in range(B) for h in range(Hq)]
    some = some if len(some) <= 400 else [some[i] for i in rng.choice(len(some), 400, replace=False)] + some[:3 * Hq]
    _check_decode(cache, q, Kp, Vp, plen, o, lse, rows=some)


@pytest.mark.parametrize("B,P", [(3, 900), (40, 900), (12, 9001), (120, 2900)])
def test_whole_prefix_without_lengths_and_a_scale(B, P):
    g = torch.Generator(device="cuda").manual_seed(3)
    cache = Cache(g, B, 2, 8, 128, 1, 4, 3, 20, [b % 20 for b in range(B)])
    q, Kp, Vp = _normal(g, B, 8, 128), _normal(g, 2, P, 128), _normal(g, 2, P, 128)
    o, lse = _decode(cache, P, q, Kp, Vp, None, 0.31)
    _check_decode(cache, q, Kp, Vp, [P] * B, o, lse, scale=float(np.float32(0.31)))
    o2, lse2 = _decode(cache, P, q, Kp, Vp, torch.full((B,), P, dtype=torch.int32, device="cuda"), 0.31)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_rows_behind_the_longest_prefix_may_hold_anything():
    g = torch.Generator(device="cuda").manual_seed(4)
    for B, P, n in ((4, 1000, 300), (4, 1000, 384), (80, 700, 1), (4, 130, 0), (80, 9000, 5000), (80, 9000, 5120),
                    (12, 40000, 39999), (200, 4000, 0)):
        cache = Cache(g, B, 1, 4, 64, 2, 4, 3, 20, [7] * B)
        q, Kp, Vp = _normal(g, B, 4, 64), _normal(g, 1, P, 64), _normal(g, 1, P, 64)
        plen = torch.randint(0, n + 1, (B,), generator=g, device="cuda").to(torch.int32)
        plen[1] = n
        o, lse = _decode(cache, P, q, Kp, Vp, plen)
        Kp[:, n:], Vp[:, n:] = float("nan"), float("inf")
        Kp[:, n + 1:] = float("-inf")
        o2, lse2 = _decode(cache, P, q, Kp, Vp, plen)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_equals_decode_of_caches_that_carry_the_prefix_themselves():
    """The same entries once shared and once in every sequence's own cache."""
    g = torch.Generator(device="cuda").manual_seed(5)
    B, Hkv, Hq, d, P = 6, 2, 8, 128, 700
    big = Cache(g, B, Hkv, Hq, d, P, 8, 8, P + 64, [P + 40] * B)
    small = Cache(g, B, Hkv, Hq, d, 0, 8, 8, 64, [40] * B)
    Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    big.Kc[:, :, :P], big.Vc[:, :, :P] = Kp, Vp
    for b in range(B):
        big.Kc[b, :, big.slots[b][P:]] = small.Kc[b, :, small.slots[b]]
        big.Vc[b, :, big.slots[b][P:]] = small.Vc[b, :, small.slots[b]]
    q = _normal(g, B, Hq, d)
    o, lse = _decode(small, P, q, Kp, Vp, None)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    ws = api.alloc_bytes(api.sepllm_decode_workspace_bytes(big.desc))
    api.sepllm_decode(big.desc, 0.0, q, big.state, big.Kc, big.Vc, o2, lse2, ws)
    torch.cuda.synchronize()
    assert (lse - lse2).abs().max() <= TOL_LSE and (o.float() - o2.float()).abs().max() <= 2 * TOL_O["max_abs"]


@pytest.mark.parametrize("Hkv,Hq,B,P", [(400, 400, 2, 3), (1, 16, 2600, 140), (200, 200, 300, 130), (1, 16, 2600, 300), (400, 400, 9, 150)])
def test_more_units_than_sms(Hkv, Hq, B, P):
    """Many kv heads, or so many sequences that one kv head has more row tiles than a launch takes:
    units that one CTA walks in full leave parts of their own."""
    g = torch.Generator(device="cuda").manual_seed(Hkv)
    rng = np.random.default_rng(Hkv)
    runs, plen = rng.integers(0, 12, B), rng.integers(0, P + 1, B)
    cache = Cache(g, B, Hkv, Hq, 64, 0, 3, 2, 12, runs.tolist())
    q, Kp, Vp = _normal(g, B, Hq, 64), _normal(g, Hkv, P, 64), _normal(g, Hkv, P, 64)
    o, lse = _decode(cache, P, q, Kp, Vp, torch.from_numpy(plen.astype(np.int32)).cuda())
    rows = [(int(rng.integers(0, B)), int(rng.integers(0, Hq))) for _ in range(150)] + [(B - 1, Hq - 1), (0, 0)]
    _check_decode(cache, q, Kp, Vp, plen, o, lse, rows=rows)


@pytest.mark.parametrize("P", [300, 30000])
def test_non_finite_inputs_reach_the_rows_that_see_them_and_no_others(P):
    g = torch.Generator(device="cuda").manual_seed(10)
    B, Hkv, Hq, d = 5, 2, 4, 64
    cache = Cache(g, B, Hkv, Hq, d, 0, 4, 3, 20, [7, 0, 5, 0, 9])
    q, Kp, Vp = _normal(g, B, Hq, d), _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    plen = torch.tensor([P, P, 0, 0, 129], dtype=torch.int32, device="cuda")
    want = _decode(cache, P, q, Kp, Vp, plen)
    q2 = q.clone()
    q2[0, 1] = float("nan")      # a query that sees both parts, one the prefix alone, one its cache alone
    q2[1, 2, 5] = float("nan")
    q2[2, 0, 7] = float("inf")
    o, lse = _decode(cache, P, q2, Kp, Vp, plen)
    hit = torch.zeros((B, Hq), dtype=torch.bool, device="cuda")
    hit[0, 1] = hit[1, 2] = hit[2, 0] = True
    assert torch.isnan(o[hit]).all() and torch.isnan(lse[0, 1]) and torch.isnan(lse[1, 2])
    assert torch.equal(o[~hit], want[0][~hit]) and torch.equal(lse[~hit], want[1][~hit])
    Kp[1, 200] = float("nan")    # a key that the first two sequences see, and heads 2 and 3 only
    o, lse = _decode(cache, P, q, Kp, Vp, plen)
    assert torch.isnan(o[:2, 2:]).all() and torch.isnan(lse[:2, 2:]).all()
    assert torch.equal(o[2:], want[0][2:]) and torch.equal(o[:2, :2], want[0][:2, :2])


@pytest.mark.parametrize("P", [600, 4000])
def test_back_to_back_calls_on_one_workspace(P):
    """Update, decode, update, decode without waiting in between, the caches' sizes and the prefix
    lengths changing: each decode gives what it gives when waited for."""
    g = torch.Generator(device="cuda").manual_seed(9)
    B, Hkv, Hq, d, steps = 40, 2, 8, 128, 12
    Kp, Vp = _normal(g, Hkv, P, d), _normal(g, Hkv, P, d)
    k, v, q = _normal(g, steps, B, Hkv, d), _normal(g, steps, B, Hkv, d), _normal(g, steps, B, Hq, d)
    ids = torch.from_numpy(inputs.decode_stream_ids(9, B, steps, 0.3).T.copy()).cuda()
    plen = torch.randint(0, P + 1, (steps, B), generator=g, device="cuda").to(torch.int32)
    outs = []
    for wait in (True, False):
        cache = Cache(g, B, Hkv, Hq, d, 1, 4, 3, 10, [0] * B)
        desc = cache.desc
        cache.Kc.zero_(), cache.Vc.zero_()
        ws = api.alloc_bytes(api.sepllm_decode_prefix_workspace_bytes(desc, P))
        o, lse = torch.empty((steps, B, Hq, d), dtype=BF, device="cuda"), torch.empty((steps, B, Hq), device="cuda")
        api.sepllm_cache_init(desc, cache.state)
        for t in range(steps):
            api.sepllm_cache_update(desc, cache.state, cache.Kc, cache.Vc, ids[t], inputs.SEP_IDS, k[t], v[t])
            api.sepllm_decode_prefix(desc, P, 0.0, q[t], cache.state, cache.Kc, cache.Vc, Kp, Vp, plen[t], o[t], lse[t], ws)
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        outs.append((o, lse))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("B,P", [(3, 2000), (100, 6000)])
def test_sharp_scores_and_growing_maxima(B, P):
    """Scores of many hundreds, rising along the prefix, so that the reference exponent moves often."""
    g = torch.Generator(device="cuda").manual_seed(6)
    d = 64
    cache = Cache(g, B, 1, 2, d, 0, 4, 3, 20, [0, 5, 19] + [1] * (B - 3))
    q = torch.ones((B, 2, d), device="cuda", dtype=BF)
    q[1] = -1
    ramp = torch.linspace(-30, 30, P, device="cuda")[None, :, None].expand(1, P, d)
    Kp = (ramp + 0.01 * torch.randn((1, P, d), generator=g, device="cuda")).to(BF)
    Vp = _normal(g, 1, P, d)
    o, lse = _decode(cache, P, q, Kp, Vp, None)
    kp, vp = Kp.double().cpu().numpy()[0], Vp.double().cpu().numpy()[0]
    for b in range(3):
        k = np.concatenate((kp, cache.Kc[b, 0].double().cpu().numpy()[cache.slots[b]]))
        v = np.concatenate((vp, cache.Vc[b, 0].double().cpu().numpy()[cache.slots[b]]))
        ref, lref = orc.decode_attention(q[b, 0].double().cpu().numpy(), k, v)
        # scores reach 240: 2^-24 of that, times a few operations, is 1e-4 on a score and on each weight
        assert abs(float(lse[b, 0]) - lref) <= TOL_LSE
        assert np.abs(o[b, 0].double().cpu().numpy() - ref).max() <= 2.0 ** -8 * np.abs(v).max() + TOL_O["max_abs"]


@pytest.mark.parametrize("B,P", [(6, 500), (60, 5000)])
def test_other_stream_graph_and_shared_workspace(B, P):
    g = torch.Generator(device="cuda").manual_seed(7)
    cache = Cache(g, B, 2, 8, 64, 2, 6, 5, 40, [30] * B)
    q, Kp, Vp = _normal(g, B, 8, 64), _normal(g, 2, P, 64), _normal(g, 2, P, 64)
    plen = torch.full((B,), P, dtype=torch.int32, device="cuda")
    want = _decode(cache, P, q, Kp, Vp, plen)
    d = cache.desc
    ws = api.alloc_bytes(api.sepllm_decode_prefix_workspace_bytes(d, P))
    outs = [(torch.zeros_like(want[0]), torch.zeros_like(want[1])) for _ in range(3)]

    def call(i):
        api.sepllm_decode_prefix(d, P, 0.0, q, cache.state, cache.Kc, cache.Vc, Kp, Vp, plen, *outs[i], ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(0)
    torch.cuda.current_stream().wait_stream(s)
    graphs = []
    for i in (1, 2):     # two graphs share the workspace and are replayed one after the other
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(i)
    for _ in range(2):
        for gr in graphs:
            gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[0]) and torch.equal(l, want[1]) for o, l in outs)
    plen.fill_(77)       # a replay reads the lengths of its time
    want = _decode(cache, P, q, Kp, Vp, plen)
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[1][0], want[0]) and torch.equal(outs[1][1], want[1])


@pytest.mark.parametrize("Hkv,d,a,s,w,c,run,P", [(1, 64, 0, 0, 1, 2, 1, 2), (2, 64, 2, 6, 5, 40, 39, 40), (3, 128, 4, 16, 8, 60, 3, 64),
                                                 (2, 128, 2, 6, 5, 40, 0, 45), (8, 128, 4, 1024, 256, 2000, 1999, 2100)])
def test_prefix_from_cache(Hkv, d, a, s, w, c, run, P):
    g = torch.Generator(device="cuda").manual_seed(run)
    cache = Cache(g, 1, Hkv, Hkv, d, a, s, w, c, [run])
    Kp, Vp = torch.full((Hkv, P, d), 7.0, dtype=BF, device="cuda"), torch.full((Hkv, P, d), 8.0, dtype=BF, device="cuda")
    n = torch.full((300,), -1, dtype=torch.int32, device="cuda")
    api.sepllm_prefix_from_cache(cache.desc, cache.state, cache.Kc, cache.Vc, P, Kp, Vp, n)
    torch.cuda.synchronize()
    assert (n == run).all()
    for x, src, fill in ((Kp, cache.Kc, 7.0), (Vp, cache.Vc, 8.0)):
        assert torch.equal(x[:, :run], src[0][:, cache.slots[0]])
        assert (x[:, run:] == fill).all()


def test_largest_batches_of_one_head_and_far_rows():
    """A prefix block of more than 2^31 elements, read near its end."""
    g = torch.Generator(device="cuda").manual_seed(8)
    B, Hkv, d = 2, 2, 128
    P = 2 ** 23 + 300          # Hkv * P * d > 2^31
    cache = Cache(g, B, Hkv, Hkv, d, 0, 4, 3, 20, [4, 0])
    Kp = torch.zeros((Hkv, P, d), dtype=BF, device="cuda")
    Vp = torch.zeros((Hkv, P, d), dtype=BF, device="cuda")
    q = torch.ones((B, Hkv, d), dtype=BF, device="cuda")
    Kp[:, P - 1] = 4.0                                   # score 45: all the weight
    Vp[:, P - 1] = torch.arange(d, device="cuda").to(BF)
    o, lse = _decode(cache, P, q, Kp, Vp, None)
    assert torch.equal(o[1], Vp[:, P - 1]) and (lse[1] - 4 * 128 / 128 ** 0.5).abs().max() <= 1e-2
