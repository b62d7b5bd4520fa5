"""Cases, plain forms and exact values of the rotary and shared-prefix operators.

Operators: rotary positions on the outputs of a fused Q/K/V projection and their gradient
(`sepllm_rope_fwd`, `sepllm_rope_bwd`), decode of one token per sequence over a prefix that the
whole batch shares plus each sequence's own cache (`sepllm_decode_prefix`), pre-filling of the
sequences' own tokens behind such a prefix (`sepllm_attn_prefix_fwd`), and the copy of one
sequence's retained cache entries into the shared prefix (`sepllm_prefix_from_cache`).

`own` false: the operators written out in elementary torch operations in 32 bits.  `own` true:
the calls that a program makes of the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
SEP_IDS = [11, 13, 29, 101, 1027, 2048, 4099, 17000, 49999]


# ------------------------------------------------------------------------------------------ cases
def _rope(name, op, B, L, Hq, Hkv, d, rot, layout, scaling="none", base=10000.0, factor=1.0, low=1.0,
          high=4.0, orig=8192.0, far=0, grad="bf16"):
    c = dict(op=op, B=B, L=L, Hq=Hq, Hkv=Hkv, d=d, rot=rot, layout=layout, scaling=scaling, base=base,
             factor=factor, low=low, high=high, orig=orig, far=far, grad=grad)
    return dict(c, name=name) if name else c


def _decode(name, B, Hq, Hkv, d, P, plen_lo, a, s, w, c, run_lo, run_hi):
    r = dict(op="decode", B=B, Hq=Hq, Hkv=Hkv, d=d, P=P, plen_lo=plen_lo, a=a, s=s, w=w, c=c, run_lo=run_lo,
             run_hi=run_hi)
    return dict(r, name=name) if name else r


def _attn(name, B, L, Hq, Hkv, d, P, plen_lo, n_neighbor, rho, ragged):
    r = dict(op="attn", B=B, L=L, Hq=Hq, Hkv=Hkv, d=d, P=P, plen_lo=plen_lo, n_neighbor=n_neighbor, rho=rho,
             ragged=ragged)
    return dict(r, name=name) if name else r


def _prefix(name, Hkv, d, a, s, w, c, run, n_len):
    r = dict(op="prefix", Hkv=Hkv, d=d, a=a, s=s, w=w, c=c, run=run, n_len=n_len)
    return dict(r, name=name) if name else r


def listed():
    return [
        # one generated token per sequence of the streaming-decode batch, at positions far into the
        # text: interleaved pairs, frequencies stretched by wavelength.  Latency counts.
        _rope("rope_step", "rope_fwd", 32, 1, 32, 8, 128, 128, "interleaved", "llama3", 500000.0, 8.0, 1.0, 4.0,
              8192.0, 1 << 20),
        # the long-context row of the benchmark, straight from the fused projection
        _rope("rope_long", "rope_fwd", 1, 65536, 32, 8, 128, 128, "half", "yarn", 500000.0, 4.0, 1.0, 32.0, 16384.0),
        # the small pre-training batch: a quarter of every head is rotated
        _rope("rope_partial", "rope_fwd", 8, 2048, 12, 12, 64, 16, "half"),
        # gradients of a training row in 32 bits, back to the projection's layout
        _rope("rope_bwd_long", "rope_bwd", 1, 16384, 32, 8, 128, 128, "half", "none", 500000.0, grad="fp32"),
        # gradients of a ragged batch whose head size is no power of two, linear stretch
        _rope("rope_bwd_odd", "rope_bwd", 3, 1999, 10, 2, 80, 40, "interleaved", "linear", 10000.0, 2.5, far=5000),
        # the streaming-decode batch behind one system prompt of 8192 entries
        _decode("decode_batch", 32, 32, 8, 128, 8192, 8192, 4, 1024, 256, 3332, 2200, 3300),
        # a few sequences of a small model just behind the fork: hardly any entries of their own,
        # some sequences that branch off early, some that do not use the prefix at all
        _decode("decode_forked", 5, 12, 12, 64, 1000, 0, 2, 64, 64, 300, 0, 40),
        # many sequences on one long document, each with a short cache of its own
        _decode("decode_many", 256, 32, 8, 128, 40000, 40000, 4, 128, 256, 800, 64, 790),
        # a short turn of every user behind the shared prompt, lengths ragged
        _attn("attn_turn", 8, 100, 32, 8, 128, 8192, 8192, 256, 0.12, True),
        # long documents pre-filled behind a shared instruction, one of them branching off early
        _attn("attn_docs", 2, 1024, 32, 8, 128, 8199, 4000, 256, 0.10, False),
        # the retained entries of a short prompt and of a long one become the shared prefix
        _prefix("prefix_small", 12, 64, 2, 64, 64, 300, 280, 5),
        _prefix("prefix_long", 8, 128, 4, 8192, 512, 16384, 15001, 256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope_fwd", "rope_bwd", "decode", "decode", "attn", "prefix"])
    if op.startswith("rope"):
        d = rng.choice([64, 80, 96, 112, 128])
        Hkv = rng.choice([1, 2, 4, 8, 12])
        Hq = Hkv * rng.choice([1, 2, 4, 5])
        tokens = _log(rng, 1, (1 << 27) // ((Hq + 2 * Hkv) * d))
        B = min(tokens, _log(rng, 1, 64))
        scaling = rng.choice(["none", "linear", "ntk", "yarn", "llama3", "factors"])
        rot = rng.choice([d, d, d // 2, 2 * rng.randint(2, d // 2)])
        return _rope(None, op, B, max(1, tokens // B), Hq, Hkv, d, rot, rng.choice(["half", "interleaved"]), scaling,
                     rng.choice([10000.0, 500000.0, 1000000.0]), 1.0 if scaling == "none" else rng.uniform(1.5, 16.0),
                     1.0, 32.0 if scaling == "yarn" else 4.0, float(_log(rng, 2048, 32768)),
                     rng.choice([0, _log(rng, 100, 1 << 24)]), rng.choice(["bf16", "fp32"]))
    if op == "decode":
        d = rng.choice([64, 128])
        Hkv = rng.choice([1, 2, 4, 8, 12])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
        B, P = _log(rng, 1, 256), _log(rng, 1, 40000)
        a, s, w = rng.randint(0, 8), rng.choice([0, _log(rng, 1, 1024)]), _log(rng, 1, 512)
        c = a + s + w + _log(rng, 1, 1024)
        while B * Hq * (P + c) > 256 * 32 * 40000 or B * Hkv * c * d > 1 << 28:
            B = (B + 1) // 2
        return _decode(None, B, Hq, Hkv, d, P, rng.choice([0, P // 2, P]), a, s, w, c, rng.choice([0, c // 2]), c - 1)
    if op == "attn":
        d = rng.choice([64, 80, 96, 112, 128])
        Hkv = rng.choice([1, 2, 4, 8])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
        B, L, P = _log(rng, 1, 16), _log(rng, 1, 1024), _log(rng, 1, 8199)
        while B * Hq * L * (P + L) > 2 * 32 * 1024 * (8199 + 1024):
            B, L = (B + 1) // 2, (L + 1) // 2
        return _attn(None, B, L, Hq, Hkv, d, P, rng.choice([0, P // 2, P]), _log(rng, 1, 512), rng.uniform(0.02, 0.3),
                     rng.random() < 0.5)
    d, Hkv = rng.choice([64, 128]), rng.choice([1, 2, 4, 8, 12])
    a, s, w = rng.randint(0, 8), _log(rng, 1, 8192), _log(rng, 1, 1024)
    c = a + s + w + _log(rng, 1, 4096)
    return _prefix(None, Hkv, d, a, s, w, c, rng.randint(1, c - 1), rng.randint(1, 256))


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _int(g, lo, hi, shape):
    """Uniform in [lo, hi], int64."""
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV)


def _queries(g, B, Hq, L, d):
    """Heads from diffuse to sharp, as trained models have them: scores of spread 0.5 to 4."""
    q = torch.randn((B, Hq, L, d), generator=g, device=DEV)
    sharp = torch.rand((1, Hq, 1, 1), generator=g, device=DEV) * 3.5 + 0.5
    return (q * sharp).to(torch.bfloat16)


def _prefix_len(g, c):
    """int32 [B], or None where every sequence sees the whole prefix."""
    if c["plen_lo"] >= c["P"]:
        return None
    n = _int(g, c["plen_lo"], c["P"], (c["B"],)).to(torch.int32)
    n[0] = c["P"]
    return n


def _cache_sizes(g, B, a, s, w, c, lo, hi):
    """Sizes and ring starts of B caches that hold between lo and hi entries."""
    run = _int(g, lo, hi, (B,))
    size_init = run.clamp(max=a)
    rest = run - size_init
    size_sep = torch.where(rest > w, (rest // 2).clamp(max=s), torch.zeros_like(rest))
    return dict(size_init=size_init, size_sep=size_sep, size_win=rest - size_sep,
                sep_start=_int(g, 0, max(0, s - 1), (B,)), win_start=_int(g, 0, c - a - 1, (B,)))


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = dict(case=c)
    if c["op"].startswith("rope"):
        B, L, H, d = c["B"], c["L"], c["Hq"] + 2 * c["Hkv"], c["d"]
        st["positions"] = None
        if c["far"]:
            st["positions"] = (_int(g, 0, c["far"], (B, 1)) + torch.arange(L, device=DEV)).contiguous()
        st["factors"] = None
        if c["scaling"] == "factors":
            st["factors"] = (1.0 + 7.0 * np.random.RandomState(seed % (1 << 32)).rand(c["rot"] // 2)).tolist()
        if c["op"] == "rope_fwd":
            st["qkv"] = _normal(g, B, L, H, d)
            st["out"] = [torch.empty((B, h, L, d), dtype=torch.bfloat16, device=DEV)
                         for h in (c["Hq"], c["Hkv"], c["Hkv"])]
        else:
            dt = torch.float32 if c["grad"] == "fp32" else torch.bfloat16
            st["grads"] = [_normal(g, B, h, L, d, dtype=dt) for h in (c["Hq"], c["Hkv"], c["Hkv"])]
            st["dqkv"] = torch.empty((B, L, H, d), dtype=torch.bfloat16, device=DEV)
    elif c["op"] == "decode":
        B, Hkv, d, slots = c["B"], c["Hkv"], c["d"], c["c"] + c["s"]
        st["q"] = _queries(g, B, c["Hq"], 1, d).reshape(B, c["Hq"], d)
        st["Kc"], st["Vc"] = _normal(g, B, Hkv, slots, d), _normal(g, B, Hkv, slots, d)
        st["Kp"], st["Vp"] = _normal(g, Hkv, c["P"], d), _normal(g, Hkv, c["P"], d)
        st["prefix_len"] = _prefix_len(g, c)
        st["sizes"] = _cache_sizes(g, B, c["a"], c["s"], c["w"], c["c"], c["run_lo"], c["run_hi"])
        st["o"] = torch.empty((B, c["Hq"], d), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.empty((B, c["Hq"]), dtype=torch.float32, device=DEV)
    elif c["op"] == "attn":
        B, L, Hq, Hkv, d = c["B"], c["L"], c["Hq"], c["Hkv"], c["d"]
        st["Q"] = _queries(g, B, Hq, L, d)
        st["K"], st["V"] = _normal(g, B, Hkv, L, d), _normal(g, B, Hkv, L, d)
        st["Kp"], st["Vp"] = _normal(g, Hkv, c["P"], d), _normal(g, Hkv, c["P"], d)
        st["prefix_len"] = _prefix_len(g, c)
        ids = _int(g, 50, 100, (B, L))
        sep = torch.rand((B, L), generator=g, device=DEV) < c["rho"]
        which = torch.tensor(SEP_IDS, device=DEV)[_int(g, 0, len(SEP_IDS) - 1, (B, L))]
        st["ids"] = torch.where(sep, which, ids).to(torch.int32)
        st["seq_len"] = _int(g, 1, L, (B,)).to(torch.int32) if c["ragged"] else torch.full(
            (B,), L, dtype=torch.int32, device=DEV)
        st["O"] = torch.zeros((B, Hq, L, d), dtype=torch.bfloat16, device=DEV)   # rows of padding stay as they are
        st["LSE"] = torch.zeros((B, Hq, L), dtype=torch.float32, device=DEV)
    else:
        slots = c["c"] + c["s"]
        st["Kc"], st["Vc"] = _normal(g, 1, c["Hkv"], slots, c["d"]), _normal(g, 1, c["Hkv"], slots, c["d"])
        st["sizes"] = _cache_sizes(g, 1, c["a"], c["s"], c["w"], c["c"], c["run"], c["run"])
        st["Kp"] = torch.zeros((c["Hkv"], c["c"], c["d"]), dtype=torch.bfloat16, device=DEV)
        st["Vp"] = torch.zeros_like(st["Kp"])
        st["len"] = torch.zeros((c["n_len"],), dtype=torch.int32, device=DEV)
    if own:
        _plan(st)
    return st


def _plan(st):
    """The handles that a program of the library keeps between calls: descriptors, the index built
    once per token batch, the cache state, workspaces."""
    from paper_2412_12094_b200 import api
    c = st["case"]
    if c["op"].startswith("rope"):
        st["desc"] = api.RopeDesc(c["B"], c["L"], c["Hq"], c["Hkv"], c["d"], rot_dim=c["rot"], layout=c["layout"],
                                  scaling=c["scaling"], base=c["base"], factor=c["factor"], low=c["low"],
                                  high=c["high"], orig_len=c["orig"], freq_factors=st["factors"])
    elif c["op"] == "attn":
        st["idesc"] = api.IndexDesc(c["B"], c["L"], 0, c["n_neighbor"], len(SEP_IDS), 128, 128, c["L"])
        ib, sb = api.sepllm_index_bytes(st["idesc"])
        st["index"], scratch = api.alloc_bytes(ib), api.alloc_bytes(sb)
        api.sepllm_build_index_varlen(st["idesc"], st["ids"], st["seq_len"], SEP_IDS, st["index"], scratch)
        st["desc"] = api.AttnDesc(c["B"], c["Hq"], c["Hkv"], c["d"], c["L"], 0.0, 0)
        st["ws"] = api.alloc_bytes(api.sepllm_attn_prefix_workspace_bytes(st["desc"], st["idesc"], c["P"]))
    else:
        B, Hq = c.get("B", 1), c.get("Hq", c["Hkv"])
        st["desc"] = api.CacheDesc(B, c["Hkv"], Hq, c["d"], c["a"], c["s"], c["w"], c["c"])
        st["state"] = api.alloc_bytes(api.sepllm_cache_bytes(st["desc"])[0])
        api.sepllm_cache_init(st["desc"], st["state"])
        seq = st["state"][256:256 + 64 * B].view(torch.int32).view(B, 16)   # the per-sequence records
        for k, name in enumerate(("size_init", "sep_start", "size_sep", "win_start", "size_win")):
            seq[:, k] = st["sizes"][name].to(torch.int32)
        if c["op"] == "decode":
            st["ws"] = api.alloc_bytes(api.sepllm_decode_prefix_workspace_bytes(st["desc"], c["P"]))


# ------------------------------------------------------------------------------------------ passes
def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


def _own(st):
    from paper_2412_12094_b200 import api
    c = st["case"]
    if c["op"] == "rope_fwd":
        Hq, Hkv = c["Hq"], c["Hkv"]
        q, k, v = st["qkv"].transpose(1, 2).split((Hq, Hkv, Hkv), 1)
        api.sepllm_rope_fwd(st["desc"], st["positions"], q, k, v, *st["out"])
        return st["out"]
    if c["op"] == "rope_bwd":
        Hq, Hkv = c["Hq"], c["Hkv"]
        dq, dk, dv = st["dqkv"].transpose(1, 2).split((Hq, Hkv, Hkv), 1)
        api.sepllm_rope_bwd(st["desc"], st["positions"], *st["grads"], dq, dk, dv)
        return st["dqkv"]
    if c["op"] == "decode":
        api.sepllm_decode_prefix(st["desc"], c["P"], 0.0, st["q"], st["state"], st["Kc"], st["Vc"], st["Kp"],
                                 st["Vp"], st["prefix_len"], st["o"], st["lse"], st["ws"])
        return st["o"], st["lse"]
    if c["op"] == "attn":
        api.sepllm_attn_prefix_fwd(st["desc"], st["idesc"], c["P"], st["Q"], st["K"], st["V"], st["index"], st["Kp"],
                                   st["Vp"], st["prefix_len"], st["O"], st["LSE"], st["ws"])
        return st["O"], st["LSE"]
    api.sepllm_prefix_from_cache(st["desc"], st["state"], st["Kc"], st["Vc"], c["c"], st["Kp"], st["Vp"], st["len"])
    return st["Kp"], st["Vp"], st["len"]


def _frequencies(c, factors):
    """Angle per position of every rotated pair (64 bits) and the factor on both rotated outputs."""
    r, base, s = c["rot"], c["base"], c["factor"]
    i = torch.arange(r // 2, dtype=torch.float64, device=DEV)
    if c["scaling"] == "ntk":
        base = base * s ** (r / (r - 2))
    f = base ** (-2.0 * i / r)
    if c["scaling"] == "linear":
        f = f / s
    if c["scaling"] == "factors":
        f = f / torch.tensor(factors, dtype=torch.float64, device=DEV)
    if c["scaling"] == "llama3":
        turns = c["orig"] * f / (2.0 * math.pi)
        keep = ((turns - c["low"]) / (c["high"] - c["low"])).clamp(0.0, 1.0)
        f = f * keep + f / s * (1.0 - keep)
    if c["scaling"] == "yarn":
        lo = max(math.floor(r * math.log(c["orig"] / (c["high"] * 2.0 * math.pi)) / (2.0 * math.log(base))), 0)
        hi = min(math.ceil(r * math.log(c["orig"] / (c["low"] * 2.0 * math.pi)) / (2.0 * math.log(base))), r - 1)
        far = ((i - lo) / (hi - lo if hi != lo else 0.001)).clamp(0.0, 1.0)
        f = f / s * far + f * (1.0 - far)
        return f, 0.1 * math.log(s) + 1.0
    return f, 1.0


def _turn(x, cos, sin, layout, r):
    """Pairs of the first r elements of x [..., H, d] turned by (cos, sin) [..., 1, r / 2]."""
    y = x.float()
    if layout == "half":
        a, b = y[..., : r // 2], y[..., r // 2: r]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned, y[..., r:]), -1)


def _cos_sin(st, inverse):
    c = st["case"]
    f, m = _frequencies(c, st["factors"])
    pos = st["positions"] if st["positions"] is not None else torch.arange(c["L"], device=DEV)[None]
    angle = pos.double()[..., None] * f                      # far positions: 64 bits
    sign = -1.0 if inverse else 1.0
    return (torch.cos(angle) * m).float(), (torch.sin(angle) * (m * sign)).float()   # [B or 1][L][r/2]


def _plain_rope_fwd(st):
    c = st["case"]
    cos, sin = _cos_sin(st, False)
    q, k, v = st["qkv"].split((c["Hq"], c["Hkv"], c["Hkv"]), 2)
    q, k = (_turn(x, cos[:, :, None], sin[:, :, None], c["layout"], c["rot"]) for x in (q, k))
    return [x.transpose(1, 2).to(torch.bfloat16).contiguous() for x in (q, k, v)]


def _plain_rope_bwd(st):
    c = st["case"]
    cos, sin = _cos_sin(st, True)
    dq, dk, dv = (x.transpose(1, 2) for x in st["grads"])
    dq, dk = (_turn(x, cos[:, :, None], sin[:, :, None], c["layout"], c["rot"]) for x in (dq, dk))
    return torch.cat((dq, dk, dv.float()), 2).to(torch.bfloat16)


def _entry_slots(sizes, a, s, c, n):
    """Slot of cache entry v of every sequence, v < n (walked as initial, separator, neighbour),
    and whether the entry is there.  [B][n]"""
    v = torch.arange(n, device=DEV)[None]
    i, q, w = (sizes[k][:, None] for k in ("size_init", "size_sep", "size_win"))
    sep = a + (sizes["sep_start"][:, None] + v - i) % max(s, 1)
    win = a + s + (sizes["win_start"][:, None] + v - i - q) % (c - a)
    return torch.where(v < i, v, torch.where(v < i + q, sep, win)), v < i + q + w


def _own_rows(st):
    c = st["case"]
    slot, there = _entry_slots(st["sizes"], c["a"], c["s"], c["c"], c["c"])
    at = torch.where(there, slot, torch.zeros_like(slot))[:, None, :, None].expand(-1, c["Hkv"], -1, c["d"])
    return st["Kc"].gather(2, at), st["Vc"].gather(2, at), there


def _in_prefix(st):
    """[B][P]: entry seen by the sequence."""
    c = st["case"]
    p = torch.arange(c["P"], device=DEV)[None]
    return (p < st["prefix_len"][:, None]) if st["prefix_len"] is not None else (p < c["P"]).expand(c["B"], -1)


def _softmax_two(sp, so, vp, vo):
    """Rows of scores over the prefix and over the sequence's own keys, masked ones at -inf, and
    their values; an empty row gives 0 and a log-sum-exp of -inf."""
    m = torch.maximum(sp.amax(-1, keepdim=True), so.amax(-1, keepdim=True))
    z = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    ep, eo = torch.exp(sp - z), torch.exp(so - z)
    total = ep.sum(-1, keepdim=True) + eo.sum(-1, keepdim=True)
    o = (torch.matmul(ep, vp) + torch.matmul(eo, vo)) / torch.where(total > 0, total, torch.ones_like(total))
    return o, (z + torch.log(total))[..., 0]


def _plain_decode(st):
    c = st["case"]
    B, Hq, Hkv, d, G = c["B"], c["Hq"], c["Hkv"], c["d"], c["Hq"] // c["Hkv"]
    q = st["q"].float().view(B, Hkv, G, d) / math.sqrt(d)
    k, v, there = _own_rows(st)
    so = torch.matmul(q, k.float().transpose(-1, -2)).masked_fill(~there[:, None, None], -math.inf)
    sp = torch.matmul(q, st["Kp"].float().transpose(-1, -2)).masked_fill(~_in_prefix(st)[:, None, None], -math.inf)
    o, lse = _softmax_two(sp, so, st["Vp"].float(), v.float())
    return o.reshape(B, Hq, d).to(torch.bfloat16), lse.reshape(B, Hq)


def _own_mask(st):
    """[B][L][L]: key j kept by query i of the sequence's own tokens."""
    c = st["case"]
    i, j = torch.arange(c["L"], device=DEV)[:, None], torch.arange(c["L"], device=DEV)[None]
    sep = torch.isin(st["ids"], torch.tensor(SEP_IDS, dtype=torch.int32, device=DEV))
    return (j <= i) & ((i - j < c["n_neighbor"]) | sep[:, None, :])


def _plain_attn(st):
    c = st["case"]
    B, L, Hkv, d, G = c["B"], c["L"], c["Hkv"], c["d"], c["Hq"] // c["Hkv"]
    q = st["Q"].float().view(B, Hkv, G * L, d) / math.sqrt(d)
    so = torch.matmul(q, st["K"].float().transpose(-1, -2)).view(B, Hkv, G, L, L)
    so = so.masked_fill(~_own_mask(st)[:, None, None], -math.inf).view(B, Hkv, G * L, L)
    sp = torch.matmul(q, st["Kp"].float().transpose(-1, -2)).masked_fill(~_in_prefix(st)[:, None, None], -math.inf)
    o, lse = _softmax_two(sp, so, st["Vp"].float(), st["V"].float())
    o, lse = o.reshape(B, c["Hq"], L, d).to(torch.bfloat16), lse.reshape(B, c["Hq"], L)
    token = (torch.arange(L, device=DEV)[None] < st["seq_len"][:, None])[:, None]
    return torch.where(token[..., None], o, st["O"]), torch.where(token, lse, st["LSE"])


def _plain_prefix(st):
    c = st["case"]
    k, v, there = _own_rows(st)
    n = there.sum(-1).to(torch.int32)
    return (torch.where(there[0][None, :, None], k[0], st["Kp"]), torch.where(there[0][None, :, None], v[0], st["Vp"]),
            n.expand(c["n_len"]).contiguous())


_PLAIN = dict(rope_fwd=_plain_rope_fwd, rope_bwd=_plain_rope_bwd, decode=_plain_decode, attn=_plain_attn,
              prefix=_plain_prefix)


# ------------------------------------------------------------------------------------------ work
def work(case):
    """Inputs read once, outputs written once; two operations per product and sum."""
    c = case
    if c["op"].startswith("rope"):
        n = c["B"] * c["L"] * (c["Hq"] + 2 * c["Hkv"]) * c["d"]
        turned = c["B"] * c["L"] * (c["Hq"] + c["Hkv"]) * c["rot"]
        src = 4 if c["op"] == "rope_bwd" and c["grad"] == "fp32" else 2
        return {"bytes": n * (src + 2) + (8 * c["B"] * c["L"] if c["far"] else 0), "flops": 3 * turned}
    if c["op"] == "prefix":
        return {"bytes": 8 * c["Hkv"] * c["run"] * c["d"] + 4 * c["n_len"], "flops": 0}
    plen = (c["plen_lo"] + c["P"]) / 2
    shared = 4 * c["Hkv"] * c["P"] * c["d"]
    if c["op"] == "decode":
        run_ = (c["run_lo"] + c["run_hi"]) / 2
        rows = c["B"] * c["Hq"]
        return {"bytes": shared + 4 * c["B"] * c["Hkv"] * run_ * c["d"] + 4 * rows * c["d"] + 4 * rows,
                "flops": 4 * rows * (plen + run_) * c["d"]}
    tokens = c["B"] * (c["L"] / 2 if c["ragged"] else c["L"])
    side, window = c["rho"] * c["L"] / 2, min(c["n_neighbor"], c["L"] / 2)
    return {"bytes": shared + tokens * (4 * c["Hkv"] + 4 * c["Hq"]) * c["d"] + 4 * tokens * c["Hq"],
            "flops": 4 * tokens * c["Hq"] * (plen + min(c["L"] / 2, side + window)) * c["d"]}


# ------------------------------------------------------------------------------------------ exact
def exact(case, seed):
    st = prepare(case, seed)
    c = case
    if c["op"].startswith("rope"):
        return _exact_rope(st)
    if c["op"] == "prefix":
        slot = _walk(st, 0)
        kp, vp = st["Kp"].double(), st["Vp"].double()
        kp[:, : len(slot)], vp[:, : len(slot)] = st["Kc"][0].double()[:, slot], st["Vc"][0].double()[:, slot]
        return kp, vp, torch.full((c["n_len"],), len(slot), dtype=torch.int32, device=DEV)
    plen = st["prefix_len"].tolist() if st["prefix_len"] is not None else [c["P"]] * c["B"]
    G = c["Hq"] // c["Hkv"]
    kp, vp = st["Kp"].double(), st["Vp"].double()
    if c["op"] == "decode":
        o = torch.zeros((c["B"], c["Hkv"], G, c["d"]), dtype=torch.float64, device=DEV)
        lse = torch.full((c["B"], c["Hkv"], G), -math.inf, dtype=torch.float64, device=DEV)
        for b in range(c["B"]):
            slot = _walk(st, b)
            k = torch.cat((kp[:, : plen[b]], st["Kc"][b].double()[:, slot]), 1)
            v = torch.cat((vp[:, : plen[b]], st["Vc"][b].double()[:, slot]), 1)
            if k.shape[1]:
                q = st["q"][b].double().view(c["Hkv"], G, c["d"])
                o[b], lse[b] = _exact_rows(q, k, v, None)
        return o.view(c["B"], c["Hq"], c["d"]), lse.view(c["B"], c["Hq"])
    o, lse = st["O"].double(), st["LSE"].double()
    sep = np.isin(st["ids"].cpu().numpy(), SEP_IDS)
    for b, n in enumerate(st["seq_len"].tolist()):
        i = np.arange(n)
        keep = ((i[:, None] >= i) & ((i[:, None] < i + c["n_neighbor"]) | sep[b, :n]))
        keep = torch.from_numpy(np.concatenate((np.ones((n, plen[b]), bool), keep), 1)).to(DEV)
        for h in range(c["Hq"]):
            k = torch.cat((kp[h // G, : plen[b]], st["K"][b, h // G, :n].double()))
            v = torch.cat((vp[h // G, : plen[b]], st["V"][b, h // G, :n].double()))
            o[b, h, :n], lse[b, h, :n] = _exact_rows(st["Q"][b, h, :n].double(), k, v, keep)
    return o, lse


def _walk(st, b):
    """Slots of the entries that sequence b holds, in order, from the layout's definition."""
    c = st["case"]
    z = {k: int(v[b]) for k, v in st["sizes"].items()}
    slots = list(range(z["size_init"]))
    slots += [c["a"] + (z["sep_start"] + k) % c["s"] for k in range(z["size_sep"])]
    slots += [c["a"] + c["s"] + (z["win_start"] + k) % (c["c"] - c["a"]) for k in range(z["size_win"])]
    return torch.tensor(slots, dtype=torch.int64, device=DEV)


def _exact_rows(q, k, v, keep):
    s = q @ k.transpose(-1, -2) / math.sqrt(q.shape[-1])
    if keep is not None:
        s = torch.where(keep, s, torch.full_like(s, -math.inf))
    lse = torch.logsumexp(s, -1)
    return torch.exp(s - lse[..., None]) @ v, lse


def _exact_rope(st):
    """Every pair as a complex number, turned by exp(i angle)."""
    c = st["case"]
    r, n = c["rot"], c["rot"] // 2
    freq = []
    for i in range(n):
        f = 1.0 / c["base"] ** (2 * i / r)
        if c["scaling"] == "linear":
            f /= c["factor"]
        elif c["scaling"] == "ntk":
            f = 1.0 / (c["base"] * c["factor"] ** (r / (r - 2))) ** (2 * i / r)
        elif c["scaling"] == "factors":
            f /= st["factors"][i]
        elif c["scaling"] == "llama3":
            wave = 2 * math.pi / f
            if wave > c["orig"] / c["low"]:
                f /= c["factor"]
            elif wave >= c["orig"] / c["high"]:
                t = (c["orig"] / wave - c["low"]) / (c["high"] - c["low"])
                f = (1 - t) * f / c["factor"] + t * f
        elif c["scaling"] == "yarn":
            def pair_of(turns):
                return r * math.log(c["orig"] / (turns * 2 * math.pi)) / (2 * math.log(c["base"]))
            lo, hi = max(0, math.floor(pair_of(c["high"]))), min(r - 1, math.ceil(pair_of(c["low"])))
            t = min(1.0, max(0.0, (i - lo) / (hi - lo if hi != lo else 0.001)))
            f = t * f / c["factor"] + (1 - t) * f
        freq.append(f)
    m = 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "yarn" else 1.0
    pos = st["positions"] if st["positions"] is not None else torch.arange(c["L"], device=DEV).expand(c["B"], -1)
    ang = pos.double()[:, None, :, None] * torch.tensor(freq, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(ang, m), ang if c["op"] == "rope_fwd" else -ang)

    def apply(x):
        x = x.double().clone()
        pairs = (x[..., :n], x[..., n:r]) if c["layout"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])
        z = torch.complex(pairs[0].contiguous(), pairs[1].contiguous()) * turn
        pairs[0].copy_(z.real)
        pairs[1].copy_(z.imag)
        return x
    if c["op"] == "rope_fwd":
        q, k, v = st["qkv"].transpose(1, 2).split((c["Hq"], c["Hkv"], c["Hkv"]), 1)
        return [apply(q), apply(k), v.double().contiguous()]
    dq, dk, dv = st["grads"]
    return torch.cat((apply(dq), apply(dk), dv.double()), 1).transpose(1, 2).contiguous()
