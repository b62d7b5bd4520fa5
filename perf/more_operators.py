"""Cases, plain forms and exact values of the head-norm and 4-bit-cache operators.

Operators: norms of every query and key head with the rotary positions in the same pass, and their
gradient (`sepllm_qknorm_rope_fwd`, `sepllm_qknorm_rope_bwd`); decode of one token per sequence over a
four-part cache held in 4 bits (`sepllm_decode_quant`); a token taken into such caches, and a
pre-filled prompt handed to them (`sepllm_cache_update_quant`, `sepllm_cache_from_prompt_quant`), each
with the retained entries read back in 16 bits (`sepllm_cache_entries_quant`).

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
GROUP = 32           # elements of a row that share a step
FLUSH = 2.0 ** -100  # groups whose largest magnitude is below are held as zeros


# ------------------------------------------------------------------------------------------ cases
def _norm(name, op, B, L, Hq, Hkv, d, rot, layout, scaling="none", base=10000.0, factor=1.0, orig=8192.0, far=0,
          grad="bf16", weight="bf16", offset=0.0):
    c = dict(op=op, B=B, L=L, Hq=Hq, Hkv=Hkv, d=d, rot=rot, layout=layout, scaling=scaling, base=base, factor=factor,
             low=1.0, high=4.0, orig=orig, far=far, grad=grad, weight=weight, offset=offset, eps=1e-6)
    return dict(c, name=name) if name else c


def _cache(name, op, B, Hq, Hkv, d, a, s, w, c, fixed, rho, **kw):
    r = dict(op=op, B=B, Hq=Hq, Hkv=Hkv, d=d, a=a, s=s, w=w, c=c, fixed=fixed, rho=rho, **kw)
    return dict(r, name=name) if name else r


def listed():
    return [
        # one generated token per sequence of the streaming-decode batch, far into the text.  Latency.
        _norm("norm_step", "norm_fwd", 32, 1, 32, 8, 128, 128, "half", "llama3", 500000.0, 8.0, far=1 << 20),
        # the long-context row of the benchmark, straight from the fused projection
        _norm("norm_long", "norm_fwd", 1, 65536, 32, 8, 128, 128, "half", "none", 500000.0),
        # a ragged batch whose head size is no power of two, neighbouring pairs, weights around zero
        _norm("norm_odd", "norm_fwd", 3, 1999, 10, 2, 80, 40, "interleaved", "linear", 10000.0, 2.5, far=5000,
              weight="fp32", offset=1.0),
        # gradients of a training row in 32 bits, back to the projection's layout
        _norm("norm_bwd_long", "norm_bwd", 1, 16384, 32, 8, 128, 128, "half", "none", 500000.0, grad="fp32"),
        # the small pre-training batch: a quarter of every head is rotated
        _norm("norm_bwd_batch", "norm_bwd", 8, 2048, 12, 12, 64, 16, "half", weight="fp32"),
        # the streaming-decode batch, its caches in 4 bits
        _cache("quant_decode_batch", "decode", 32, 32, 8, 128, 4, 1024, 256, 3332, False, 0.12, lo=2200, hi=3300),
        # a few sequences of a small model, some only just begun, one with nothing in its cache
        _cache("quant_decode_few", "decode", 5, 12, 12, 64, 2, 64, 64, 300, False, 0.12, lo=0, hi=299),
        # two long texts in the fundamental design: every separator's entry is kept
        _cache("quant_decode_long", "decode", 2, 32, 8, 128, 4, 120000, 4096, 130000, True, 0.12, lo=100000, hi=124000),
        # a token taken in by two small caches, which then move to another engine in 16 bits
        _cache("quant_append_small", "append", 2, 4, 2, 64, 2, 32, 64, 300, False, 0.3, lo=250, hi=299),
        # the same for a batch, some of its sequences at the point where the cache is compacted
        _cache("quant_append_batch", "append", 16, 32, 8, 128, 4, 256, 256, 1200, False, 0.12, lo=1190, hi=1199),
        # short ragged prompts handed to caches of the fundamental design and read back
        _cache("quant_prompt_short", "prompt", 8, 12, 12, 64, 4, 64, 64, 180, True, 0.12, L=300, ragged=True),
        # long prompts handed to the streaming caches and read back
        _cache("quant_prompt_long", "prompt", 4, 32, 8, 128, 4, 1024, 256, 3332, False, 0.10, L=16384, ragged=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "decode", "decode", "append", "prompt"])
    if op.startswith("norm"):
        d = rng.choice([64, 80, 96, 112, 128])
        Hkv = rng.choice([1, 2, 4, 8, 12])
        Hq = Hkv * rng.choice([1, 2, 4, 5])
        most = (1 << 28) if op == "norm_fwd" else (100 << 20)
        tokens = _log(rng, 1, most // ((Hq + 2 * Hkv) * d))
        B = min(tokens, _log(rng, 1, 64))
        scaling = rng.choice(["none", "linear", "llama3"])
        return _norm(None, op, B, max(1, tokens // B), Hq, Hkv, d, rng.choice([d, d, d // 2, 2 * rng.randint(2, d // 2)]),
                     rng.choice(["half", "interleaved"]), scaling, rng.choice([10000.0, 500000.0, 1000000.0]),
                     1.0 if scaling == "none" else rng.uniform(1.5, 16.0), float(_log(rng, 2048, 32768)),
                     rng.choice([0, _log(rng, 100, 1 << 24)]), rng.choice(["bf16", "fp32"]),
                     rng.choice(["bf16", "fp32"]), rng.choice([0.0, 1.0]))
    d = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 8, 12])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 8, 16])
    a, w, fixed = rng.randint(0, 8), _log(rng, 1, 512), rng.random() < 0.4
    rho = rng.uniform(0.02, 0.4)
    if op == "decode":
        B, run = _log(rng, 1, 256), _log(rng, 1, 100000)
        while B * Hkv * run * d > 32 * 8 * 3300 * 128 or B * Hq * run > 2 * 32 * 124000:
            B, run = (B + 1) // 2, max(1, run * 3 // 4)
        s = max(run - a - w, 0) if fixed else rng.choice([0, _log(rng, 1, 1024)])
        c = max(run, a + s + w) + _log(rng, 1, 256)
        return _cache(None, op, B, Hq, Hkv, d, a, s, w, c, fixed, rho, lo=rng.choice([0, run // 2, run]), hi=run)
    s = rng.choice([0, _log(rng, 1, 1024)])
    c = a + s + w + _log(rng, 16, 1024)
    B = _log(rng, 1, 32)
    if op == "append":
        while B * Hkv * c * d > 16 * 8 * 1200 * 128:
            B = (B + 1) // 2
            Hkv, Hq = (Hkv, Hq) if B > 1 else (1, Hq // Hkv)
        hi = a + s + w if fixed else c - 1
        return _cache(None, op, B, Hq, Hkv, d, a, s, w, c, fixed, rho, lo=rng.choice([0, hi]), hi=hi)
    L = _log(rng, 1, min(16384, 32 * (c - a - s - w)))
    while B * Hkv * L * d > 4 * 8 * 16384 * 128 or B * Hkv * c * d > 4 * 8 * 3332 * 128:
        B, L = (B + 1) // 2, max(1, L // 2)
        if B == 1:
            Hkv, Hq = 1, Hq // Hkv
    return _cache(None, op, B, Hq, Hkv, d, a, s, w, c, fixed, rho, L=L, ragged=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _int(g, lo, hi, shape):
    """Uniform in [lo, hi], int64."""
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV)


def _ids(g, rho, *shape):
    which = torch.tensor(SEP_IDS, device=DEV)[_int(g, 0, len(SEP_IDS) - 1, shape)]
    sep = torch.rand(shape, generator=g, device=DEV) < rho
    return torch.where(sep, which, _int(g, 50, 100, shape)).to(torch.int32)


def _is_sep(ids):
    return torch.isin(ids, torch.tensor(SEP_IDS, dtype=torch.int32, device=DEV))


def _channels(g, Hkv, d):
    """Sizes of a key head's elements: some channels are several times the others, as in trained models."""
    c = torch.exp(0.4 * torch.randn((Hkv, 1, d), generator=g, device=DEV))
    return c * torch.where(torch.rand((Hkv, 1, d), generator=g, device=DEV) < 0.03, 5.0, 1.0)


def _quantise(x):
    """Codes (int8, -8 .. 7) and steps (bf16) of rows of 16-bit values: 32 neighbouring elements share
    the step -m / 8, m their element of largest magnitude (the positive one of two equal ones), and an
    element's code is the whole number nearest to it in steps (even at a tie), at most 7."""
    y = x.float().unflatten(-1, (-1, GROUP))
    most, least = y.amax(-1), y.amin(-1)
    m = torch.where(most >= -least, most, least)
    step = torch.where(m.abs() < FLUSH, torch.zeros_like(m), m / -8.0)
    code = torch.round(y / torch.where(step == 0, torch.ones_like(step), step)[..., None]).clamp(-8, 7)
    code = torch.where((step == 0)[..., None], torch.zeros_like(code), code)
    return code.to(torch.int8).flatten(-2), step.to(torch.bfloat16)


def _values(code, step):
    """What codes and steps stand for, 32 bits (exact)."""
    return (code.float().unflatten(-1, (-1, GROUP)) * step.float()[..., None]).flatten(-2)


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = dict(case=c)
    if c["op"].startswith("norm"):
        B, L, H, d = c["B"], c["L"], c["Hq"] + 2 * c["Hkv"], c["d"]
        st["positions"] = None
        if c["far"]:
            st["positions"] = (_int(g, 0, c["far"], (B, 1)) + torch.arange(L, device=DEV)).contiguous()
        size = torch.exp(0.7 * torch.randn((1, 1, H, 1), generator=g, device=DEV))     # heads differ in size
        st["qkv"] = (torch.randn((B, L, H, d), generator=g, device=DEV) * size).to(torch.bfloat16)
        dt = torch.bfloat16 if c["weight"] == "bf16" else torch.float32
        st["wq"], st["wk"] = ((1.0 - c["offset"] + 0.2 * torch.randn(d, generator=g, device=DEV)).to(dt) for _ in "qk")
        if c["op"] == "norm_fwd":
            st["out"] = [torch.empty((B, h, L, d), dtype=torch.bfloat16, device=DEV)
                         for h in (c["Hq"], c["Hkv"], c["Hkv"])]
        else:
            gt = torch.float32 if c["grad"] == "fp32" else torch.bfloat16
            st["grads"] = [_normal(g, B, h, L, d, dtype=gt) for h in (c["Hq"], c["Hkv"], c["Hkv"])]
            st["dqkv"] = torch.empty((B, L, H, d), dtype=torch.bfloat16, device=DEV)
            st["dw"] = [torch.empty(d, dtype=torch.float32, device=DEV) for _ in "qk"]
    else:
        _prepare_cache(c, g, st)
    if own:
        _plan(st)
    return st


def _prepare_cache(c, g, st):
    B, Hq, Hkv, d, a, s, w = (c[k] for k in ("B", "Hq", "Hkv", "d", "a", "s", "w"))
    slots = c["c"] + s
    chan = _channels(g, Hkv, d)
    if c["op"] == "prompt":
        L = c["L"]
        st["ids"] = _ids(g, c["rho"], B, L)
        st["K"] = (torch.randn((B, Hkv, L, d), generator=g, device=DEV) * chan).to(torch.bfloat16)
        st["V"] = _normal(g, B, Hkv, L, d)
        st["prompt_len"] = _int(g, 1, L, (B,)).to(torch.int32) if c["ragged"] else None
    else:
        # caches in the middle of a text: sizes, where the rings start, which slots hold separators
        run = _int(g, c["lo"], c["hi"], (B,))
        init = run.clamp(max=a)
        rest = run - init
        win = rest.clamp(max=w) if c["fixed"] else torch.maximum(rest - s, torch.minimum(rest, w + (rest - w) // 2))
        sizes = dict(size_init=init, size_sep=rest - win, size_win=win, sep_start=_int(g, 0, max(0, s - 1), (B,)),
                     win_start=_int(g, 0, c["c"] - a - 1, (B,)))
        st["sizes"] = sizes
        st["is_sep"] = torch.rand((B, slots + 1), generator=g, device=DEV) < c["rho"]
        # one row more than the cache has: where rows that are not kept go
        st["code"] = [torch.zeros((B, Hkv, slots + 1, d), dtype=torch.int8, device=DEV) for _ in "kv"]
        st["step"] = [torch.zeros((B, Hkv, slots + 1, d // GROUP), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
        for b in range(B):
            for i, scale in enumerate((chan, 1.0)):
                x = torch.randn((Hkv, slots, d), generator=g, device=DEV) * scale
                st["code"][i][b, :, :slots], st["step"][i][b, :, :slots] = _quantise(x.to(torch.bfloat16))
    if c["op"] == "decode":
        sharp = torch.rand((1, Hq, 1), generator=g, device=DEV) * 2.5 + 0.5      # heads from diffuse to sharp
        st["q"] = (torch.randn((B, Hq, d), generator=g, device=DEV) * sharp).to(torch.bfloat16)
        st["o"] = torch.empty((B, Hq, d), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.empty((B, Hq), dtype=torch.float32, device=DEV)
        return
    if c["op"] == "append":
        st["new_ids"] = _ids(g, c["rho"], B)
        st["k_new"] = (torch.randn((B, Hkv, 1, d), generator=g, device=DEV) * chan).to(torch.bfloat16)[:, :, 0].contiguous()
        st["v_new"] = _normal(g, B, Hkv, d)
    st["Kout"], st["Vout"] = (torch.zeros((B, Hkv, c["c"], d), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    st["len"] = torch.zeros((B,), dtype=torch.int32, device=DEV)


def _packed(code, step, unit):
    """A cache buffer of the library: two codes (+ 8) to a byte in the order (unit, group, place in the
    unit), then, 256-byte aligned, the steps."""
    slots = code.shape[2] - 1
    n = (code[:, :, :slots] + 8).to(torch.uint8)
    n = n.unflatten(-1, (-1, GROUP // unit, unit)).transpose(-3, -2).flatten(-3).unflatten(-1, (-1, 2))
    codes = (n[..., 0] | (n[..., 1] << 4)).flatten()
    steps = step[:, :, :slots].contiguous().flatten().view(torch.uint8)
    gap = torch.zeros((-codes.numel()) % 256, dtype=torch.uint8, device=DEV)
    return torch.cat((codes, gap, steps))


def _plan(st):
    """The handles that a program of the library keeps between calls: descriptors, weights, the index
    built once per token batch, the caches, workspaces."""
    from paper_2412_12094_b200 import api
    c = st["case"]
    if c["op"].startswith("norm"):
        st["desc"] = api.RopeDesc(c["B"], c["L"], c["Hq"], c["Hkv"], c["d"], rot_dim=c["rot"], layout=c["layout"],
                                  scaling=c["scaling"], base=c["base"], factor=c["factor"], low=c["low"],
                                  high=c["high"], orig_len=c["orig"])
        st["norm"] = api.QkNorm(st["wq"], st["wk"], eps=c["eps"], offset=c["offset"])
        if c["op"] == "norm_bwd":
            st["ws"] = api.alloc_bytes(api.sepllm_qknorm_rope_bwd_workspace_bytes(st["desc"]))
        return
    B = c["B"]
    st["desc"] = api.CacheDesc(B, c["Hkv"], c["Hq"], c["d"], c["a"], c["s"], c["w"], c["c"],
                               api.CACHE_FIXED_WINDOW if c["fixed"] else 0)
    state_bytes, kv_bytes = api.sepllm_cache_bytes_quant(st["desc"])
    st["state"], st["Kc"], st["Vc"] = (api.alloc_bytes(n) for n in (state_bytes, kv_bytes, kv_bytes))
    if c["op"] == "prompt":
        st["idesc"] = api.IndexDesc(B, c["L"], c["a"], 64, len(SEP_IDS), 128, 128, c["L"])
        ib, sb = api.sepllm_index_bytes(st["idesc"])
        st["index"], scratch = api.alloc_bytes(ib), api.alloc_bytes(sb)
        api.sepllm_build_index(st["idesc"], st["ids"], SEP_IDS, st["index"], scratch)
        return
    api.sepllm_cache_init(st["desc"], st["state"])
    head = api.CacheHeader.from_buffer_copy(bytes(st["state"][:256].tolist()))
    seq = st["state"][head.off_seq:head.off_seq + 64 * B].view(torch.int32).view(B, 16)
    for k, name in enumerate(("size_init", "sep_start", "size_sep", "win_start", "size_win")):
        seq[:, k] = st["sizes"][name].to(torch.int32)
    flags = st["state"][head.off_slot_is_sep:head.off_slot_is_sep + B * head.slots].view(B, head.slots)
    flags.copy_(st["is_sep"][:, : head.slots])
    for buf, code, step, unit in zip((st["Kc"], st["Vc"]), st["code"], st["step"], (8, 4)):
        packed = _packed(code, step, unit)
        buf[: packed.numel()] = packed
    del st["code"], st["step"]
    if c["op"] == "decode":
        st["ws"] = api.alloc_bytes(api.sepllm_decode_quant_workspace_bytes(st["desc"]))


# ------------------------------------------------------------------------------------------ passes
def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


def _own(st):
    from paper_2412_12094_b200 import api
    c = st["case"]
    if c["op"].startswith("norm"):
        heads = (c["Hq"], c["Hkv"], c["Hkv"])
        q, k, v = st["qkv"].transpose(1, 2).split(heads, 1)
        if c["op"] == "norm_fwd":
            api.sepllm_qknorm_rope_fwd(st["desc"], st["norm"], st["positions"], q, k, v, *st["out"])
            return st["out"]
        dq, dk, dv = st["dqkv"].transpose(1, 2).split(heads, 1)
        api.sepllm_qknorm_rope_bwd(st["desc"], st["norm"], st["positions"], q, k, *st["grads"], dq, dk, dv, *st["dw"],
                                   st["ws"])
        return st["dqkv"], *st["dw"]
    if c["op"] == "decode":
        api.sepllm_decode_quant(st["desc"], 0.0, st["q"], st["state"], st["Kc"], st["Vc"], st["o"], st["lse"], st["ws"])
        return st["o"], st["lse"]
    if c["op"] == "append":
        api.sepllm_cache_update_quant(st["desc"], st["state"], st["Kc"], st["Vc"], st["new_ids"], SEP_IDS, st["k_new"],
                                      st["v_new"])
    else:
        api.sepllm_cache_from_prompt_quant(st["desc"], st["idesc"], st["index"], st["prompt_len"], st["K"], st["V"],
                                           st["state"], st["Kc"], st["Vc"])
    api.sepllm_cache_entries_quant(st["desc"], st["state"], st["Kc"], st["Vc"], c["c"], st["Kout"], st["Vout"],
                                   st["len"])
    return st["Kout"], st["Vout"], st["len"]


def _cos_sin(st):
    c = st["case"]
    f = c["base"] ** (-2.0 * torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEV) / c["rot"])
    if c["scaling"] == "linear":
        f = f / c["factor"]
    if c["scaling"] == "llama3":
        turns = c["orig"] * f / (2.0 * math.pi)
        keep = ((turns - c["low"]) / (c["high"] - c["low"])).clamp(0.0, 1.0)
        f = f * keep + f / c["factor"] * (1.0 - keep)
    pos = st["positions"] if st["positions"] is not None else torch.arange(c["L"], device=DEV)[None]
    angle = pos.double()[..., None] * f                       # far positions: 64 bits
    return torch.cos(angle).float(), torch.sin(angle).float()  # [B or 1][L][rot / 2]


def _turn(y, cos, sin, layout, r):
    """Pairs of the first r elements of y [..., d] (32 bits) turned by (cos, sin) [..., r / 2]."""
    if layout == "half":
        a, b = y[..., : r // 2], y[..., r // 2: r]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned, y[..., r:]), -1)


def _plain_norm_fwd(st):
    c = st["case"]
    cos, sin = (t[:, :, None] for t in _cos_sin(st))
    out = []
    for x, w in zip(st["qkv"].split((c["Hq"], c["Hkv"], c["Hkv"]), 2), (st["wq"], st["wk"], None)):
        if w is not None:
            y = x.float()
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + c["eps"]) * (c["offset"] + w.float())
            x = _turn(y, cos, sin, c["layout"], c["rot"])
        out.append(x.transpose(1, 2).to(torch.bfloat16).contiguous())
    return out


def _plain_norm_bwd(st):
    c = st["case"]
    cos, sin = (t[:, :, None] for t in _cos_sin(st))
    dx, dw = [], []
    for x, dy, w in zip(st["qkv"].split((c["Hq"], c["Hkv"], c["Hkv"]), 2), st["grads"], (st["wq"], st["wk"], None)):
        dy = dy.transpose(1, 2).float()
        if w is None:
            dx.append(dy)
            continue
        g = _turn(dy, cos, -sin, c["layout"], c["rot"])
        y = x.float()
        r = torch.rsqrt(y.square().mean(-1, keepdim=True) + c["eps"])
        n, u = y * r, g * (c["offset"] + w.float())
        dx.append(r * (u - n * (n * u).mean(-1, keepdim=True)))
        dw.append((g * n).sum((0, 1, 2), dtype=torch.float64).float())     # a long sum
    return torch.cat(dx, 2).to(torch.bfloat16), *dw


def _entry_slots(z, c, n):
    """Slot of cache entry v of every sequence, v < n (walked as initial, separator, neighbour),
    and whether the entry is there.  [B][n]"""
    a, s = c["a"], c["s"]
    v = torch.arange(n, device=DEV)[None]
    i, q, w = (z[k][:, None] for k in ("size_init", "size_sep", "size_win"))
    sep = a + (z["sep_start"][:, None] + v - i) % max(s, 1)
    win = a + s + (z["win_start"][:, None] + v - i - q) % (c["c"] - a)
    return torch.where(v < i, v, torch.where(v < i + q, sep, win)), v < i + q + w


def _rows(x, slot):
    """Rows [B][H][n] of x [B][H][slots][m] at slot [B][n]."""
    return x.gather(2, slot[:, None, :, None].expand(-1, x.shape[1], -1, x.shape[3]))


def _plain_decode(st):
    c = st["case"]
    B, Hkv, d, G = c["B"], c["Hkv"], c["d"], c["Hq"] // c["Hkv"]
    q = st["q"].float().view(B, Hkv, G, d) / math.sqrt(d)
    slot, there = _entry_slots(st["sizes"], c, max(c["hi"], 1))
    slot = torch.where(there, slot, torch.zeros_like(slot))
    k, v = (_values(_rows(x, slot), _rows(e, slot)) for x, e in zip(st["code"], st["step"]))
    sc = torch.matmul(q, k.transpose(-1, -2)).masked_fill(~there[:, None, None], -math.inf)
    m = sc.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    e = torch.exp(sc - m)
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.reshape(B, c["Hq"], d).to(torch.bfloat16), (m + torch.log(total)).reshape(B, c["Hq"])


def _plain_append(st):
    """One token per sequence; where the cache is full (or a token leaves a fixed window) the separators
    among the entries that leave the window join the separator ring, which keeps its newest."""
    c, z, flag = st["case"], st["sizes"], st["is_sep"]
    a, s, w, ring = c["a"], c["s"], c["w"], c["c"] - c["a"]
    B, dump, seq = c["B"], c["c"] + s, torch.arange(c["B"], device=DEV)
    first = z["size_init"] < a
    slot = torch.where(first, z["size_init"], a + s + (z["win_start"] + z["size_win"]) % ring)
    flag[seq, slot] = _is_sep(st["new_ids"])
    for code, step, x in zip(st["code"], st["step"], (st["k_new"], st["v_new"])):
        code[seq, :, slot], step[seq, :, slot] = _quantise(x)
    z["size_init"] = z["size_init"] + first
    z["size_win"] = z["size_win"] + ~first
    full = z["size_win"] > w if c["fixed"] else z["size_init"] + z["size_sep"] + z["size_win"] == c["c"]
    full = full & ~first
    n_past = torch.where(full, z["size_win"] - w, torch.zeros_like(z["size_win"]))
    if s > 0:
        k = torch.arange(1 if c["fixed"] else ring - w, device=DEV)[None]
        src = a + s + (z["win_start"][:, None] + k) % ring
        moves = flag.gather(1, src) & (k < n_past[:, None])
        drop = (z["size_sep"] + moves.sum(1) - s).clamp(min=0)
        place = z["size_sep"][:, None] + moves.cumsum(1) - 1
        kept = moves & (place >= drop[:, None])
        dst = torch.where(kept, a + (z["sep_start"][:, None] + place) % s, torch.full_like(src, dump))
        for x in (*st["code"], *st["step"]):
            rows = _rows(x, src)
            x.scatter_(2, dst[:, None, :, None].expand_as(rows), rows)
        flag.scatter_(1, dst, torch.ones_like(kept))
        z["size_sep"] = z["size_sep"] + moves.sum(1) - drop
        z["sep_start"] = (z["sep_start"] + drop) % s
    z["win_start"] = (z["win_start"] + n_past) % ring
    z["size_win"] = z["size_win"] - n_past
    at, there = _entry_slots(z, c, c["c"])
    at = torch.where(there, at, torch.zeros_like(at))
    return _entries(st, *(_values(_rows(x, at), _rows(e, at)) for x, e in zip(st["code"], st["step"])), there)


def _entries(st, k, v, there):
    """Retained entries in 16 bits; other rows stay as they are."""
    for out, x in ((st["Kout"], k), (st["Vout"], v)):
        out.copy_(torch.where(there[:, None, :, None], x.to(torch.bfloat16), out))
    st["len"].copy_(there.sum(1))
    return st["Kout"], st["Vout"], st["len"]


def _plain_prompt(st):
    """What a prompt leaves: its first a tokens, its last ones from `lo` on, and the newest s separators
    between; lo and the separators held follow the compactions that the text went through."""
    c = st["case"]
    B, L, a, s, w = c["B"], c["L"], c["a"], c["s"], c["w"]
    sep, pos = _is_sep(st["ids"]), torch.arange(L, device=DEV)[None]
    T = st["prompt_len"].long() if st["prompt_len"] is not None else torch.full((B,), L, device=DEV)
    before = torch.nn.functional.pad((sep & (pos >= a)).cumsum(1), (1, 0))          # [B][L + 1]

    def count(at):
        return before.gather(1, at.clamp(0, L)[:, None])[:, 0]

    if c["fixed"]:
        lo = (T - w).clamp(min=a)
        held = (count(lo) - count(torch.full_like(lo, a))).clamp(max=s)
    else:
        lo, held = torch.full_like(T, a), torch.zeros_like(T)
        for _ in range(L // (c["c"] - a - s - w) + 1):
            full = c["c"] - a - held + lo              # tokens seen when the cache is full
            now = (T > a) & (full <= T)
            held = torch.where(now, (held + count(full - w) - count(lo)).clamp(max=s), held)
            lo = torch.where(now, full - w, lo)
    rank = before[:, 1:]                               # separators from a on, up to and with this position
    newest = sep & (pos >= a) & (pos < lo[:, None]) & (rank > (count(lo) - held)[:, None])
    kept = ((pos < a) | newest | (pos >= lo[:, None])) & (pos < T[:, None])
    n = min(c["c"], L)
    order = torch.sort((~kept).to(torch.uint8), dim=1, stable=True).indices[:, :n]   # kept positions first, in order
    there = torch.nn.functional.pad(kept.gather(1, order), (0, c["c"] - n))
    k, v = (torch.nn.functional.pad(_values(*_quantise(_rows(x, order))), (0, 0, 0, c["c"] - n))
            for x in (st["K"], st["V"]))
    return _entries(st, k, v, there)


_PLAIN = dict(norm_fwd=_plain_norm_fwd, norm_bwd=_plain_norm_bwd, decode=_plain_decode, append=_plain_append,
              prompt=_plain_prompt)


# ------------------------------------------------------------------------------------------ work
def work(case):
    """Inputs read once, outputs written once; two operations per product and sum."""
    c = case
    d = c["d"]
    if c["op"].startswith("norm"):
        tokens = c["B"] * c["L"]
        normed, all_ = tokens * (c["Hq"] + c["Hkv"]) * d, tokens * (c["Hq"] + 2 * c["Hkv"]) * d
        pos = 8 * tokens if c["far"] else 0
        if c["op"] == "norm_fwd":
            return {"bytes": 4 * all_ + pos, "flops": 7 * normed}
        return {"bytes": 2 * normed + all_ * ((4 if c["grad"] == "fp32" else 2) + 2) + pos, "flops": 15 * normed}
    held = 2 * (d // 2 + 2 * (d // GROUP))             # a cache entry of one kv head, K and V
    rows = c["B"] * c["Hkv"]
    if c["op"] == "decode":
        run_ = (c["lo"] + c["hi"]) / 2
        heads = c["B"] * c["Hq"]
        return {"bytes": rows * run_ * held + heads * (4 * d + 4), "flops": 4 * heads * run_ * d}
    if c["op"] == "append":
        run_ = (c["lo"] + c["hi"]) / 2
        return {"bytes": rows * (run_ * (held + 4 * d) + 4 * d + held), "flops": 2 * rows * run_ * d}
    T = c["L"] / 2 if c["ragged"] else c["L"]
    if c["fixed"]:
        run_ = min(T, c["a"] + c["w"]) + min(c["s"], c["rho"] * max(0, T - c["a"] - c["w"]))
    else:
        run_ = T if T < c["c"] else (c["a"] + c["s"] + c["w"] + c["c"]) / 2
    return {"bytes": rows * run_ * (4 * d + held + 4 * d), "flops": 6 * rows * run_ * d}


# ------------------------------------------------------------------------------------------ exact
def exact(case, seed):
    c = case
    st = prepare(case, seed)
    if own and "code" not in st and c["op"] in ("decode", "append"):
        st.update(_uncoded(case, seed))
    if c["op"].startswith("norm"):
        return _exact_norm(st)
    if c["op"] == "decode":
        return _exact_decode(st)
    return _exact_entries(st)


def _uncoded(case, seed):
    st = dict(case=case)
    _prepare_cache(case, _gen(seed), st)
    return st


def _exact_norm(st):
    """Every pair as a complex number, turned by exp(i angle); the gradient is taken through the
    definition of the forward."""
    c = st["case"]
    r, n = c["rot"], c["rot"] // 2
    freq = []
    for i in range(n):
        f = 1.0 / c["base"] ** (2 * i / r)
        if c["scaling"] == "linear":
            f /= c["factor"]
        elif c["scaling"] == "llama3":
            wave = 2 * math.pi / f
            if wave > c["orig"] / c["low"]:
                f /= c["factor"]
            elif wave >= c["orig"] / c["high"]:
                t = (c["orig"] / wave - c["low"]) / (c["high"] - c["low"])
                f = (1 - t) * f / c["factor"] + t * f
        freq.append(f)
    pos = st["positions"] if st["positions"] is not None else torch.arange(c["L"], device=DEV).expand(c["B"], -1)
    ang = pos.double()[:, :, None] * torch.tensor(freq, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.ones_like(ang), ang)

    def apply(x, w):
        """x [B][L][d] of one head"""
        y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["d"] + c["eps"]) * (w + c["offset"])
        if c["layout"] == "half":
            z = torch.complex(y[..., :n], y[..., n:r]) * turn
            return torch.cat((z.real, z.imag, y[..., r:]), -1)
        z = torch.complex(y[..., 0:r:2], y[..., 1:r:2]) * turn
        return torch.cat((torch.view_as_real(z).flatten(-2), y[..., r:]), -1)

    heads = st["qkv"].split((c["Hq"], c["Hkv"], c["Hkv"]), 2)
    if c["op"] == "norm_fwd":
        out = []
        for x, w in zip(heads, (st["wq"], st["wk"], None)):
            y = torch.empty((c["B"], x.shape[2], c["L"], c["d"]), dtype=torch.float64, device=DEV)
            for h in range(x.shape[2]):
                y[:, h] = x[:, :, h].double() if w is None else apply(x[:, :, h].double(), w.double())
            out.append(y)
        return out
    dqkv = torch.empty(st["qkv"].shape, dtype=torch.float64, device=DEV)
    sums, h0 = [], 0
    for x, dy, w in zip(heads, st["grads"], (st["wq"], st["wk"], None)):
        total = torch.zeros(c["d"], dtype=torch.float64, device=DEV)
        for h in range(x.shape[2]):
            if w is None:
                dqkv[:, :, h0 + h] = dy[:, h].double()
                continue
            xx, ww = x[:, :, h].double().requires_grad_(True), w.double().requires_grad_(True)
            with torch.enable_grad():
                gx, gw = torch.autograd.grad(apply(xx, ww), (xx, ww), dy[:, h].double())
            dqkv[:, :, h0 + h] = gx
            total += gw
        h0 += x.shape[2]
        if w is not None:
            sums.append(total)
    return dqkv, *sums


def _walk(z, b, c):
    """Slots that sequence b holds as initial, separator and neighbour entries, in order."""
    i, q, w, s0, w0 = (int(z[k][b]) for k in ("size_init", "size_sep", "size_win", "sep_start", "win_start"))
    return ([v for v in range(i)], [c["a"] + (s0 + v) % c["s"] for v in range(q)],
            [c["a"] + c["s"] + (w0 + v) % (c["c"] - c["a"]) for v in range(w)])


def _held(st, which, b, slots):
    """Values [Hkv][n][d] of entries, 64 bits."""
    at = torch.tensor(slots, dtype=torch.int64, device=DEV)
    code, step = st["code"][which][b][:, at].double(), st["step"][which][b][:, at].double()
    return code * step.repeat_interleave(GROUP, -1)


def _exact_decode(st):
    c = st["case"]
    G = c["Hq"] // c["Hkv"]
    o = torch.zeros((c["B"], c["Hkv"], G, c["d"]), dtype=torch.float64, device=DEV)
    lse = torch.full((c["B"], c["Hkv"], G), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(c["B"]):
        slots = sum(_walk(st["sizes"], b, c), [])
        if slots:
            q = st["q"][b].double().view(c["Hkv"], G, c["d"])
            s = q @ _held(st, 0, b, slots).transpose(-1, -2) / math.sqrt(c["d"])
            lse[b] = torch.logsumexp(s, -1)
            o[b] = torch.exp(s - lse[b][..., None]) @ _held(st, 1, b, slots)
    return o.view(c["B"], c["Hq"], c["d"]), lse.view(c["B"], c["Hq"])


def _nearest(x):
    """The values that rows of x are held as: of the 16 multiples -8 .. 7 of the group's step the
    nearest, of two as near the even one."""
    y = x.double().unflatten(-1, (-1, GROUP))
    size, sign = y.abs().amax(-1, keepdim=True), 1.0
    sign = torch.where((y == size).any(-1, keepdim=True), -1.0, 1.0)     # a positive largest element: code -8
    step = torch.where(size < FLUSH, torch.zeros_like(size), sign * size / 8)
    best, off = torch.zeros_like(y), torch.full_like(y, math.inf)
    for n in sorted(range(-8, 8), key=lambda n: n % 2):                  # even multiples first: they win ties
        e = (y - n * step).abs()
        best, off = torch.where(e < off, n * step, best), torch.minimum(e, off)
    return best.flatten(-2)


def _exact_entries(st):
    c = st["case"]
    a, s, w = c["a"], c["s"], c["w"]
    K, V = st["Kout"].double(), st["Vout"].double()
    n = []
    for b in range(c["B"]):
        if c["op"] == "append":
            init, sep, win = _walk(st["sizes"], b, c)
            flag = st["is_sep"][b].tolist()
            texts, flag = [(-1, int(st["new_ids"][b]) in SEP_IDS)], {x: flag[x] for x in init + sep + win}
        else:
            T = int(st["prompt_len"][b]) if st["prompt_len"] is not None else c["L"]
            init, sep, win, flag = [], [], [], {}
            texts = [(t, i in SEP_IDS) for t, i in enumerate(st["ids"][b, :T].tolist())]
        for t, is_sep in texts:                       # token by token
            flag[t] = is_sep
            if len(init) < a:
                init.append(t)
                continue
            win.append(t)
            if (len(win) > w) if c["fixed"] else (len(init) + len(sep) + len(win) == c["c"]):
                past, win = win[:-w], win[-w:]
                sep = (sep + [x for x in past if flag[x]])[-s:] if s else []
        held = init + sep + win
        n.append(len(held))
        for which, out in ((0, K), (1, V)):
            if c["op"] == "append":
                out[b, :, : len(held)] = _held(st, which, b, [max(x, 0) for x in held])
                if -1 in held:
                    new = (st["k_new"], st["v_new"])[which]
                    out[b, :, held.index(-1)] = _nearest(new[b])
            else:
                at = torch.tensor(held, dtype=torch.int64, device=DEV)
                out[b, :, : len(held)] = _nearest((st["K"], st["V"])[which][b][:, at])
    return K, V, torch.tensor(n, dtype=torch.int32, device=DEV)
