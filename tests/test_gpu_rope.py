"""sepllm_rope_fwd / sepllm_rope_bwd against the oracle's rotation in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, inputs
from tests._gpu_util import TOL_GRAD, TOL_O, attn_bwd, attn_fwd, assert_close, build_index, flags_of

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
HALF_STEP = {BF: 2.0 ** -8, F32: 2.0 ** -24}


def _check(got, x, pos, freq, layout, m, inverse, what=""):
    """|error| <= half a step of the output type + what 32 bits cost.  The angle, reduced to half a
    turn, carries 2^-24 * pi (its rounding) and up to 5e-7 rad (two 64-bit roundings of a product
    of 2^31 / 2 pi turns, here and in the oracle), its sine and cosine two steps of 2^-24 each, the
    two products and their sum three: under 2e-6 of m (|x| + |y|)."""
    n = len(freq)
    x = x.double().cpu().numpy()
    ref = orc.rope_apply(x, pos, freq, layout, m, inverse)
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    mag = np.zeros_like(ref)
    mag[..., a] = mag[..., b] = m * (np.abs(x[..., a]) + np.abs(x[..., b]))
    err = np.abs(got.double().cpu().numpy() - ref)
    tol = HALF_STEP[got.dtype] * np.abs(ref) * (1 + 2.0 ** -8) + 2e-6 * mag
    if got.dtype == F32:
        tol[..., 2 * n:] = 0.0   # copied
    assert (err <= tol).all(), (what, float((err - tol).max()))


def _tensors(g, B, L, Hq, Hkv, d, dtype, fused):
    if fused:
        t = torch.randn((B, L, Hq + 2 * Hkv, d), generator=g, device="cuda").to(dtype)
        return t, t.transpose(1, 2).split((Hq, Hkv, Hkv), 1)
    return None, [torch.randn((B, h, L, d), generator=g, device="cuda").to(dtype) for h in (Hq, Hkv, Hkv)]


def _outputs(B, L, Hq, Hkv, d, dtype, fused):
    if fused:
        t = torch.full((B, L, Hq + 2 * Hkv, d), float("nan"), dtype=dtype, device="cuda")
        return t.transpose(1, 2).split((Hq, Hkv, Hkv), 1)
    return [torch.full((B, h, L, d), float("nan"), dtype=dtype, device="cuda") for h in (Hq, Hkv, Hkv)]


CASES = [
    # B, L, Hq, Hkv, d, rot
    (1, 1, 1, 1, 64, 64), (3, 7, 4, 2, 64, 16), (2, 33, 5, 1, 80, 20), (2, 5, 3, 3, 80, 80), (1, 130, 2, 1, 96, 24),
    (2, 17, 4, 4, 112, 112), (2, 65, 8, 2, 128, 128), (1, 9, 10, 2, 128, 64), (2, 3, 2, 1, 128, 2),
    (1, 1000, 32, 8, 128, 128), (32, 1, 32, 8, 128, 128), (2, 6, 2, 1, 96, 40),
    (3, 11, 3, 1, 64, 6), (2, 13, 5, 2, 112, 90), (1, 25, 2, 2, 128, 118), (2, 10, 1, 1, 80, 78),
]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("B,L,Hq,Hkv,d,rot", CASES)
def test_forward_and_gradient(B, L, Hq, Hkv, d, rot, layout):
    g = torch.Generator(device="cuda").manual_seed(B * 1000 + L + d + rot)
    desc = api.RopeDesc(B, L, Hq, Hkv, d, rot_dim=rot, layout=layout, scaling="linear", factor=1.5, attn_factor=1.3)
    freq, m = api.sepllm_rope_frequencies(desc)
    pos = torch.randint(-50, 5000, (B, L), generator=g, device="cuda")
    pn = pos.cpu().numpy()[:, None]
    # the forward splits a fused projection, the gradient goes back into one, in both types
    for fn, fused_in, inverse in ((api.sepllm_rope_fwd, True, False), (api.sepllm_rope_bwd, False, True)):
        for din, dout in ((BF, BF), (F32, BF), (BF, F32), (F32, F32)):
            _, x = _tensors(g, B, L, Hq, Hkv, d, din, fused_in)
            y = _outputs(B, L, Hq, Hkv, d, dout, not fused_in)
            fn(desc, pos, *x, *y)
            torch.cuda.synchronize()
            for i in (0, 1):
                _check(y[i], x[i], pn, freq, layout, m, inverse, (fn.__name__, din, dout, i))
            assert torch.equal(y[2], x[2].to(dout))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("scaling,kw", [("none", {}), ("ntk", dict(factor=4.0)),
                                        ("yarn", dict(factor=4.0, high=32.0, orig_len=4096.0)),
                                        ("llama3", dict(factor=8.0, orig_len=8192.0)),
                                        ("factors", dict(freq_factors=np.linspace(1.0, 9.0, 64)))])
def test_stretched_frequencies_and_far_positions(scaling, kw, layout):
    """Positions up to 2^31 and behind zero; one row of positions for every sequence."""
    B, L = 2, 12
    desc = api.RopeDesc(B, L, 2, 1, 128, layout=layout, scaling=scaling, base=500000.0, pos_stride=0, **kw)
    freq, m = api.sepllm_rope_frequencies(desc)
    assert np.allclose(freq, orc.rope_frequencies(128, 500000.0, scaling, **kw), rtol=1e-13)
    pos = torch.tensor([0, 1, 127, 8191, 65535, 10 ** 6, 2 ** 24 + 1, 10 ** 8 + 7, 2 ** 31 - 1, 2 ** 31, -1, -(2 ** 30)],
                       device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    _, x = _tensors(g, B, L, 2, 1, 128, F32, False)
    y = _outputs(B, L, 2, 1, 128, F32, False)
    api.sepllm_rope_fwd(desc, pos, *x, *y)
    torch.cuda.synchronize()
    for i in (0, 1):
        _check(y[i], x[i], pos.cpu().numpy()[None, None], freq, layout, m, False, scaling)


def test_positions_from_a_first_one_and_tensors_left_out():
    B, L, Hq, Hkv, d = 2, 19, 3, 1, 64
    desc = api.RopeDesc(B, L, Hq, Hkv, d, pos_first=777)
    freq, m = api.sepllm_rope_frequencies(desc)
    g = torch.Generator(device="cuda").manual_seed(6)
    _, x = _tensors(g, B, L, Hq, Hkv, d, BF, False)
    y = _outputs(B, L, Hq, Hkv, d, BF, False)
    api.sepllm_rope_fwd(desc, None, None, x[1], None, None, y[1], None)      # keys alone
    api.sepllm_rope_fwd(desc, None, x[0], None, None, y[0], None, None)      # queries alone
    api.sepllm_rope_fwd(desc, None, None, None, x[2], None, None, y[2])      # values alone: a copy
    torch.cuda.synchronize()
    for i in (0, 1):
        _check(y[i], x[i], 777 + np.arange(L), freq, "half", m, False)
    assert torch.equal(y[2], x[2])


@pytest.mark.parametrize("rot,layout", [(64, "half"), (16, "interleaved"), (10, "half"), (6, "interleaved")])
def test_in_place_equals_out_of_place_and_back(rot, layout):
    B, L, Hq, Hkv, d = 2, 37, 4, 2, 64
    desc = api.RopeDesc(B, L, Hq, Hkv, d, rot_dim=rot, layout=layout)
    g = torch.Generator(device="cuda").manual_seed(7)
    t, x = _tensors(g, B, L, Hq, Hkv, d, F32, True)
    y = _outputs(B, L, Hq, Hkv, d, F32, False)
    api.sepllm_rope_fwd(desc, None, *x, *y)
    before = t.clone()
    api.sepllm_rope_fwd(desc, None, *x, *x)
    for a, b in zip(x, y):
        assert torch.equal(a, b)
    api.sepllm_rope_bwd(desc, None, *x, *x)
    # both rotations together: two times three roundings of 2^-24 and the angles' 2e-6, per pair
    assert ((t - before).abs() <= 1e-5 * (before.abs().amax())).all()
    assert torch.equal(t[..., rot:], before[..., rot:])


@pytest.mark.parametrize("rot,layout", [(64, "half"), (16, "half"), (24, "interleaved")])
def test_odd_strides_offsets_and_broadcast_inputs(rot, layout):
    """Views at odd element offsets and strides (no 16-byte accesses possible), inputs broadcast over
    the batch; the elements between the rows of the outputs stay as they are."""
    B, L, H, d = 3, 11, 2, 64
    desc = api.RopeDesc(B, L, H, H, d, rot_dim=rot, layout=layout)
    freq, m = api.sepllm_rope_frequencies(desc)
    g = torch.Generator(device="cuda").manual_seed(8)
    src = torch.randn(1 + H * L * 67, generator=g, device="cuda").to(BF)
    x = src.as_strided((B, H, L, d), (0, L * 67, 67, 1), 1)
    buf = torch.full((3 + B * H * L * 71,), -7.0, dtype=BF, device="cuda")
    y = buf.as_strided((B, H, L, d), (H * L * 71, L * 71, 71, 1), 3)
    ref = torch.empty((B, H, L, d), dtype=BF, device="cuda")
    api.sepllm_rope_fwd(desc, None, x, None, x, y, None, ref)
    torch.cuda.synchronize()
    _check(y, x, np.arange(L), freq, layout, m, False)
    assert torch.equal(ref, x)
    gap = torch.ones_like(buf, dtype=torch.bool)
    gap.as_strided((B, H, L, d), (H * L * 71, L * 71, 71, 1), 3).fill_(False)
    assert (buf[gap] == -7.0).all()


def test_non_finite_values_stay_in_their_pair():
    """A NaN or infinity reaches its own pair only; copied elements are exact whatever they hold."""
    for layout, rot in (("half", 32), ("interleaved", 32), ("half", 20), ("interleaved", 20)):
        desc = api.RopeDesc(1, 4, 2, 1, 64, rot_dim=rot, layout=layout)
        x = torch.ones((1, 2, 4, 64), dtype=BF, device="cuda")
        x[0, 0, 1, 3] = float("nan")
        x[0, 1, 2, 40] = float("inf")
        x[0, 1, 3, 41] = float("nan")
        y = torch.empty_like(x)
        api.sepllm_rope_fwd(desc, None, x, None, None, y, None, None)
        bad = ~torch.isfinite(y)
        pair = (3, 3 + rot // 2) if layout == "half" else (2, 3)
        want = {(0, 0, 1, pair[0]), (0, 0, 1, pair[1]), (0, 1, 2, 40), (0, 1, 3, 41)}
        assert {tuple(i) for i in bad.nonzero().tolist()} == want
        assert torch.isinf(y[0, 1, 2, 40])


def test_offsets_past_two_to_the_31():
    """Sequence 1 of a view starts more than 2^31 elements behind sequence 0."""
    far, B, L, H, d = 2 ** 31 + 8, 2, 3, 1, 64
    desc = api.RopeDesc(B, L, H, H, d)
    freq, m = api.sepllm_rope_frequencies(desc)
    buf = torch.empty(far + L * d, dtype=BF, device="cuda")
    y = buf.as_strided((B, H, L, d), (far, L * d, d, 1))
    x = torch.randn((B, H, L, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(9)).to(BF)
    api.sepllm_rope_fwd(desc, None, x, None, None, y, None, None)
    z = torch.empty_like(x)
    api.sepllm_rope_bwd(desc, None, y, None, None, z, None, None)
    torch.cuda.synchronize()
    _check(y, x, np.arange(L), freq, "half", m, False)
    _check(z, y, np.arange(L), freq, "half", m, True)


def test_captured_in_a_graph_and_on_another_stream():
    B, L, Hq, Hkv, d = 2, 50, 4, 2, 128
    desc = api.RopeDesc(B, L, Hq, Hkv, d)
    freq, m = api.sepllm_rope_frequencies(desc)
    g = torch.Generator(device="cuda").manual_seed(10)
    t, x = _tensors(g, B, L, Hq, Hkv, d, BF, True)
    y = _outputs(B, L, Hq, Hkv, d, BF, False)
    pos = torch.randint(0, 100, (B, L), generator=g, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        api.sepllm_rope_fwd(desc, pos, *x, *y)
    torch.cuda.synchronize()
    _check(y[0], x[0], pos.cpu().numpy()[:, None], freq, "half", m, False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.sepllm_rope_fwd(desc, pos, *x, *y)
    for k in range(2):     # replays read what the buffers hold then
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        pos.add_(1000 + k)
        graph.replay()
        torch.cuda.synchronize()
        for i in (0, 1):
            _check(y[i], x[i], pos.cpu().numpy()[:, None], freq, "half", m, False)
        assert torch.equal(y[2], x[2])


@pytest.mark.parametrize("layout,d,rot,Hq,Hkv", [("half", 64, 16, 4, 4), ("interleaved", 128, 128, 4, 1)])
def test_a_training_step_through_the_rotation(layout, d, rot, Hq, Hkv):
    """Fused projection -> rotation -> separator-masked attention -> its gradients -> rotation back,
    as one run, against the oracle of the whole."""
    B, L, a, n = 2, 200, 3, 24
    ids = inputs.token_ids(31, B, L, 0.15)
    f = flags_of(ids, inputs.SEP_IDS)
    idesc, index = build_index(ids, inputs.SEP_IDS, a, n)
    g = torch.Generator(device="cuda").manual_seed(11)
    _, x = _tensors(g, B, L, Hq, Hkv, d, BF, True)
    dO = torch.randn((B, Hq, L, d), generator=g, device="cuda").to(BF)
    desc = api.RopeDesc(B, L, Hq, Hkv, d, rot_dim=rot, layout=layout, base=10000.0)
    freq, m = api.sepllm_rope_frequencies(desc)
    Q, K, V = _outputs(B, L, Hq, Hkv, d, BF, False)
    api.sepllm_rope_fwd(desc, None, *x, Q, K, V)
    O, LSE = attn_fwd(Q, K, V, idesc, index)
    grads = attn_bwd(dO, Q, K, V, O, LSE, idesc, index, grad_dtype=1)
    out = _outputs(B, L, Hq, Hkv, d, BF, True)
    api.sepllm_rope_bwd(desc, None, *grads, *out)
    torch.cuda.synchronize()
    pos = np.arange(L)
    for i, z in ((0, Q), (1, K)):
        _check(z, x[i], pos, freq, layout, m, False)
    Qn, Kn, Vn, dOn = (z.double().cpu().numpy() for z in (Q, K, V, dO))
    Oref, _ = orc.attn_fwd(Qn, Kn, Vn, f, a, n)
    assert_close(O.float().cpu().numpy(), Oref, TOL_O, "O")
    refs = orc.attn_bwd(Qn, Kn, Vn, dOn, f, a, n)
    for i, (got, ref) in enumerate(zip(out, refs)):
        if i < 2:
            _check(got, grads[i], pos, freq, layout, m, True)
            ref = orc.rope_apply(ref, pos, freq, layout, m, inverse=True)
        ref_err = np.linalg.norm(got.double().cpu().numpy() - ref) / np.linalg.norm(ref)
        # a rotation keeps the norm of the attention gradient's error; the bf16 output adds 2^-8 at most
        assert ref_err <= TOL_GRAD["rel_fro"] + 2.0 ** -8, (i, ref_err)
