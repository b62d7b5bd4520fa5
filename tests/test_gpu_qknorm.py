"""sepllm_qknorm_rope_fwd / sepllm_qknorm_rope_bwd against the oracle's norm, rotation and gradient in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, inputs
from tests._gpu_util import TOL_GRAD, TOL_O, assert_close, attn_bwd, attn_fwd, build_index, flags_of

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
HALF_STEP = {BF: 2.0 ** -8, F32: 2.0 ** -24}


def _np(t):
    return t.double().cpu().numpy()


def _pair_size(y, n, layout, m):
    """|a| + |b| of every rotated pair times m; |y| of the other elements."""
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    mag = np.abs(y)
    s = m * (mag[..., a] + mag[..., b])
    mag[..., a] = mag[..., b] = s
    return mag


def check_fwd(got, x, w, eps, offset, pos, freq, layout, m, what=""):
    """Half a step of the output's type, and what 32 bits cost: the sum of squares of up to 128 elements (16 in a
    row, then a tree: 24 roundings of 2^-24 at most, half of it in r), the root (two steps of 2^-23), three
    products: 2e-6 relative; the rotation's 2e-6 of the pair (as for the rotation alone): 4e-6 in all."""
    y = orc.head_norm(_np(x), None if w is None else _np(w), eps, offset)
    ref = orc.rope_apply(y, pos, freq, layout, m)
    tol = HALF_STEP[got.dtype] * np.abs(ref) + 4e-6 * _pair_size(y, len(freq), layout, m)
    err = np.abs(_np(got) - ref)
    assert (err <= tol).all(), (what, float((err - tol).max()))


def check_bwd(dx, dw, x, w, dy, eps, offset, pos, freq, layout, m, what=""):
    """As above with a second sum over the head: 6e-6 of the terms' sizes.  Sums for the weights: 6e-6 of
    the terms, and at most 256 additions behind one another of 2^-24 of their sizes' sum (2e-5 in all)."""
    xn, n = _np(x), len(freq)
    g = orc.rope_apply(_np(dy), pos, freq, layout, m, inverse=True)
    size = _pair_size(_np(dy), n, layout, m)
    rx, rw = orc.head_norm_bwd(xn, None if w is None else _np(w), g, eps, offset)
    wn = np.ones(xn.shape[-1]) if w is None else offset + _np(w)
    r = 1.0 / np.sqrt((xn * xn).mean(-1, keepdims=True) + eps)
    nn = np.abs(xn * r)
    mag = r * (size * np.abs(wn) + nn * (nn * size * np.abs(wn)).mean(-1, keepdims=True))
    err = np.abs(_np(dx) - rx)
    tol = HALF_STEP[dx.dtype] * np.abs(rx) + 6e-6 * mag
    assert (err <= tol).all(), (what, float((err - tol).max()))
    if dw is not None:
        tol = 2e-5 * (size * nn).reshape(-1, xn.shape[-1]).sum(0) + 1e-30
        assert (np.abs(_np(dw) - rw) <= tol).all(), (what, float((np.abs(_np(dw) - rw) / tol).max()))


def _tensors(g, B, L, Hq, Hkv, d, dtype, fused):
    """Heads of different sizes, as a fused projection or as three tensors."""
    size = torch.exp(torch.randn((1, 1, Hq + 2 * Hkv, 1), generator=g, device="cuda"))
    t = (torch.randn((B, L, Hq + 2 * Hkv, d), generator=g, device="cuda") * size).to(dtype)
    views = t.transpose(1, 2).split((Hq, Hkv, Hkv), 1)
    return views if fused else [v.contiguous() for v in views]


def _outputs(B, L, Hq, Hkv, d, dtype, fused):
    t = torch.full((B, L, Hq + 2 * Hkv, d), float("nan"), dtype=dtype, device="cuda")
    views = t.transpose(1, 2).split((Hq, Hkv, Hkv), 1)
    return views if fused else [v.contiguous() for v in views]


def _weights(g, d, dtype, offset):
    return [(1.0 - offset + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dtype) for _ in "qk"]


def run_bwd(desc, norm, pos, x, dy, dx, want=(True, True)):
    ws = api.alloc_bytes(api.sepllm_qknorm_rope_bwd_workspace_bytes(desc))
    ws.fill_(0xFF)                               # (NaN bit patterns: nothing of it may be read before it is written)
    dw = [torch.full((desc.d,), float("nan"), device="cuda") if k else None for k in want]
    api.sepllm_qknorm_rope_bwd(desc, norm, pos, x[0], x[1], *dy, *dx, *dw, ws)
    torch.cuda.synchronize()
    return dw


CASES = [
    # B, L, Hq, Hkv, d, rot
    (1, 1, 1, 1, 64, 64), (3, 7, 4, 2, 64, 16), (2, 33, 5, 1, 80, 20), (2, 5, 3, 3, 80, 80), (1, 130, 2, 1, 96, 32),
    (2, 17, 4, 4, 112, 112), (2, 65, 8, 2, 128, 128), (1, 9, 10, 2, 128, 64), (2, 3, 2, 1, 128, 2),
    (1, 700, 32, 8, 128, 128), (32, 1, 32, 8, 128, 128), (2, 6, 2, 1, 96, 40),
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
    for i, (dx_t, dy_t) in enumerate(((BF, BF), (F32, BF), (BF, F32), (F32, F32))):
        offset = float(i % 2)
        w = _weights(g, d, (BF, F32)[i // 2], offset)
        norm = api.QkNorm(*w, eps=1e-5, offset=offset)
        x = _tensors(g, B, L, Hq, Hkv, d, dx_t, True)
        y = _outputs(B, L, Hq, Hkv, d, dy_t, False)
        api.sepllm_qknorm_rope_fwd(desc, norm, pos, *x, *y)
        torch.cuda.synchronize()
        for k in (0, 1):
            check_fwd(y[k], x[k], w[k], norm.eps, offset, pn, freq, layout, m, (i, k))
        assert torch.equal(y[2], x[2].to(dy_t))
        dy = _tensors(g, B, L, Hq, Hkv, d, dy_t, False)
        dx = _outputs(B, L, Hq, Hkv, d, dx_t, True)
        dw = run_bwd(desc, norm, pos, x, dy, dx)
        for k in (0, 1):
            check_bwd(dx[k], dw[k], x[k], w[k], dy[k], norm.eps, offset, pn, freq, layout, m, (i, k))
        assert torch.equal(dx[2], dy[2].to(dx_t))


@pytest.mark.parametrize("rot,layout", [(128, "half"), (64, "interleaved"), (20, "half")])
def test_gradient_against_differences(rot, layout):
    """The gradient's inner product with a direction against the forward's change along it, in 32 bits.  The
    step's relative error: the forward's 4e-6 of the outputs' sizes over the step of 1/64, and the third
    derivative's share, (1/64)^2 / 6 of the terms' sizes (with |direction| up to 4, sizes of a few)."""
    B, L, Hq, Hkv, d, eps = 2, 9, 3, 1, 128, 0.05
    g = torch.Generator(device="cuda").manual_seed(12)
    desc = api.RopeDesc(B, L, Hq, Hkv, d, rot_dim=rot, layout=layout)
    w = _weights(g, d, F32, 0.0)
    x = [torch.randn(s, generator=g, device="cuda") for s in ((B, Hq, L, d), (B, Hkv, L, d), (B, Hkv, L, d))]
    dy, v = ([torch.randn(t.shape, generator=g, device="cuda") for t in x] for _ in range(2))
    vw = [torch.randn(d, generator=g, device="cuda") for _ in "qk"]
    dx = [torch.empty_like(t) for t in x]
    dw = run_bwd(desc, api.QkNorm(*w, eps=eps), None, x, dy, dx)

    def loss(sign, h=1.0 / 64):
        xs, y = [t + sign * h * u for t, u in zip(x, v)], [torch.empty_like(t) for t in x]
        ws = [t + sign * h * u for t, u in zip(w, vw)]
        api.sepllm_qknorm_rope_fwd(desc, api.QkNorm(*ws, eps=eps), None, *xs, *y)
        return [(a.double() * b.double()).sum() / h for a, b in zip(y, dy)]
    up, down = loss(1.0), loss(-1.0)
    for k in range(3):
        got = (dx[k].double() * v[k].double()).sum() + ((dw[k].double() * vw[k].double()).sum() if k < 2 else 0.0)
        size = float((dy[k].double().abs() * 4).sum())
        assert abs(float((up[k] - down[k]) / 2 - got)) <= size * (4e-6 * 64 + 64.0 ** -2)


def test_without_weights_and_with_tensors_left_out():
    B, L, Hq, Hkv, d = 2, 19, 3, 1, 64
    desc = api.RopeDesc(B, L, Hq, Hkv, d, pos_first=777)
    freq, m = api.sepllm_rope_frequencies(desc)
    g = torch.Generator(device="cuda").manual_seed(6)
    pos = 777 + np.arange(L)
    w = _weights(g, d, BF, 0.0)
    x, y = _tensors(g, B, L, Hq, Hkv, d, BF, False), _outputs(B, L, Hq, Hkv, d, BF, False)
    none, only_k = api.QkNorm(eps=1e-5, offset=5.0), api.QkNorm(None, w[1], eps=1e-5)
    api.sepllm_qknorm_rope_fwd(desc, only_k, None, None, x[1], None, None, y[1], None)     # keys alone
    api.sepllm_qknorm_rope_fwd(desc, none, None, x[0], None, None, y[0], None, None)       # queries alone
    api.sepllm_qknorm_rope_fwd(desc, none, None, None, None, x[2], None, None, y[2])       # values alone: a copy
    torch.cuda.synchronize()
    check_fwd(y[0], x[0], None, 1e-5, 0.0, pos, freq, "half", m)
    check_fwd(y[1], x[1], w[1], 1e-5, 0.0, pos, freq, "half", m)
    assert torch.equal(y[2], x[2])
    dy, dx = _tensors(g, B, L, Hq, Hkv, d, BF, False), _outputs(B, L, Hq, Hkv, d, BF, False)
    dw = run_bwd(desc, only_k, None, x, dy, dx, (False, True))
    check_bwd(dx[0], None, x[0], None, dy[0], 1e-5, 0.0, pos, freq, "half", m)
    check_bwd(dx[1], dw[1], x[1], w[1], dy[1], 1e-5, 0.0, pos, freq, "half", m)
    # keys alone; weights whose tensor is left out get zeros
    both = api.QkNorm(*w, eps=1e-5)
    dx1 = torch.empty_like(dx[1])
    dw2 = run_bwd(desc, both, None, (None, x[1]), (None, dy[1], None), (None, dx1, None))
    assert torch.equal(dx1, dx[1]) and torch.equal(dw2[1], dw[1]) and (dw2[0] == 0).all()
    # no gradient of the weights wanted
    run_bwd(desc, both, None, x, dy, dx, (False, False))
    check_bwd(dx[0], None, x[0], w[0], dy[0], 1e-5, 0.0, pos, freq, "half", m)


@pytest.mark.parametrize("rot,layout", [(64, "half"), (16, "interleaved"), (10, "half")])
def test_in_place(rot, layout):
    """Outputs over the inputs; gradients over the gradients that came in, and over the forward's inputs."""
    B, L, Hq, Hkv, d = 2, 37, 4, 2, 64
    desc = api.RopeDesc(B, L, Hq, Hkv, d, rot_dim=rot, layout=layout)
    g = torch.Generator(device="cuda").manual_seed(7)
    norm = api.QkNorm(*_weights(g, d, F32, 0.0))
    x, y = _tensors(g, B, L, Hq, Hkv, d, BF, False), _outputs(B, L, Hq, Hkv, d, BF, False)
    dy, dx = _tensors(g, B, L, Hq, Hkv, d, BF, False), _outputs(B, L, Hq, Hkv, d, BF, False)
    api.sepllm_qknorm_rope_fwd(desc, norm, None, *x, *y)
    dw = run_bwd(desc, norm, None, x, dy, dx)
    x2, dy2, x3 = ([t.clone() for t in ts] for ts in (x, dy, x))
    api.sepllm_qknorm_rope_fwd(desc, norm, None, *x2, *x2)
    dwa = run_bwd(desc, norm, None, x, dy2, dy2)
    dwb = run_bwd(desc, norm, None, x3, dy, (x3[0], x3[1], x3[2]))
    for a, b, c, e, f in zip(x2, y, dy2, x3, dx):
        assert torch.equal(a, b) and torch.equal(c, f) and torch.equal(e, f)
    for a, b, c in zip(dw, dwa, dwb):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("rot,layout", [(64, "half"), (24, "interleaved")])
def test_odd_strides_offsets_and_broadcast_inputs(rot, layout):
    """Views at odd element offsets and strides, inputs and gradients broadcast over the batch; the elements
    between the rows of the outputs stay as they are."""
    B, L, H, d = 3, 11, 2, 64
    desc = api.RopeDesc(B, L, H, H, d, rot_dim=rot, layout=layout)
    freq, m = api.sepllm_rope_frequencies(desc)
    g = torch.Generator(device="cuda").manual_seed(8)
    w = _weights(g, d, BF, 1.0)
    wide = [torch.randn(d + 1, generator=g, device="cuda").to(BF) for _ in "qk"]
    w = [t[1:].copy_(s) for t, s in zip(wide, w)]                # weights at an odd address
    norm = api.QkNorm(*w, eps=1e-5, offset=1.0)
    src = torch.randn(1 + H * L * 67, generator=g, device="cuda").to(BF)
    x = src.as_strided((B, H, L, d), (0, L * 67, 67, 1), 1)
    gap = torch.ones(3 + B * H * L * 71, dtype=torch.bool, device="cuda")
    shape = ((B, H, L, d), (H * L * 71, L * 71, 71, 1), 3)
    gap.as_strided(*shape).fill_(False)
    for call in ("fwd", "bwd"):
        buf = torch.full((3 + B * H * L * 71,), -7.0, dtype=BF, device="cuda")
        y, other = buf.as_strided(*shape), torch.empty((B, H, L, d), dtype=BF, device="cuda")
        if call == "fwd":
            api.sepllm_qknorm_rope_fwd(desc, norm, None, x, x, None, y, other, None)
            torch.cuda.synchronize()
            check_fwd(y, x, w[0], 1e-5, 1.0, np.arange(L), freq, layout, m)
            check_fwd(other, x, w[1], 1e-5, 1.0, np.arange(L), freq, layout, m)
        else:
            dy = torch.randn((1, H, L, d), generator=g, device="cuda").expand(B, H, L, d)
            dw = run_bwd(desc, norm, None, (x, x), (dy, dy, None), (y, other, None))
            check_bwd(y, dw[0], x, w[0], dy, 1e-5, 1.0, np.arange(L), freq, layout, m)
            check_bwd(other, dw[1], x, w[1], dy, 1e-5, 1.0, np.arange(L), freq, layout, m)
        assert (buf[gap] == -7.0).all()


@pytest.mark.parametrize("rot,layout", [(32, "half"), (20, "half"), (32, "interleaved")])
def test_rows_of_zeros_small_rows_and_numbers_that_are_not_finite(rot, layout):
    """A row of zeros gives zeros (and the gradient r u); rows far below and above 1; a NaN or infinity reaches its
    own row and the weights' gradient, and no other row."""
    B, L, H, d, eps = 1, 6, 2, 64, 1e-6
    desc = api.RopeDesc(B, L, H, 1, d, rot_dim=rot, layout=layout)
    freq, m = api.sepllm_rope_frequencies(desc)
    g = torch.Generator(device="cuda").manual_seed(9)
    w = _weights(g, d, F32, 0.0)
    norm = api.QkNorm(*w, eps=eps)
    x = torch.randn((B, H, L, d), generator=g, device="cuda")
    x[0, 0, 1] = 0
    x[0, 0, 2] *= 1e-10
    x[0, 0, 3] *= 1e15
    x[0, 0, 4] *= 1e-4
    dy, dx, y = torch.randn(x.shape, generator=g, device="cuda"), torch.empty_like(x), torch.empty_like(x)
    api.sepllm_qknorm_rope_fwd(desc, norm, None, x, None, None, y, None, None)
    dw = run_bwd(desc, norm, None, (x, None), (dy, None, None), (dx, None, None))
    check_fwd(y, x, w[0], eps, 0.0, np.arange(L), freq, layout, m)
    check_bwd(dx, dw[0], x, w[0], dy, eps, 0.0, np.arange(L), freq, layout, m)
    assert (y[0, 0, 1] == 0).all() and (dw[1] == 0).all()
    x2, dy2 = x.clone(), dy.clone()
    x2[0, 1, 2, 3] = float("nan")
    x2[0, 0, 5, 60] = float("inf")
    dy2[0, 1, 4, 63] = float("inf")
    y2, dx2 = torch.empty_like(x), torch.empty_like(x)
    api.sepllm_qknorm_rope_fwd(desc, norm, None, x2, None, None, y2, None, None)
    run_bwd(desc, norm, None, (x2, None), (dy2, None, None), (dx2, None, None))
    rows = torch.ones((B, H, L), dtype=torch.bool, device="cuda")
    rows[0, 1, 2] = rows[0, 0, 5] = False
    assert torch.equal(y2[rows], y[rows]) and torch.isnan(y2[0, 1, 2]).all() and torch.isnan(y2[0, 0, 5]).any()
    rows[0, 1, 4] = False
    assert torch.equal(dx2[rows], dx[rows]) and not torch.isfinite(dx2[~rows]).all()


def test_offsets_past_two_to_the_31():
    """Sequence 1 of a view starts more than 2^31 elements behind sequence 0."""
    far, B, L, H, d = 2 ** 31 + 8, 2, 3, 1, 64
    desc = api.RopeDesc(B, L, H, H, d)
    freq, m = api.sepllm_rope_frequencies(desc)
    g = torch.Generator(device="cuda").manual_seed(10)
    w = _weights(g, d, BF, 0.0)
    norm = api.QkNorm(*w)
    buf = torch.empty(far + L * d, dtype=BF, device="cuda")
    y = buf.as_strided((B, H, L, d), (far, L * d, d, 1))
    x, dy = (torch.randn((B, H, L, d), device="cuda", generator=g).to(BF) for _ in range(2))
    api.sepllm_qknorm_rope_fwd(desc, norm, None, x, None, None, y, None, None)
    torch.cuda.synchronize()
    check_fwd(y, x, w[0], norm.eps, 0.0, np.arange(L), freq, "half", m)
    y.copy_(x)
    dx = torch.empty_like(x)
    dw = run_bwd(desc, norm, None, (y, None), (dy, None, None), (dx, None, None))
    check_bwd(dx, dw[0], x, w[0], dy, norm.eps, 0.0, np.arange(L), freq, "half", m)
    dw2 = run_bwd(desc, norm, None, (x, None), (dy, None, None), (y, None, None))
    assert torch.equal(y, dx) and torch.equal(dw[0], dw2[0])


def test_captured_in_a_graph_on_two_streams_and_the_same_every_time():
    B, L, Hq, Hkv, d = 2, 300, 8, 2, 128
    desc = api.RopeDesc(B, L, Hq, Hkv, d)
    freq, m = api.sepllm_rope_frequencies(desc)
    runs = []
    for k in range(2):
        g = torch.Generator(device="cuda").manual_seed(20 + k)
        w = _weights(g, d, BF, 0.0)
        norm = api.QkNorm(*w)
        x, y = _tensors(g, B, L, Hq, Hkv, d, BF, True), _outputs(B, L, Hq, Hkv, d, BF, False)
        dy, dx = _tensors(g, B, L, Hq, Hkv, d, F32, False), _outputs(B, L, Hq, Hkv, d, BF, True)
        dw = [torch.empty(d, device="cuda") for _ in "qk"]
        ws = api.alloc_bytes(api.sepllm_qknorm_rope_bwd_workspace_bytes(desc))
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            api.sepllm_qknorm_rope_fwd(desc, norm, None, *x, *y)
            api.sepllm_qknorm_rope_bwd(desc, norm, None, x[0], x[1], *dy, *dx, *dw, ws)
        runs.append((g, w, norm, x, y, dy, dx, dw, ws, stream, graph))
    for _ in range(3):
        for g, w, norm, x, y, dy, *_ in runs:
            for t in (*x, *dy, *w):
                t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        torch.cuda.synchronize()
        for *_, stream, graph in runs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for g, w, norm, x, y, dy, dx, dw, *_ in runs:
            for i in (0, 1):
                check_fwd(y[i], x[i], w[i], norm.eps, 0.0, np.arange(L), freq, "half", m)
                check_bwd(dx[i], dw[i], x[i], w[i], dy[i], norm.eps, 0.0, np.arange(L), freq, "half", m)
            dx2 = _outputs(B, L, Hq, Hkv, d, BF, True)
            dw2 = run_bwd(desc, norm, None, x, dy, dx2)
            for a, b in zip((*dx, *dw), (*dx2, *dw2)):
                assert torch.equal(a, b)


@pytest.mark.parametrize("layout,d,rot,Hq,Hkv", [("half", 64, 16, 4, 4), ("interleaved", 128, 128, 4, 1)])
def test_a_training_step_through_norm_and_rotation(layout, d, rot, Hq, Hkv):
    """Fused projection -> norm and rotation -> separator-masked attention -> its gradients -> back, as one
    run, against the oracle of the whole."""
    B, L, a, n, eps = 2, 200, 3, 24, 1e-6
    ids = inputs.token_ids(31, B, L, 0.15)
    f = flags_of(ids, inputs.SEP_IDS)
    idesc, index = build_index(ids, inputs.SEP_IDS, a, n)
    g = torch.Generator(device="cuda").manual_seed(11)
    w = _weights(g, d, F32, 0.0)
    norm = api.QkNorm(*w, eps=eps)
    x = _tensors(g, B, L, Hq, Hkv, d, BF, True)
    dO = torch.randn((B, Hq, L, d), generator=g, device="cuda").to(BF)
    desc = api.RopeDesc(B, L, Hq, Hkv, d, rot_dim=rot, layout=layout, base=10000.0)
    freq, m = api.sepllm_rope_frequencies(desc)
    Q, K, V = _outputs(B, L, Hq, Hkv, d, BF, False)
    api.sepllm_qknorm_rope_fwd(desc, norm, None, *x, Q, K, V)
    O, LSE = attn_fwd(Q, K, V, idesc, index)
    grads = attn_bwd(dO, Q, K, V, O, LSE, idesc, index, grad_dtype=1)
    out = _outputs(B, L, Hq, Hkv, d, BF, True)
    dw = run_bwd(desc, norm, None, x, grads, out)
    pos = np.arange(L)
    Qn, Kn, Vn, dOn = (_np(z) for z in (Q, K, V, dO))
    Oref, _ = orc.attn_fwd(Qn, Kn, Vn, f, a, n)
    assert_close(_np(O), Oref, TOL_O, "O")
    refs = orc.attn_bwd(Qn, Kn, Vn, dOn, f, a, n)
    for i, ref in enumerate(refs):
        if i < 2:
            check_fwd((Q, K)[i], x[i], w[i], eps, 0.0, pos, freq, layout, m)
            check_bwd(out[i], dw[i], x[i], w[i], grads[i], eps, 0.0, pos, freq, layout, m)
            gref, wref = orc.head_norm_bwd(_np(x[i]), _np(w[i]), orc.rope_apply(ref, pos, freq, layout, m, True), eps)
            # the weights' gradient is linear in the attention's, whose error is at most 1e-2 of its norm
            n2 = np.linalg.norm(ref) * np.linalg.norm(orc.head_norm(_np(x[i]), None, eps))
            assert np.linalg.norm(_np(dw[i]) - wref) <= TOL_GRAD["rel_fro"] * n2
            # each row's map has norm r max|w|: the attention gradient's error row by row
            r = 1.0 / np.sqrt((_np(x[i]) ** 2).mean(-1) + eps)
            bound = np.sqrt(((r * np.linalg.norm(_np(grads[i]) - ref, axis=-1)) ** 2).sum()) * np.abs(_np(w[i])).max()
            assert np.linalg.norm(_np(out[i]) - gref) <= 1.01 * bound + 2.0 ** -8 * np.linalg.norm(gref)
        else:
            assert np.linalg.norm(_np(out[i]) - ref) <= (TOL_GRAD["rel_fro"] + 2.0 ** -8) * np.linalg.norm(ref)
