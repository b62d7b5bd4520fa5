"""Gradients of the head norms against differences of the forward, row by row; and, on the CPU, that the comparison
notices a gradient with a term left out."""
import numpy as np
import pytest
import torch

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api
from tests.test_gpu_qknorm import _pair_size

B, H, L, D, EPS, H_STEP, RHO = 2, 3, 9, 128, 0.05, 1.0 / 64, 0.25
ROTATIONS = [(128, "half"), (64, "interleaved"), (20, "half")]


def grid(g, *shape):
    """Normal numbers in steps of 2^-8: with a power of two times one of them added, still exact in 32 bits."""
    return np.rint(g.normal(size=shape) * 256) / 256


def data(rot):
    g = np.random.default_rng(rot)
    desc = api.RopeDesc(B, L, H, 1, D, rot_dim=rot)
    x, dy = grid(g, B, H, L, D), grid(g, B, H, L, D)
    return desc, x, 1 + grid(g, D) / 4, dy, {"along x": x, "any": grid(g, B, H, L, D)}


def ratios(forward, dx, dw, x, w, dy, directions, n, layout):
    """How far dx and dw are off, over the bounds: for each row and direction the slope of sum(dy y) along it, and for
    some weights the slope along each.  forward(x, w): outputs whose errors are 4e-6 of a rotated pair's size at most.

    Slope along v: the central differences at h and h / 2, extrapolated.  Outputs' errors enter (4 * 2 + 1) / 3 times over h.
    With t complex, |t| <= rho, the sum of (x + t v)^2 has a real part of at least |x|^2 - 2 rho |x v| - rho^2 |v|^2, so
    |sum dy y| <= M = sum |g w| (|x| + rho |v|) r(that), its k-th coefficient is at most M / rho^k, and what the
    extrapolation leaves of them is below M / rho * (h / rho)^4 / 2.  dx itself: 6e-6 of its terms.  The slope along a
    weight is a difference without a remainder, of two elements of each row; dw itself: 2e-5 of its terms."""
    h, out = H_STEP, []
    size_g = _pair_size(dy, n, layout, 1.0)
    rounding = lambda y: 4e-6 * (np.abs(dy) * _pair_size(y, n, layout, 1.0))  # noqa: E731
    norm = lambda x, w: orc.head_norm(x, w, EPS)  # noqa: E731
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
    mag = r * size_g * np.abs(w)
    mag = mag + np.abs(x) * r ** 2 * (np.abs(x) * mag).mean(-1, keepdims=True)
    for v in directions.values():
        def central(h):
            up, down = forward(x + h * v, w), forward(x - h * v, w)
            return ((up - down) * dy).sum(-1) / (2 * h)
        slope = (4 * central(h / 2) - central(h)) / 3
        low = (x * x).sum(-1) - 2 * RHO * np.abs((x * v).sum(-1)) - RHO ** 2 * (v * v).sum(-1)
        most = (size_g * np.abs(w) * (np.abs(x) + RHO * np.abs(v))).sum(-1) / np.sqrt(low / D + EPS)
        assert (low > 0).all()
        widest = sum(rounding(norm(x + s * h * v, w)) for s in (1, -1)) / 2 + rounding(norm(x, w))
        tol = 3 / h * widest.sum(-1) + most / RHO * (h / RHO) ** 4 / 2 + 6e-6 * (mag * np.abs(v)).sum(-1)
        out.append(np.abs((dx * v).sum(-1) - slope) / tol)
    for k in (0, 9, 19, 63, 64, 100, 127):
        e = np.zeros(D)
        e[k] = 0.25
        up, down = forward(x, w + e), forward(x, w - e)
        err = sum((rounding(norm(x, w + s * e)) * (up != down)).sum() for s in (1, -1)) / 0.5
        tol = err + 2e-5 * (size_g * np.abs(x * r))[..., k].sum()
        out.append(np.abs(((up - down) * dy).sum() / 0.5 - dw[k]).reshape(1) / tol)
    return out


@pytest.mark.parametrize("rot,layout", ROTATIONS)
def test_the_comparison_notices_what_is_left_out(rot, layout):
    desc, x, w, dy, directions = data(rot)
    freq, _ = api.sepllm_rope_frequencies(desc)
    pos = np.arange(L)
    forward = lambda x, w: orc.rope_apply(orc.head_norm(x, w, EPS), pos, freq, layout)  # noqa: E731
    g = orc.rope_apply(dy, pos, freq, layout, inverse=True)
    dx, dw = orc.head_norm_bwd(x, w, g, EPS)
    n = rot // 2
    worst = lambda dx, dw: ratios(forward, dx, dw, x, w, dy, directions, n, layout)  # noqa: E731
    assert max(a.max() for a in worst(dx, dw)) <= 0.25       # (what is left for the kernel's own errors)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
    projection = x * r ** 2 * (x * r * g * w).mean(-1, keepdims=True)
    for wrong in (dx + projection, dx + 0.5 * projection, dx * 1.05,
                  orc.head_norm_bwd(x, w, dy, EPS)[0]):      # no projection, half of it, another r, not turned back
        along, free, *_ = worst(wrong, dw)
        assert np.mean(np.maximum(along, free) > 1) > 0.5
    for wrong in (dw * 1.01, orc.head_norm_bwd(x * 1.05, w, g, 0.0)[1]):
        assert max(a[0] for a in worst(dx, wrong)[2:]) > 1


@pytest.mark.gpu
@pytest.mark.parametrize("rot,layout", ROTATIONS)
def test_gradients_against_differences_row_by_row(rot, layout):
    desc, x, w, dy, directions = data(rot)
    desc.layout = api.ROPE_LAYOUTS[layout]
    freq, _ = api.sepllm_rope_frequencies(desc)

    def gpu(a):
        t = torch.from_numpy(a).float().cuda()
        assert np.array_equal(t.double().cpu().numpy(), a)
        return t

    def forward(x, w):
        xs, y = gpu(x), torch.empty((B, H, L, D), device="cuda")
        api.sepllm_qknorm_rope_fwd(desc, api.QkNorm(gpu(w), eps=EPS), None, xs, None, None, y, None, None)
        return y.double().cpu().numpy()
    dx, dw = torch.empty((B, H, L, D), device="cuda"), torch.empty(D, device="cuda")
    ws = api.alloc_bytes(api.sepllm_qknorm_rope_bwd_workspace_bytes(desc))
    api.sepllm_qknorm_rope_bwd(desc, api.QkNorm(gpu(w), eps=EPS), None, gpu(x), None, gpu(dy), None, None, dx, None, None, dw,
                               None, ws)
    got = ratios(forward, dx.double().cpu().numpy(), dw.double().cpu().numpy(), x, w, dy, directions, rot // 2, layout)
    assert max(a.max() for a in got) <= 1, [float(a.max()) for a in got]
