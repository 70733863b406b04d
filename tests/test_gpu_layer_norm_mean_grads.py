"""Layer norm's gradients in fp32 for rows whose mean is large beside their deviation, against the formula in 64 bits from the
row itself: the mean, as it is handed over, is rounded to fp32.

With n = (v - mu) rho: n is formed with 4 u of its magnitude and that of h, the rounding of mu times rho (below 1 in the cases
here), and less its own mean, a sum of 45 u of mean |n| <= 1 + h; rho is off by 130 u (test_gpu_layer_norm_means.py), so n by
(130 + 5) |n| + 100 (1 + h) u in all, less than 340 u (1 + |n|).  The row sums add 45 u of their terms' magnitudes, the
subtraction of h times one of them twice as much."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("mean,std", [(0.5, 1.0), (1e3, 1.0), (1e5, 1.0), (-1e6, 1.0), (1e8, 20.0)])
@pytest.mark.parametrize("rows,cols", [(3, 8), (70, 37), (33, 127), (41, 512), (300, 1000), (37, 2047), (19, 4099), (9, 8192),
                                       (7, 9000), (40, 16_384), (130, 16_385), (5, 32_768)])
def test_gradients(rows, cols, mean, std):
    print(f"[layer norm] gradients, mean {mean} deviation {std}, {rows}x{cols}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = mean + std * torch.randn(rows, cols, generator=g, device="cuda")
    dy, dv = torch.randn(rows, cols, generator=g, device="cuda"), torch.randn(rows, cols, generator=g, device="cuda")
    w = 1 + 0.3 * torch.randn(cols, generator=g, device="cuda")
    y, v, mu, rstd = ops.add_layer_norm(x, w, eps=1e-5)
    dx, dw, db = ops.layer_norm_backward(dy, v, w, mu, rstd, dv=dv)
    X, DY, W = x.double(), dy.double(), w.double()
    M = X.mean(1, keepdim=True)
    R = ((X - M).square().mean(1, keepdim=True) + 1e-5).rsqrt()
    N, G = (X - M) * R, DY * W
    off = 340 * U * (1 + N.abs())  # of n
    along = (G * N).mean(1, keepdim=True)
    lost = 140 * U * (G.abs() * (1 + N.abs())).mean(1, keepdim=True) + (G.abs() * off).mean(1, keepdim=True)
    ref = R * (G - G.mean(1, keepdim=True) - N * along) + dv.double()
    tol = R * (140 * U * (G.abs() + G.abs().mean(1, keepdim=True) + N.abs() * along.abs()) + off * along.abs() + N.abs() * lost +
               45 * U * G.abs().mean(1, keepdim=True)) + U * ref.abs()
    worst = float(((dx.double() - ref).abs() / tol).max())
    assert worst <= 1, f"dx off by {worst:.3g} times the bound"
    adds = rows / 64 + 150  # (as in test_gpu_layer_norm.py)
    tol = adds * U * (DY * N).abs().sum(0) + (DY.abs() * off).sum(0)
    worst = float(((dw.double() - (DY * N).sum(0)).abs() / tol).max())
    assert worst <= 1, f"dweight off by {worst:.3g} times the bound"
    assert bool(((db.double() - DY.sum(0)).abs() <= adds * U * DY.abs().sum(0)).all())
