"""Row operators where magnitudes come near the ends of fp32: the norm and its gradients of finite rows whose squares no
longer fit fp32, against the formulas in 64 bits on the host.

Tolerances as in test_gpu_ops_rows.py (u = 2^-24 per fp32 operation, half a bf16 step where a result is rounded), and
the result's smallest step (fp32 2^-149, bf16 2^-133) where a value itself is near it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = {torch.bfloat16: 2.0 ** -133, torch.float32: 2.0 ** -149}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
DTYPES = [torch.bfloat16, torch.float32]
# every count of threads a row: 4, 16, 64 (8 to 32 elements each), 256, 1024
COLS = [7, 64, 500, 1024, 2001, 3000, 8200, 9000, 20_000]


def _rows(gen, cols, dtype):
    """Rows of every magnitude: past the square root of the largest value, single values at the type's lowest, rows of
    nothing else, and ordinary rows between them."""
    x = gen.standard_normal((7, cols)).astype(np.float32)
    low = torch.finfo(dtype).min
    x[0] *= np.float32(1e25)
    x[1, cols // 2] = low
    x[2] = low
    x[3] = -low
    x[4] *= np.float32(2e19)
    return torch.from_numpy(x).to(dtype).cuda()


def _f64(t):
    return t.detach().double().cpu().numpy()


def _close(got, ref, tol, what):
    got = _f64(got)
    assert got.shape == ref.shape, what
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first {np.argwhere(bad)[0]}"


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp32"])
@pytest.mark.parametrize("cols", COLS)
def test_norm_of_large_rows(cols, dtype):
    print(f"[range] norm {cols} {dtype}", flush=True)
    gen = np.random.default_rng(cols)
    x = _rows(gen, cols, dtype)
    r = torch.from_numpy(gen.standard_normal((7, cols)).astype(np.float32)).to(dtype).cuda()
    w = torch.from_numpy((1 + 0.3 * gen.standard_normal(cols)).astype(np.float32)).cuda()
    y, v, rstd = ops.add_rms_norm(x, w, residual=r, eps=1e-5)
    q, scale, v8 = ops.add_rms_norm_q8(x, w, residual=r, eps=1e-5)
    a = _f64(x.float() + r.float())
    rho = 1 / np.sqrt((a ** 2).mean(1) + 1e-5)
    ref = a * rho[:, None] * _f64(w)
    assert torch.equal(v, (x.float() + r.float()).to(dtype)) and torch.equal(v, v8)
    _close(rstd, rho, 64 * U * rho + TINY[torch.float32], "rstd")
    # (a value 2^46 times smaller than its row's largest may lose bits below 2^-126)
    _close(y, ref, np.abs(ref) * (HALF[dtype] + 70 * U) + 2.0 ** -120, "y")
    m = np.abs(ref).max(1)
    _close(scale, m / 127, 80 * U * m, "scale")
    value = _f64(q) * _f64(scale)[:, None]
    assert (np.abs(_f64(q)).max(1) == 127).all()
    assert (np.abs(value - ref) <= (0.5 + 127 * 160 * U) * m[:, None] / 127).all(), "codes"


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp32"])
@pytest.mark.parametrize("cols", COLS)
def test_norm_gradients_of_large_rows(cols, dtype):
    print(f"[range] norm backward {cols} {dtype}", flush=True)
    gen = np.random.default_rng(cols + 1)
    v = _rows(gen, cols, dtype)
    dy, ds = (torch.from_numpy(s * gen.standard_normal((7, cols)).astype(np.float32)).to(dtype).cuda() for s in (4, 1))
    w = torch.from_numpy((1 + 0.3 * gen.standard_normal(cols)).astype(np.float32)).cuda()
    V, DY, DS, W = _f64(v), _f64(dy), _f64(ds), _f64(w)
    rstd = torch.from_numpy((1 / np.sqrt((V ** 2).mean(1) + 1e-5)).astype(np.float32)).cuda()
    R = _f64(rstd)[:, None]
    g = DY * W
    mag = (np.abs(g) + np.abs(V) * R ** 2 / cols * np.abs(g * V).sum(1, keepdims=True)) * R
    for dv in (ds, None):
        dx, dw = ops.rms_norm_backward(dy, v, w, rstd, dv=dv)
        add = 0 if dv is None else DS
        ref = R * (g - V * R ** 2 / cols * (g * V).sum(1, keepdims=True)) + add
        _close(dx, ref, np.abs(ref) * HALF[dtype] + 64 * U * (mag + np.abs(add)) + 4 * TINY[dtype],
               "dx")
        _close(dw, (DY * V * R).sum(0), 96 * U * np.abs(DY * V * R).sum(0), "dweight")
