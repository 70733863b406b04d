"""Layer norm of a student network against the formula in 64 bits, and its gradients against the formula's and against
differences.

Tolerances follow from the arithmetic: u = 2^-24 per fp32 operation.  A row's sum is added by at most 32 elements a thread
and a tree of at most 10 levels, so a mean is off by 43 u of the mean magnitude; the deviation by about half of twice
that, and what is formed from them by a few u more.  Half a bf16 step (2^-8 relative) where a result is rounded to it."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
DTYPES = [torch.bfloat16, torch.float32]
IDS = ["bf16", "fp32"]
# rows, cols: every owner layout (4 to 1024 threads a row) at its edges, odd and aligned lengths
SHAPES = [(1, 1), (1, 8), (70, 32), (3, 7), (41, 33), (5, 512), (9, 513), (4, 1024), (300, 37), (2, 2048), (3, 2049),
          (2, 4099), (2, 8200), (2, 16385), (1, 32768), (4099, 64)]


def _dev(t, dtype, pad=0, shift=0):
    """t on the device in rows `pad` elements apart that start `shift` elements into a buffer of NaN."""
    t = t.to(dtype)
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v


def _close(got, ref, tol, what):
    assert got.shape == ref.shape, what
    off = (got.double() - ref).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(off.nan_to_num().max())}"


def _stats(v, eps):
    mean = v.mean(1, keepdim=True)
    return mean, ((v - mean).square().mean(1, keepdim=True) + eps).rsqrt()


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (3, 1)], ids=["dense", "strided", "unaligned"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(rows, cols, pad, shift, dtype):
    print(f"[layer norm] forward {rows}x{cols} pad {pad} shift {shift} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(rows * 40_000 + cols)
    x, r = (_dev(s * torch.randn(rows, cols, generator=g, device="cuda") + 0.5, dtype, pad, shift) for s in (1, 3))
    w, b = 1 + 0.3 * torch.randn(cols, generator=g, device="cuda"), torch.randn(cols, generator=g, device="cuda")
    for res, bias in ((r, b), (None, None)):
        y, v, mean, rstd = ops.add_layer_norm(x, w, bias, residual=res, eps=1e-5)
        s = x.double() if res is None else (x.float() + res.float()).double()
        assert v is x if res is None else torch.equal(v, s.float().to(dtype))
        mu, rho = _stats(s, 1e-5)
        mag = s.abs().mean(1, keepdim=True) + s.abs().amax(1, keepdim=True) * 2 ** -3
        off = 50 * U * mag  # of the mean
        _close(mean[:, None], mu, off, "mean")
        # (v - mean)^2 moves by 2 |v - mean| off + off^2, its mean by off^2 as the differences cancel; the sum by 45 u
        part = 60 * U + (off * rho) ** 2 + 2 * off * rho * 45 * U
        _close(rstd[:, None], rho, rho * part, "rstd")
        n = (s - mu) * rho
        ref = n * w.double() + (0 if bias is None else bias.double())
        err = w.double().abs() * ((off + U * s.abs()) * rho + n.abs() * (part + 4 * U)) + ref.abs() * (HALF[dtype] + U)
        _close(y, ref, err + U * n.abs() * w.double().abs(), "y")


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("rows,cols,pad,shift", [s + p for s in SHAPES for p in ((0, 0), (3, 1))] +
                         [(66_000, 8, 0, 0), (5_003, 1024, 0, 0), (2_100, 2049, 0, 0), (1_100, 9000, 0, 0),
                          (300, 20_000, 0, 0)])
def test_backward(rows, cols, pad, shift, dtype):
    print(f"[layer norm] backward {rows}x{cols} pad {pad} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(rows * 50_000 + cols)
    v, dy, dv = (_dev(torch.randn(rows, cols, generator=g, device="cuda") + m, dtype, pad, shift) for m in (0.7, 0.1, 0))
    w = 1 + 0.3 * torch.randn(cols, generator=g, device="cuda")
    mean, rstd = (t[:, 0].float().contiguous() for t in _stats(v.double(), 1e-5))
    V, DY, W, M, R = v.double(), dy.double(), w.double(), mean.double()[:, None], rstd.double()[:, None]
    N, G = (V - M) * R, DY * W
    sums = (G.abs().mean(1, keepdim=True), (G * N).abs().mean(1, keepdim=True))
    # n is off by 4 u and by u of v's and the mean's magnitudes; the row sums by 45 u of their terms' magnitudes
    noff = 4 * U * N.abs() + 2 * U * R * (V.abs() + M.abs())
    terms = G.abs() + sums[0] + N.abs() * sums[1]
    along = (G.abs() * noff).mean(1, keepdim=True)
    for d in (dv, None):
        dx, dw, db = ops.layer_norm_backward(dy, v, w, mean, rstd, dv=d)
        again = ops.layer_norm_backward(dy, v, w, mean, rstd, dv=d)
        assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), again))
        D = 0 if d is None else d.double()
        ref = R * (G - G.mean(1, keepdim=True) - N * (G * N).mean(1, keepdim=True)) + D
        err = R * (50 * U * terms + noff * sums[1] + N.abs() * along) + (HALF[dtype] + U) * ref.abs()
        _close(dx, ref, err, "dx")
        # rows one after the other in a block, its groups, the blocks' 64 streams: at most rows / 1024 + 1 + 64 + 16 + 64
        adds = rows / 64 + 150
        _close(dw, (DY * N).sum(0), adds * U * (DY * N).abs().sum(0) + (DY.abs() * noff).sum(0), "dweight")
        _close(db, DY.sum(0), adds * U * DY.abs().sum(0), "dbias")


def test_gradients_against_differences():
    """Of the whole operator, sum and statistics included: (f(x + h e) - f(x - h e)) / 2h in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(3)
    rows, cols = 5, 19
    x, r, dy, dv = (torch.randn(rows, cols, generator=g, device="cuda") for _ in range(4))
    w, b = torch.randn(cols, generator=g, device="cuda"), torch.randn(cols, generator=g, device="cuda")
    _, v, mean, rstd = ops.add_layer_norm(x, w, b, residual=r, eps=1e-3)
    got = ops.layer_norm_backward(dy, v, w, mean, rstd, dv=dv)

    def loss(x, w, b):
        s = x + r.double()
        mu, rho = _stats(s, 1e-3)
        return (((s - mu) * rho * w + b) * dy.double()).sum() + (s * dv.double()).sum()

    at = [t.double() for t in (x, w, b)]
    for i, grad in enumerate(got):
        want = torch.empty_like(at[i])
        for j in range(want.numel()):
            h = 1e-5
            ends = []
            for s in (h, -h):
                p = [t.clone() for t in at]
                p[i].view(-1)[j] += s
                ends.append(loss(*p))
            want.view(-1)[j] = (ends[0] - ends[1]) / (2 * h)
        # fp32 sums of 19 terms of order 1 (some 25 u of up to 40), and h^2 / 6 of a third derivative of order 100
        assert float((grad.double() - want).abs().max()) < 1e-4


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("cols", [5, 700, 3000, 20_000])
def test_rows_at_the_ends_of_the_range(cols, dtype):
    """Values whose sum or squares overflow fp32, a large mean beside a small deviation, equal values, non-finite ones."""
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(6, cols, generator=g, device="cuda")
    x[0] *= 1e37
    x[1] = 3.0e38 * torch.where(torch.arange(cols, device="cuda") % 2 == 0, 1.0, -0.75)
    x[2] = 5.0
    x[4, cols // 2] = float("inf")
    x[5, cols - 1] = float("nan")
    x = x.to(dtype)
    w, b = torch.ones(cols, device="cuda"), torch.full((cols,), 0.25, device="cuda")
    y, _, mean, rstd = ops.add_layer_norm(x, w, b, eps=1e-6)
    mu, rho = _stats(x.double(), 1e-6)
    ref = (x.double() - mu) * rho + 0.25
    part = HALF[dtype] + 200 * U
    for row in (0, 1, 3):
        _close(y[row], ref[row], part * ref[row].abs() + 200 * U * (1 + mu[row].abs() * rho[row]), f"y of row {row}")
        _close(rstd[row], rho[row, 0], 200 * U * rho[row, 0], "rstd")
    assert bool((y[2] == 0.25).all()) and bool(y[4:].isnan().all())
    dy = torch.randn(6, cols, generator=g, device="cuda").to(dtype)
    dx, _, _ = ops.layer_norm_backward(dy[:2].contiguous(), x[:2].contiguous(), w, mean[:2].contiguous(),
                                       rstd[:2].contiguous())
    n, G = (x.double() - mu) * rho, dy.double()
    ref = rho * (G - G.mean(1, keepdim=True) - n * (G * n).mean(1, keepdim=True))
    tol = rho * 300 * U * (G.abs() + G.abs().mean(1, keepdim=True) + n.abs() * (G * n).abs().mean(1, keepdim=True))
    # (gradients of 1e-37 lie below the smallest normal value, where a step is 2^-149 (fp32) or 2^-133 (bf16))
    _close(dx, ref[:2], tol[:2] + HALF[dtype] * ref[:2].abs() + (2.0 ** -133 if dtype is torch.bfloat16 else 2.0 ** -147),
           "dx of large rows")


def test_mean_far_above_the_deviation():
    """x = 1000 + noise of 1: a difference of mean squares would lose 20 bits of the deviation."""
    g = torch.Generator(device="cuda").manual_seed(8)
    x = 1000 + torch.randn(64, 1024, generator=g, device="cuda")
    y, _, _, rstd = ops.add_layer_norm(x, torch.ones(1024, device="cuda"), eps=0.0)
    mu, rho = _stats(x.double(), 0.0)
    # the mean is off by some 20 u of 1000, the same for the whole row
    _close(rstd[:, None], rho, rho * (100 * U + (50 * U * 1000) ** 2), "rstd")
    _close(y, (x.double() - mu) * rho, torch.full_like(y, 60 * U * 1000, dtype=torch.float64), "y")


def test_empty_and_in_place():
    w = torch.ones(40, device="cuda")
    y, v, mean, rstd = ops.add_layer_norm(torch.empty(0, 40, device="cuda"), w)
    assert y.shape == (0, 40) and mean.shape == (0,)
    dx, dw, db = ops.layer_norm_backward(y, v, w, mean, rstd)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()
