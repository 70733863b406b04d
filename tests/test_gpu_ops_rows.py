"""Row operators of a student network (norm, 8-bit rows, distillation) against plain 64-bit formulas on the host.

Tolerances follow from the arithmetic: u = 2^-24 per fp32 operation, at most 32 elements a thread and a tree of at
most 10 levels above them per row sum, and half a bf16 step (8 significant bits: 2^-8 relative) where a result is rounded to bf16."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops, tabpack  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
DTYPES = [torch.bfloat16, torch.float32]
# rows, cols: every owner layout (64, 256, 1024 threads a row) at its edges, odd and aligned lengths
SHAPES = [(1, 1), (1, 8), (3, 7), (5, 512), (9, 513), (4, 1024), (300, 37), (2, 2048), (3, 2049), (2, 8200),
          (2, 16385), (1, 32768), (4099, 64)]


def _rand(gen, *shape):
    return torch.from_numpy(gen.standard_normal(shape).astype(np.float32))


def _dev(t, dtype, pad=0, shift=0):
    """t on the device, optionally in rows `pad` elements apart that start `shift` elements into a buffer of NaN."""
    t = t.to(dtype)
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(t.cuda())
    return v


def _f64(t):
    return t.detach().double().cpu().numpy()


def _close(got, ref, tol, what):
    got, ref = _f64(got), np.asarray(ref)
    assert got.shape == ref.shape, what
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - ref))}"


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp32"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (3, 1)], ids=["dense", "strided", "unaligned"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_forward_and_codes(rows, cols, pad, shift, dtype):
    print(f"[rows] norm {rows}x{cols} pad {pad} shift {shift} {dtype}", flush=True)
    gen = np.random.default_rng(rows * 40_000 + cols)
    x, r = _dev(_rand(gen, rows, cols), dtype, pad, shift), _dev(_rand(gen, rows, cols) * 3, dtype, pad, shift)
    w = (1 + 0.3 * _rand(gen, cols)).cuda()
    y, v, rstd = ops.add_rms_norm(x, w, residual=r, eps=1e-5)
    q, scale, v8 = ops.add_rms_norm_q8(x, w, residual=r, eps=1e-5)
    y0, v0, rstd0 = ops.add_rms_norm(x, w, eps=1e-5)
    torch.cuda.synchronize()
    assert v0 is x and torch.equal(v, v8)
    for a, yy, rr in ((_f64(x) + _f64(r), y, rstd), (_f64(x), y0, rstd0)):
        rho = 1 / np.sqrt((a ** 2).mean(1) + 1e-5)
        _close(rr, rho, 64 * U * rho, "rstd")
        ref = a * rho[:, None] * _f64(w)
        _close(yy, ref, np.abs(ref) * (HALF[dtype] + 70 * U), "y")
    a32 = x.float().cpu().numpy() + r.float().cpu().numpy()
    assert torch.equal(v.cpu(), torch.from_numpy(a32).to(dtype))
    t = a32 * w.cpu().numpy()
    m = np.abs(t).max(1, keepdims=True)
    codes = np.rint(t * (np.float32(127) / m))
    np.testing.assert_array_equal(q.cpu().numpy(), codes.astype(np.int8))
    a = _f64(x) + _f64(r)
    ref = m[:, 0].astype(np.float64) / 127 / np.sqrt((a ** 2).mean(1) + 1e-5)
    _close(scale, ref, 70 * U * ref, "scale")
    # plain rows
    q, scale = ops.quantize_rows(x)
    x32 = x.float().cpu().numpy()
    m = np.abs(x32).max(1, keepdims=True)
    np.testing.assert_array_equal(q.cpu().numpy(), np.rint(x32 * (np.float32(127) / m)).astype(np.int8))
    np.testing.assert_array_equal(scale.cpu().numpy(), (m / np.float32(127))[:, 0])


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp32"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (3, 1)], ids=["dense", "strided", "unaligned"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_backward(rows, cols, pad, shift, dtype):
    print(f"[rows] norm backward {rows}x{cols} pad {pad} shift {shift} {dtype}", flush=True)
    gen = np.random.default_rng(rows * 40_000 + cols + 1)
    v, dy, ds = (_dev(_rand(gen, rows, cols), dtype, pad, shift) for _ in range(3))
    w = (1 + 0.3 * _rand(gen, cols)).cuda()
    V, DY, DS, W = _f64(v), _f64(dy), _f64(ds), _f64(w)
    rstd = torch.from_numpy((1 / np.sqrt((V ** 2).mean(1) + 1e-5)).astype(np.float32)).cuda()
    R = _f64(rstd)[:, None]
    g = DY * W
    mag = (np.abs(g) + np.abs(V) * R ** 2 / cols * np.abs(g * V).sum(1, keepdims=True)) * R
    for dv in (ds, None):
        dx, dw = ops.rms_norm_backward(dy, v, w, rstd, dv=dv)
        again = ops.rms_norm_backward(dy, v, w, rstd, dv=dv)
        assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
        add = 0 if dv is None else DS
        ref = R * (g - V * R ** 2 / cols * (g * V).sum(1, keepdims=True)) + add
        _close(dx, ref, np.abs(ref) * HALF[dtype] + 64 * U * (mag + np.abs(add)), "dx")
        # a thread adds up to rows / 4096 + 1 rows, then 4 row groups, then 64 blocks a stream and 16 streams
        _close(dw, (DY * V * R).sum(0), (rows / 4096 + 96) * U * np.abs(DY * V * R).sum(0), "dweight")


def test_norm_gradient_against_differences():
    gen = np.random.default_rng(5)
    x, w, c = gen.standard_normal((3, 21)), 1 + 0.2 * gen.standard_normal(21), gen.standard_normal((3, 21))

    def loss(x, w):  # 64 bits
        return (c * x / np.sqrt((x ** 2).mean(1, keepdims=True) + 1e-3) * w).sum()

    h = 1e-6
    nx, nw = np.zeros_like(x), np.zeros_like(w)
    for i in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[i] = h
        nx[i] = (loss(x + d, w) - loss(x - d, w)) / (2 * h)
    for i in range(21):
        d = np.zeros_like(w)
        d[i] = h
        nw[i] = (loss(x, w + d) - loss(x, w - d)) / (2 * h)
    X, Wt, C = (torch.from_numpy(a.astype(np.float32)).cuda() for a in (x, w, c))
    _, v, rstd = ops.add_rms_norm(X, Wt, eps=1e-3)
    dx, dw = ops.rms_norm_backward(C, v, Wt, rstd)
    # differences: h^2 and 2^-53 / h; inputs and arithmetic in fp32: values of order 1 to within 100 u
    _close(dx, nx, 1e-5, "dx")
    _close(dw, nw, 1e-5, "dweight")


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp32"])
@pytest.mark.parametrize("cols", [16, 21, 3000])
def test_rows_without_finite_magnitude(cols, dtype):
    x = torch.ones(6, cols)
    x[0] = 0.0
    x[1, cols - 1] = float("inf")
    x[2, 0] = float("nan")
    x[3] = 1e-38
    x[4, 1] = -float("inf")
    q, scale = ops.quantize_rows(_dev(x, dtype))
    qn, sn, _ = ops.add_rms_norm_q8(_dev(x, dtype), torch.ones(cols, device="cuda"))
    for codes, s in ((q, scale), (qn, sn)):
        assert not codes[:5].any() and (codes[5] == 127).all()
        s = s.cpu()
        assert s[0] == 0 and s[3] == 0 and torch.isnan(s[[1, 2, 4]]).all() and s[5] > 0
    y, _, rstd = ops.add_rms_norm(_dev(torch.zeros(2, cols), dtype), torch.ones(cols, device="cuda"), eps=1e-6)
    assert not y.any() and torch.allclose(rstd.cpu(), torch.full((2,), 1e3))


def test_rows_empty_and_far_apart():
    for dtype in DTYPES:
        e = torch.empty(0, 24, dtype=dtype, device="cuda")
        w = torch.ones(24, device="cuda")
        assert ops.add_rms_norm(e, w, residual=e)[0].shape == (0, 24)
        assert ops.quantize_rows(e)[1].shape == (0,)
        dx, dw = ops.rms_norm_backward(e, e, w, torch.empty(0, device="cuda"))
        assert dx.shape == (0, 24) and not dw.any()
    # element offsets past 2^31: three rows 2^30 + 8 elements apart
    ld, cols = (1 << 30) + 8, 1024
    buf = torch.empty(2 * ld + cols, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, cols), (ld, 1))
    x.copy_(torch.randn(3, cols, device="cuda"))
    near = x.contiguous()
    w = torch.rand(cols, device="cuda")
    for a, b in zip(ops.add_rms_norm(x, w, residual=x), ops.add_rms_norm(near, w, residual=near)):
        assert torch.equal(a, b)
    for a, b in zip(ops.quantize_rows(x), ops.quantize_rows(near)):
        assert torch.equal(a, b)
    rstd = torch.rand(3, device="cuda")
    for a, b in zip(ops.rms_norm_backward(x, x, w, rstd, dv=x), ops.rms_norm_backward(near, near, w, rstd, dv=near)):
        assert torch.equal(a, b)
    idx = torch.tensor([[0, 5, 1023]] * 3, dtype=torch.int32, device="cuda")
    t = torch.randn(3, 3, device="cuda")
    for a, b in zip(ops.distill_topk(x, idx, t), ops.distill_topk(near, idx, t)):
        assert torch.equal(a, b)


def test_rows_past_one_launch_and_another_stream():
    # more rows than a launch has row slots (2^20 blocks of 4 rows): the blocks go on
    rows = (1 << 22) + 77
    x = torch.randn(rows, 8, device="cuda").to(torch.bfloat16)
    q, scale = ops.quantize_rows(x)
    x32 = x.float()
    m = x32.abs().amax(1)
    assert torch.equal(scale, torch.div(m, torch.full_like(m, 127.0)))  # (m / 127 multiplies by a rounded 1 / 127)
    assert torch.equal(q.float(), torch.round(x32 * torch.div(torch.full_like(m, 127.0), m)[:, None]))
    w = torch.rand(8, device="cuda")
    ref = ops.add_rms_norm(x, w)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = ops.add_rms_norm(x * 1, w)[0]
    s.synchronize()
    assert torch.equal(y, ref)


# ------------------------------------------------------------ distillation
def _distill_ref(z, idx, t, tau, w):
    """64-bit loss, gradient and the error scales of both."""
    rows, V = z.shape
    loss, grad = np.zeros(rows), np.zeros((rows, V))
    tl, tg = np.zeros(rows), np.zeros((rows, V))
    for r in range(rows):
        here = [j for j in range(idx.shape[1]) if idx[r, j] >= 0 and t[r, j] != -np.inf]
        if not here or w[r] == 0:
            continue
        a = z[r] / tau
        lq = a - a.max() - np.log(np.exp(a - a.max()).sum())
        b = t[r, here] / tau
        lp = b - b.max() - np.log(np.exp(b - b.max()).sum())
        p, at = np.exp(lp), idx[r, here]
        keep = p > 0
        loss[r] = w[r] * tau ** 2 * (p[keep] * (lp - lq[at])[keep]).sum()
        target = np.zeros(V)
        np.add.at(target, at, p)
        grad[r] = w[r] * tau * (np.exp(lq) - target)
        # an exponent x / tau is off by at most 3 u |x / tau|, a sum by 80 u; p and q inherit both
        fin = np.isfinite(a)
        e = (3 * (np.ptp(a[fin]) + np.ptp(b)) + 120) * U
        tl[r] = abs(w[r]) * tau ** 2 * (p[keep] * (np.abs(lp) + np.abs(lq[at]) + 1)[keep]).sum() * e
        tg[r] = abs(w[r]) * tau * (np.exp(lq) + target) * e + 1e-37
    return loss, grad, tl, tg


DISTILL = [(1, 1, 1), (3, 2, 1), (5, 10, 4), (7, 16, 16), (70, 128, 5), (9, 129, 64), (6, 1000, 256), (5, 1025, 3),
           (3, 4097, 33), (4, 16384, 32), (2, 20_001, 8), (3, 32_000, 64), (2, 50_000, 7), (2, 65_537, 9),
           (2, 70_000, 256)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp32"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (3, 1)], ids=["dense", "strided", "unaligned"])
@pytest.mark.parametrize("rows,V,k", DISTILL)
def test_distill(rows, V, k, pad, shift, dtype):
    print(f"[rows] distill {rows}x{V} k {k} pad {pad} shift {shift} {dtype}", flush=True)
    gen = np.random.default_rng(rows * 100_000 + V + k)
    z = _dev(2 * _rand(gen, rows, V), dtype, pad, shift)
    idx = gen.integers(0, V, (rows, k)).astype(np.int32)      # classes named several times among them
    t = 2 * gen.standard_normal((rows, k)).astype(np.float32)
    idx[gen.random((rows, k)) < 0.1] = -1
    t[gen.random((rows, k)) < 0.05] = -np.inf
    w = gen.random(rows).astype(np.float32) + 0.1
    if rows > 2:
        idx[0] = -3
        w[1] = 0.0
    tau = 1.7
    w32, tau32 = w.astype(np.float64), float(np.float32(tau))
    ref = _distill_ref(_f64(z), idx, t.astype(np.float64), tau32, w32)
    I, T, W = (torch.from_numpy(a).cuda() for a in (idx, t, w))
    loss, grad = ops.distill_topk(z, I, T, temperature=tau, row_weight=W)
    only, none = ops.distill_topk(z, I, T, temperature=tau, row_weight=W, grad=False)
    assert none is None and torch.equal(only, loss)
    _close(loss, ref[0], ref[2], "loss")
    _close(grad, ref[1], ref[3] + np.abs(ref[1]) * HALF[dtype], "grad")
    loss1, _ = ops.distill_topk(z, I, T, temperature=tau)
    ref1 = _distill_ref(_f64(z), idx, t.astype(np.float64), tau32, np.ones(rows))
    _close(loss1, ref1[0], ref1[2], "loss without weights")


@pytest.mark.parametrize("V", [10, 200, 3000, 66_000])
def test_distill_masked_and_non_finite_rows(V):
    gen = np.random.default_rng(V)
    low = torch.finfo(torch.float32).min
    z = _rand(gen, 9, V)
    z[0, V // 2:] = low                # masked classes at the type's lowest value
    z[1, V // 2:] = -float("inf")
    z[2] = low                         # nothing but the lowest value: uniform
    z[3, 1] = float("nan")             # NaN in a live row
    z[4] = float("nan")                # NaN in a row of weight 0
    z[5, V - 1] = float("nan")         # NaN in a row without entries
    z[6] = -float("inf")               # a live row with nothing left
    idx = torch.tensor([[0, 1, 2]] * 9, dtype=torch.int32)
    t = _rand(gen, 9, 3)
    idx[5] = -1
    idx[7, 2] = V                      # no such class
    t[8, 0] = float("nan")
    w = torch.ones(9)
    w[4] = 0.0
    loss, grad = ops.distill_topk(z.cuda(), idx.cuda(), t.cuda(), temperature=0.5, row_weight=w.cuda())
    loss, grad = loss.cpu(), grad.cpu()
    for r in (3, 6, 7, 8):
        assert torch.isnan(loss[r]) and torch.isnan(grad[r]).all(), r
    for r in (4, 5):
        assert loss[r] == 0 and not grad[r].any(), r
    zz = z.double().numpy()
    with np.errstate(over="ignore"):
        ref = _distill_ref(zz[:3], idx[:3].numpy(), t[:3].double().numpy(), 0.5, np.ones(3))
    e = (3 * 40 + 120) * U             # the finite classes span less than 20 / tau
    for r in range(3):
        assert abs(float(loss[r]) - ref[0][r]) <= e * 40
        assert np.abs(grad[r].double().numpy() - ref[1][r]).max() <= e
    assert not grad[0, V // 2:].any() and not grad[1, V // 2:].any()


def test_distill_gradient_against_differences():
    gen = np.random.default_rng(3)
    z = gen.standard_normal((2, 9))
    idx = np.array([[1, 4, 1], [8, -1, 0]], np.int32)
    t = gen.standard_normal((2, 3))
    w, tau, h = np.array([0.5, 2.0]), 1.5, 1e-6
    num = np.zeros_like(z)
    for i in np.ndindex(z.shape):
        d = np.zeros_like(z)
        d[i] = h
        num[i] = (_distill_ref(z + d, idx, t, tau, w)[0] - _distill_ref(z - d, idx, t, tau, w)[0]).sum() / (2 * h)
    _, grad = ops.distill_topk(torch.from_numpy(z.astype(np.float32)).cuda(), torch.from_numpy(idx).cuda(),
                               torch.from_numpy(t.astype(np.float32)).cuda(), temperature=tau,
                               row_weight=torch.from_numpy(w.astype(np.float32)).cuda())
    _close(grad, num, 1e-5, "grad")


def test_binding_refuses_shapes_strides_and_types():
    x = torch.zeros(4, 8, device="cuda")
    w = torch.ones(8, device="cuda")
    i3 = torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    for call in (lambda: ops.add_rms_norm(x.t(), torch.ones(4, device="cuda")),
                 lambda: ops.add_rms_norm(x[:, ::2], w[:4]),
                 lambda: ops.add_rms_norm(x[:1].expand(4, 8), w),
                 lambda: ops.add_rms_norm(x, w, residual=x[:3]),
                 lambda: ops.add_rms_norm(x, w, residual=x.bfloat16()),
                 lambda: ops.add_rms_norm(x, w[:7]),
                 lambda: ops.add_rms_norm(x, w.bfloat16()),
                 lambda: ops.add_rms_norm(x, w.cpu()),
                 lambda: ops.add_rms_norm(x, w, eps=-1.0),
                 lambda: ops.add_rms_norm(x.half(), w),
                 lambda: ops.add_rms_norm(x[0], w),
                 lambda: ops.quantize_rows(torch.zeros(2, 40_000, device="cuda")),
                 lambda: ops.rms_norm_backward(x[:3], x, w, torch.ones(4, device="cuda")),
                 lambda: ops.rms_norm_backward(x, x, w, torch.ones(3, device="cuda")),
                 lambda: ops.distill_topk(x, i3.long(), i3.float()),
                 lambda: ops.distill_topk(x, i3, i3.float()[:, :2]),
                 lambda: ops.distill_topk(x, i3[:3], i3.float()[:3]),
                 lambda: ops.distill_topk(x, i3, i3.float(), temperature=0.0),
                 lambda: ops.distill_topk(x, i3, i3.float(), row_weight=w[:3])):
        with pytest.raises(tabpack.PackError):
            call()
