"""Dropout whose mask is never stored: the mask bit for bit against the oracle's generator, the values to one rounding."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle.philox import philox4x32_10  # noqa: E402
from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
DTYPES = [torch.bfloat16, torch.float32]
IDS = ["bf16", "fp32"]


def _mask(rows, cols, p, seed, step, site):
    groups = -(-cols // 8)
    c, r = np.meshgrid(np.arange(groups, dtype=np.uint64), np.arange(rows, dtype=np.uint64))
    one = np.ones_like(c)
    words = philox4x32_10(c, r, one * np.uint64(site), one * np.uint64(step & 0xFFFFFFFF), seed & 0xFFFFFFFF,
                          (seed >> 32) ^ (4 << 28))
    w = np.stack([np.asarray(x, dtype=np.uint64) for x in words], -1)
    half = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(rows, groups * 8)[:, :cols]
    return torch.from_numpy(half >= np.uint64(int(p * 65536))).cuda()


def _strided(t, pad, shift):
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=t.dtype, device="cuda")
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (1, 8, 0, 0), (7, 9, 0, 0), (300, 301, 0, 0),
                                                 (300, 301, 4, 1), (129, 1024, 8, 8), (3, 10_007, 1, 3), (5000, 3, 0, 0)])
@pytest.mark.parametrize("p", [0.0, 1e-6, 0.1, 0.5, 0.9, 1.0])
def test_values_and_mask(rows, cols, pad, shift, p, dtype):
    print(f"[dropout] {rows}x{cols} pad {pad} p {p} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    x, r = (_strided(torch.randn(rows, cols, generator=g, device="cuda").to(dtype), pad, shift) for _ in range(2))
    seed, step, site = 0xFEDC_BA98_7654_3210, 77, 2
    keep = _mask(rows, cols, p, seed, step, site)
    f = 1 / (1 - p) if p < 1 else 0.0
    part = torch.where(keep, x.double() * f, 0.0)
    y = ops.dropout(x, p, seed, step, site=site)
    assert bool(((y.double() - part).abs() <= (HALF[dtype] + 2 * U) * part.abs()).all())
    assert bool((y[~keep] == 0).all())
    z = ops.dropout(x, p, seed, step, site=site, residual=r)
    ref = part + r.double()
    assert bool(((z.double() - ref).abs() <= HALF[dtype] * ref.abs() + 2 * U * (part.abs() + r.double().abs())).all())
    assert torch.equal(z[~keep], r[~keep])


def test_the_mask_depends_on_nothing_else():
    """Not on the type, the row length or the rows beside it; on seed, step and site it does."""
    one = torch.ones(64, 200, device="cuda")
    base = ops.dropout(one, 0.5, 5, 9, site=1)
    assert torch.equal(ops.dropout(one[:, :37].contiguous(), 0.5, 5, 9, site=1), base[:, :37])
    assert torch.equal(ops.dropout(one[:10].bfloat16(), 0.5, 5, 9, site=1).float(), base[:10])
    others = [ops.dropout(one, 0.5, 6, 9, site=1), ops.dropout(one, 0.5, 5, 10, site=1), ops.dropout(one, 0.5, 5, 9),
              ops.dropout(one, 0.5, 5 + (1 << 40), 9, site=1)]
    assert all(0.4 < float((o == base).float().mean()) < 0.6 for o in others)
    assert torch.equal(ops.dropout(one, 0.5, 5, 9 + (1 << 32), site=1), base)  # (step mod 2^32)


def test_rate():
    y = ops.dropout(torch.ones(4096, 1024, device="cuda"), 0.3, 1, 2)
    # 4 M draws: a standard deviation of 2.2e-4
    assert abs(float((y == 0).float().mean()) - 0.3) < 1.2e-3


def test_dropped_elements_count_for_nothing():
    x = torch.full((16, 64), float("nan"), device="cuda")
    keep = _mask(16, 64, 0.4, 3, 4, 0)
    y = ops.dropout(x, 0.4, 3, 4)
    assert bool((y[~keep] == 0).all()) and bool(y[keep].isnan().all())
    x = torch.where(keep, 1.0, float("inf"))
    assert bool(ops.dropout(x, 0.4, 3, 4, residual=torch.ones_like(x)).isfinite().all())


def test_gradient_is_the_same_call():
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r, dy = (torch.randn(33, 47, generator=g, device="cuda") for _ in range(3))
    keep = _mask(33, 47, 0.25, 11, 12, 13).double()
    dx = ops.dropout(dy, 0.25, 11, 12, site=13)
    X = x.double().requires_grad_()
    ((r.double() + X * keep / 0.75) * dy.double()).sum().backward()
    assert float((dx.double() - X.grad).abs().max()) <= 2 * U * float(X.grad.abs().max())
    # (y(x + h) - y(x - h)) / 2h along a direction, y linear in x: exact but for the roundings of y
    d = torch.randn(33, 47, generator=g, device="cuda")
    up, down = (ops.dropout(x + s * d, 0.25, 11, 12, site=13, residual=r).double() for s in (0.5, -0.5))
    diff = ((up - down) * dy.double()).sum()
    along = (dx.double() * d.double()).sum()
    scale = float(((x.abs() + d.abs() + r.abs()).double() * dy.abs().double()).sum()) * 1.4
    assert abs(float(diff - along)) <= 8 * U * scale


def test_a_captured_step_draws_new_masks():
    x = torch.ones(100, 100, device="cuda")
    step = torch.zeros((), dtype=torch.int64, device="cuda")
    ops.dropout(x, 0.5, 21, step)  # (the library is loaded before the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ops.dropout(x, 0.5, 21, step)
        step += 1
    for t in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ops.dropout(x, 0.5, 21, t))
        assert int(step) == t + 1


def test_empty():
    assert ops.dropout(torch.empty(0, 5, device="cuda"), 0.5, 1, 1).shape == (0, 5)
