"""Layer norm of rows whose mean is large beside their deviation, against the formula in 64 bits.

With m the mean as it was first rounded, the kernel takes the differences d = v - m, their mean e out of them, and e^2 out of
their mean square.  u = 2^-24: a sum over a row is off by 45 u of its terms' magnitudes (32 elements a thread, 10 levels), and
e^2 is at most the variance s^2, so that mean |d| <= 1.5 s.  Then e is off by 70 u s, a difference d - e by u (|d| + |e|) more, the
variance by 45 u of s^2 + e^2 and 2 |e| 70 u s, below 240 u s^2, and its root by half of that: with n = (v - mu) / s the
result is off by at most (70 + 5 + 3 |n| + 120 |n| + 5 |n|) u, less than 130 u (1 + |n|)."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
# every owner layout of a row (4 to 1024 threads), whole and odd lengths
COLS = [8, 37, 127, 512, 1000, 1024, 2047, 4099, 8192, 9000, 20_000, 32_768]


def _check(x, r, eps, dtype):
    cols = x.shape[1]
    s = x.double() if r is None else (x.float() + r.float()).double()
    mu = s.mean(1, keepdim=True)
    dev = ((s - mu).square().mean(1, keepdim=True) + eps).sqrt()
    n = (s - mu) / dev
    y, _, mean, rstd = ops.add_layer_norm(x, torch.ones(cols, device="cuda"), residual=r, eps=eps)
    off = (y.double() - n).abs() / (130 * U * (1 + n.abs()) + HALF[dtype] * n.abs())
    assert float(off.max()) <= 1, f"y off by {float(off.max()):.3g} times the bound"
    assert float(((mean.double() - mu[:, 0]).abs() / (mu[:, 0].abs() * U + 130 * U * dev[:, 0])).max()) <= 1
    assert float((rstd.double() * dev[:, 0] - 1).abs().max()) <= 130 * U


@pytest.mark.parametrize("mean,std", [(1e3, 1.0), (1e5, 1.0), (-1e6, 1.0), (1e8, 20.0), (3e12, 1e6), (1.0, 1e-4)])
@pytest.mark.parametrize("cols", COLS)
def test_fp32(cols, mean, std):
    print(f"[layer norm] mean {mean} deviation {std} of {cols}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(cols)
    x, r = (mean + std * torch.randn(37, cols, generator=g, device="cuda") for _ in range(2))
    _check(x, None, 0.0, torch.float32)
    _check(x, r, 1e-5, torch.float32)


@pytest.mark.parametrize("cols", COLS)
def test_bf16(cols):
    """Values on steps of 4 about 1000: the differences are exact, the mean is between the steps."""
    print(f"[layer norm] bf16, mean 1000, of {cols}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(cols)
    x, r = ((800 + 8 * torch.randn(37, cols, generator=g, device="cuda")).bfloat16() for _ in range(2))
    _check(x, None, 0.0, torch.bfloat16)
    _check(x, r, 1e-5, torch.bfloat16)


@pytest.mark.parametrize("cols", COLS)
def test_one_element_apart(cols):
    """Rows of one value but for one element, a step of fp32 away: the least deviation that a mean can have."""
    for value in (1.0, 1e3, 1e6):
        x = torch.full((5, cols), value, device="cuda")
        up = torch.nextafter(x[:, 0], torch.full_like(x[:, 0], float("inf")))
        x[torch.arange(5), torch.tensor([0, 1, cols // 2, cols - 2, cols - 1])] = up
        _check(x, None, 0.0, torch.float32)


@pytest.mark.parametrize("cols", COLS)
def test_equal_values(cols):
    """A row of equal values is its bias, and its deviation that of eps, whatever the value."""
    x = torch.tensor([0.1, 1000.1, 1e6 / 3, 1e9 / 7, 1e15, -3.3e18], device="cuda")[:, None].expand(6, cols).contiguous()
    b = torch.randn(cols, device="cuda")
    y, _, mean, rstd = ops.add_layer_norm(x, torch.ones(cols, device="cuda"), b, eps=1e-5)
    # what is left of a difference counts for less than 2^-6 of eps^(1/2), off by 70 u of itself
    assert float((y - b).abs().max()) <= 4 * U + 2 * U * float(b.abs().max())
    assert float((mean / x[:, 0] - 1).abs().max()) <= 2 * U
    assert float((rstd * 1e-5 ** 0.5 - 1).abs().max()) <= 130 * U


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("cols", COLS)
def test_equal_values_at_the_ends_of_the_range(cols, dtype):
    """Where the row goes on at another scale: its bias all the same, with eps of any size that a root has."""
    x = torch.tensor([1e22 / 7, -3e30, 3.3e38, 1e-30, 1e-42, 0.0], device="cuda").to(dtype)
    x = x[:, None].expand(6, cols).contiguous()
    b = torch.randn(cols, device="cuda")
    for eps in (1e-5, 1e-37, 1e30):
        y, _, mean, rstd = ops.add_layer_norm(x, torch.ones(cols, device="cuda"), b, eps=eps)
        assert torch.equal(y, b.to(dtype).expand(6, cols))
        # (past half of the largest value a sum of the scaled row may round to the next step)
        assert float((mean.double() - x[:, 0].double()).abs().max()) <= 2 * U * 3.3e38
        assert bool(((mean - x[:, 0].float()).abs() <= 2 * U * x[:, 0].float().abs())[:4].all())
        assert float((rstd.double() * eps ** 0.5 - 1).abs().max()) <= 4 * U
    y, _, _, _ = ops.add_layer_norm(x, torch.ones(cols, device="cuda"), b, eps=0.0)
    assert bool(y.isnan().all())


@pytest.mark.parametrize("size", [1e-18, 1e-23, 1e-30, 1e-36])
@pytest.mark.parametrize("cols", COLS)
def test_small_deviations(cols, size):
    """Squares below fp32's smallest value, without an eps that would outweigh them: the norm is what it is at any other
    scale."""
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = size * (1 + torch.randn(9, cols, generator=g, device="cuda"))
    for eps in (0.0, 1e-42):  # (1e-42: not seen beside 1e-36; beside 1e-72 all there is)
        s = x.double()
        mu = s.mean(1, keepdim=True)
        at = float(torch.tensor(eps, dtype=torch.float32))
        dev = ((s - mu).square().mean(1, keepdim=True) + at).sqrt()
        n = (s - mu) / dev
        y, _, mean, rstd = ops.add_layer_norm(x, torch.ones(cols, device="cuda"), eps=eps)
        # (values of 1e-36 have their own steps of 2^-149, below 130 U of them)
        assert float(((y.double() - n).abs() / (130 * U * (1 + n.abs()))).max()) <= 1
        assert float((mean.double() - mu[:, 0]).abs().max()) <= 130 * U * size * 4
        assert float((rstd.double() * dev[:, 0] - 1).abs().max()) <= 130 * U
