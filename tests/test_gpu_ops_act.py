"""Activations of the gated block and of gated 8-bit products on their own, relative to the activation's value: the
products around them are exact (one gate value and one up value a row), so what is off is the activation's.

Bounds (u = 2^-24): an exponent g log2(e) is rounded twice beside its constant, 1.5 u |g| of the exponential, and the
half square of g three times, 1.25 u g^2; the hardware's exponential and reciprocal are off by 2 u each, a polynomial of
eight terms and the products around it by less than 20 u.  bf16 results add half a step each time they are rounded."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from scipy.special import erfc  # noqa: E402

from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
DTYPES = [torch.bfloat16, torch.float32]


def _act(name, g):
    """act(g) and the relative error allowed; act'(g) and the absolute one."""
    if name == "silu":
        p = 1 / (1 + np.exp(-g))
        rel = (2 * np.abs(g) + 16) * U
        a, b = p, g * p * (1 - p)
        return g * p, rel, a + b, (np.abs(a) + np.abs(b)) * ((3 * np.abs(g) + 24) * U)
    c = 0.5 * erfc(-g / np.sqrt(2))
    rel = (1.5 * g * g + 32) * U
    a, b = c, g * np.exp(-0.5 * g * g) / np.sqrt(2 * np.pi)
    return g * c, rel, a + b, (np.abs(a) + np.abs(b)) * rel


def _off(got, ref, tol):
    off = np.abs(got.detach().double().cpu().numpy() - ref)
    worst = int(np.argmax(off - tol))
    return None if (off <= tol).all() else (worst, off[worst], tol[worst])


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "fp32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("tokens", [5, 300, 4001])
def test_gated_ff_activation(tokens, act, dtype):
    print(f"[act] {tokens} {act} {dtype}", flush=True)
    # multiples of 1/8 up to 12 have at most 7 bits, so bf16 holds them
    g = (np.round(np.linspace(-12, 12, tokens) * 8) / 8).astype(np.float32)
    x = torch.from_numpy(np.stack([g, np.ones_like(g)], 1)).to(dtype).cuda()
    eye, one = torch.eye(2, device="cuda").to(dtype), torch.ones(1, 1, device="cuda").to(dtype)
    y, saved = ops.gated_ff(x, eye, one, act=act, save=True)
    g = g.astype(np.float64)
    v, rel, d, dtol = _act(act, g)
    assert torch.equal(saved[0], x.float())
    tol = np.abs(v) * (rel + 2 * HALF[dtype]) + 1e-40
    assert _off(y[:, 0], v, tol) is None, _off(y[:, 0], v, tol)
    dy = torch.ones(tokens, 1, device="cuda").to(dtype)
    dx, _, _ = ops.gated_ff_backward(dy, x, eye, one, saved, act=act)
    assert _off(dx[:, 1], v, tol) is None, _off(dx[:, 1], v, tol)
    tol = dtol + np.abs(d) * 2 * HALF[dtype] + 1e-40
    assert _off(dx[:, 0], d, tol) is None, _off(dx[:, 0], d, tol)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows", [1, 256, 4096])
def test_q8_activation(rows, act):
    print(f"[act] q8 {rows} {act}", flush=True)
    # codes times 1/16: gates in [-8, 8), the up value 1/16
    a = np.resize(np.arange(-128, 128), rows)
    a[0] = -100
    x = torch.from_numpy(np.stack([a, np.ones_like(a)], 1).astype(np.int8)).cuda()
    out = ops.q8_matmul(x, torch.full((rows,), 1 / 16, device="cuda"), torch.eye(2, device="cuda").to(torch.int8),
                        torch.ones(2, device="cuda"), gate=act, dtype=torch.float32)
    v, rel, _, _ = _act(act, a / 16.0)
    assert _off(out[:, 0], v / 16, np.abs(v) / 16 * rel) is None, _off(out[:, 0], v / 16, np.abs(v) / 16 * rel)
