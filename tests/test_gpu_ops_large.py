"""Student operators at sizes that fill the chip (the largest tiles, split depths of the weight gradients) against the
formulas in float64 on the device, and under HIP graph capture.  Error bounds as in test_gpu_ops_block.py."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


def _act(name, g):
    """act(g), act'(g) and their errors where g is exact (an exponent is off by up to 3 u (|g| + g^2))."""
    if name == "silu":
        p = torch.sigmoid(g)
        v, d = g * p, p * (1 + g * (1 - p))
    else:
        c = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
        v, d = g * c, c + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    e = (1 + g.abs()) * (4 * g.abs() + 16) * U
    return v, d, e, e * (1 + g.abs())


def _close(got, ref, tol, what):
    off = (got.double() - ref).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst ratio {float((off / tol).max())}"


def _sum_err(n):
    return 2 * (n + 2) * U


@pytest.mark.parametrize("T,D,F,O,act,dtype", [
    (4100, 520, 2056, 1032, "silu", torch.bfloat16),     # 256 x 256 tiles with edges in both directions
    (4100, 515, 2051, 1029, "gelu", torch.bfloat16),     # the same from aligned copies
    (9000, 128, 1024, 128, "silu", torch.bfloat16),      # long token axis: split weight gradients
    (1500, 264, 520, 136, "gelu", torch.float32),
    (100, 2048, 4096, 2048, "silu", torch.bfloat16)], ids=str)
def test_gated_ff_large(T, D, F, O, act, dtype):
    print(f"[large] {T} {D} {F} {O} {act} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(T + D)

    def rand(r, c, std=1.0):
        return (torch.randn(r, c, generator=g, device="cuda") * std).to(dtype)

    x, wg, wd = rand(T, D), rand(2 * F, D, D ** -0.5), rand(O, F, F ** -0.5)
    r, dy = rand(T, O), rand(T, O)
    y, saved = ops.gated_ff(x, wg, wd, act=act, residual=r, save=True)
    gu, h = saved
    dx, dwg, dwd = ops.gated_ff_backward(dy, x, wg, wd, saved, act=act)
    X, WG, WD, DY = (t.double() for t in (x, wg, wd, dy))
    half = HALF[dtype]
    GU = X @ WG.t()
    eGU = _sum_err(D) * (X.abs() @ WG.abs().t())
    _close(gu, GU, eGU + half * (GU.abs() + eGU), "gate and up")
    V, _, eV, _ = _act(act, GU[:, :F])
    eV = eV + 1.2 * eGU[:, :F]
    UP, eU = GU[:, F:], eGU[:, F:]
    H = V * UP
    eH = eV * (UP.abs() + eU) + V.abs() * eU + 2 * U * H.abs()
    eH = eH + half * (H.abs() + eH)
    _close(h, H, eH, "hidden")
    Y = H @ WD.t()
    eY = eH @ WD.abs().t() + _sum_err(F) * ((H.abs() + eH) @ WD.abs().t())
    Y = Y + r.double()
    _close(y, Y, eY + 2 * half * (Y.abs() + eY), "y + residual")
    S, HS = gu.double(), h.double()
    V, DV, eV, eDV = _act(act, S[:, :F])
    UP = S[:, F:]
    DH = DY @ WD
    eDH = _sum_err(O) * (DY.abs() @ WD.abs())
    DG, DU = DH * UP * DV, DH * V
    eDG = UP.abs() * (eDH * (DV.abs() + eDV) + DH.abs() * eDV) + 4 * U * DG.abs()
    eDU = eDH * (V.abs() + eV) + DH.abs() * eV + 4 * U * DU.abs()
    DGU, eDGU = torch.cat([DG, DU], 1), torch.cat([eDG, eDU], 1)
    eDGU = eDGU + half * (DGU.abs() + eDGU)

    def product(a, b, e, what, got):
        ref = a @ b
        tol = e @ b.abs() + _sum_err(a.shape[1]) * ((a.abs() + e) @ b.abs())
        _close(got, ref, tol + half * (ref.abs() + tol), what)

    product(DGU, WG, eDGU, "dx", dx)
    product(DGU.t(), X, eDGU.t(), "dw_gate_up", dwg)
    product(DY.t(), HS, torch.zeros_like(DY.t()), "dw_down", dwd)
    again, saved2 = ops.gated_ff(x, wg, wd, act=act, residual=r, save=True)
    assert torch.equal(again, y)
    for a, b in zip(ops.gated_ff_backward(dy, x, wg, wd, saved2, act=act), (dx, dwg, dwd)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("gate", [None, "silu", "gelu"])
@pytest.mark.parametrize("M,N,K", [(4100, 2056, 1040), (4099, 2051, 1035), (9000, 520, 256), (300, 256, 20_000)])
def test_q8_matmul_large(M, N, K, gate):
    print(f"[large] q8 {M} {N} {K} {gate}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    rows = 2 * N if gate else N
    x = torch.randint(-127, 128, (M, K), generator=g, device="cuda").to(torch.int8)
    w = torch.randint(-127, 128, (rows, K), generator=g, device="cuda").to(torch.int8)
    xs = torch.rand(M, generator=g, device="cuda") * 1e-2 + 1e-3
    ws = torch.rand(rows, generator=g, device="cuda") / (60 * math.sqrt(K)) + 1e-5
    b = torch.randn(rows, generator=g, device="cuda")
    S = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()
    Z = S + b.double()
    e = 4 * U * (S.abs() + Z.abs())
    if gate is None:
        ref, tol = Z, e
    else:
        V, _, eV, _ = _act(gate, Z[:, :N])
        eV = eV + 1.2 * e[:, :N]
        ref = V * Z[:, N:]
        tol = eV * (Z[:, N:].abs() + e[:, N:]) + V.abs() * e[:, N:] + 2 * U * ref.abs()
    for dtype in (torch.bfloat16, torch.float32):
        out = ops.q8_matmul(x, xs, w, ws, bias=b, gate=gate, dtype=dtype)
        _close(out, ref, tol + HALF[dtype] * (ref.abs() + tol), f"{gate} {dtype}")


@pytest.mark.parametrize("T", [1, 37, 700])
def test_ops_in_a_graph(T):
    """A block's serving and training calls captured once and replayed, with eager work between the replays."""
    D, F, V = 136, 264, 40
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    norm = torch.rand(D, generator=g, device="cuda") + 0.5
    wg = torch.randn(2 * F, D, generator=g, device="cuda").bfloat16()
    wd = torch.randn(D, F, generator=g, device="cuda").bfloat16()
    wh = torch.randn(V, D, generator=g, device="cuda").bfloat16()
    (qg, sg), (qd, sd), (qh, sh) = (ops.quantize_rows(t) for t in (wg, wd, wh))
    idx = torch.randint(0, V, (T, 5), generator=g, device="cuda", dtype=torch.int32)
    teacher = torch.randn(T, 5, generator=g, device="cuda")

    def step(x):
        n, v, rstd = ops.add_rms_norm(x, norm, residual=x)
        y, saved = ops.gated_ff(n, wg, wd, residual=v, save=True)
        q, s, _ = ops.add_rms_norm_q8(y, norm)
        h = ops.q8_matmul(q, s, qg, sg, gate="silu")
        q, s = ops.quantize_rows(h)
        z = ops.q8_matmul(*ops.quantize_rows(ops.q8_matmul(q, s, qd, sd)), qh, sh)
        loss, dz = ops.distill_topk(z, idx, teacher, temperature=2.0)
        dn, dwg, dwd = ops.gated_ff_backward(y, n, wg, wd, saved)
        dx, dw = ops.rms_norm_backward(dn, v, norm, rstd, dv=y)
        return y, z, loss, dz, dwg, dwd, dx, dw

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(x)
    for turn in range(4):
        x.copy_(torch.randn(T, D, generator=g, device="cuda"))
        refs = step(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(outs, refs)):
            assert torch.equal(a, b), (turn, i)
