"""Products whose rows end inside a 16-byte vector, at sizes where their operands are copied to aligned rows first: what
lies behind a row (NaN here), where rows start and what memory held before must not reach a result."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu


def _view(t, ld, shift):
    """t's values in rows ld apart from element shift on, the rest NaN (int8: a large code)."""
    rows, cols = t.shape
    buf = torch.full((rows * ld + shift + 16,), float("nan") if t.is_floating_point() else 101, dtype=t.dtype,
                     device="cuda")
    v = buf[shift:shift + rows * ld].view(rows, ld)[:, :cols]
    v.copy_(t)
    return v


def _poison():
    """Leaves NaN in the memory that the next allocations get."""
    for n in (1 << 16, 1 << 20, 1 << 22, 1 << 24):
        held = [torch.full((n,), float("nan"), device="cuda") for _ in range(3)]
        del held


# tokens, d_in, hidden, d_out: one extent odd at a time and all, a split depth of the gate projections
BLOCKS = [(2050, 515, 1027, 261), (2048, 512, 1025, 256), (2048, 513, 1024, 256), (2051, 512, 1024, 259),
          (300, 9001, 203, 101), (4000, 510, 2044, 514)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("case", BLOCKS, ids=lambda c: "x".join(map(str, c)))
def test_gated_ff_odd(case, dtype):
    T, D, F, O = case
    VE = 16 // dtype.itemsize
    print(f"[odd] {T} {D} {F} {O} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(T + D + F)

    def rand(r, c, std=1.0):
        return (torch.randn(r, c, generator=g, device="cuda") * std).to(dtype)

    x, wg, wd = rand(T, D), rand(2 * F, D, D ** -0.5), rand(O, F, F ** -0.5)
    r, dy = rand(T, O), rand(T, O)
    _poison()
    y, saved = ops.gated_ff(x, wg, wd, residual=r, save=True)
    grads = ops.gated_ff_backward(dy, x, wg, wd, saved)
    torch.cuda.synchronize()
    # (far from the rounding bounds, which the other tests check: a NaN or a misplaced row is what is looked for)
    G = x.double() @ wg.double().t()
    H = torch.nn.functional.silu(G[:, :F]) * G[:, F:]
    Y = H @ wd.double().t() + r.double()
    assert float((y.double() - Y).abs().max()) <= 0.05 * float(Y.abs().max())
    S, HS = saved[0].double(), saved[1].double()
    s = torch.sigmoid(S[:, :F])
    DH = dy.double() @ wd.double()
    DGU = torch.cat([DH * S[:, F:] * s * (1 + S[:, :F] * (1 - s)), DH * S[:, :F] * s], 1)
    for got, ref in zip(grads, (DGU @ wg.double(), DGU.t() @ x.double(), dy.double().t() @ HS)):
        assert float((got.double() - ref).abs().max()) <= 0.05 * float(ref.abs().max())
    # rows at 16 bytes with NaN inside their last vector, and rows at any element: the same products of the same copies
    for pad, shift in ((VE - 1, 0), (3, 1)):
        ld = [(n + pad) // VE * VE if shift == 0 else n + pad for n in (D, F, O)]
        a = (_view(x, ld[0], shift), _view(wg, ld[0], shift), _view(wd, ld[1], shift))
        rv, dv = _view(r, ld[2], shift), _view(dy, ld[2], shift)
        _poison()
        y2, saved2 = ops.gated_ff(*a, residual=rv, save=True)
        if all(n % VE for n in (D, F, O)):  # (otherwise unaligned views of aligned extents pass through registers)
            assert torch.equal(y2, y)
        assert float((y2.double() - Y).abs().max()) <= 0.05 * float(Y.abs().max())
        again = ops.gated_ff_backward(dv, *a, saved)
        for got, ref in zip(again, grads):
            if all(n % VE for n in (D, F, O)):
                assert torch.equal(got, ref)
            assert float((got.double() - ref.double()).abs().max()) <= 0.05 * float(ref.abs().max())
    # saved values that went through a copy
    _poison()
    kept = (saved[0].clone(), saved[1].cpu().cuda().contiguous())
    for got, ref in zip(ops.gated_ff_backward(dy, x, wg, wd, kept), grads):
        assert torch.equal(got, ref)


@pytest.mark.parametrize("gate", [None, "gelu"])
@pytest.mark.parametrize("M,N,K", [(8011, 1027, 1023), (6000, 4095, 1010), (3001, 1024, 4095)])
def test_q8_matmul_odd(M, N, K, gate):
    print(f"[odd] q8 {M} {N} {K} {gate}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    rows = 2 * N if gate else N
    x = torch.randint(-127, 128, (M, K), generator=g, device="cuda").to(torch.int8)
    w = torch.randint(-127, 128, (rows, K), generator=g, device="cuda").to(torch.int8)
    xs, ws = torch.rand(M, generator=g, device="cuda") * 1e-3, torch.rand(rows, generator=g, device="cuda") * 1e-2
    _poison()
    out = ops.q8_matmul(x, xs, w, ws, gate=gate, dtype=torch.float32)
    # sums in integers are exact, so any path gives these bits
    few = torch.arange(0, M, 97, device="cuda")
    Z = (x[few].double() @ w.double().t()) * xs[few].double()[:, None] * ws.double()
    ref = Z if gate is None else torch.nn.functional.gelu(Z[:, :N]) * Z[:, N:]
    tol = 64 * 2.0 ** -24 * (ref.abs() + float(ref.abs().max()))
    assert bool(((out[few].double() - ref).abs() <= tol).all())
    for pad, shift in ((15, 0), (3, 5)):
        ld = (K + pad) // 16 * 16 if shift == 0 else K + pad
        _poison()
        got = ops.q8_matmul(_view(x, ld, shift), xs, _view(w, ld, shift), ws, gate=gate, dtype=torch.float32)
        assert torch.equal(got, out)
