"""8-bit floating point products on each kind of tile, whole and split depths, straight to LDS and through registers
(tests/test_f8_tiles.py holds the sizes to the tiles): within the bounds of test_gpu_f8.py, and exactly where sums of whole numbers times powers of two are exact."""
import pytest

torch = pytest.importorskip("torch")
from f8_tile_cases import ALL  # noqa: E402
from paper_2607_05380_amd import ops  # noqa: E402
from test_gpu_f8 import _check_product, _strided  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("case,layout", ALL, ids=str)
def test_product(case, layout, bias):
    print(f"[f8 tiles] {case} on {layout} bias {bias}", flush=True)
    M, N, K, gate, fp32, pad, shift = case
    _check_product(M, N, K, gate, pad, shift, bias, torch.float32 if fp32 else torch.bfloat16)


@pytest.mark.parametrize("case,layout", ALL, ids=str)
def test_exact_sums(case, layout):
    """Codes of -1, 0 and 1 and scales 2^-3 .. 2^3 of their own for each block: sums are multiples of 2^-6, at most 64 a
    product, so below 2^18 at depth 4096 (past it, scales 2^-1 .. 2^1: at most 4 a product): exact in fp32 in any order, and no product
    lies far enough below another one to be cut off.  A row, a column or a block of the depth that is left out, taken
    twice or scaled by another one's scale shows."""
    print(f"[f8 tiles] exact {case} on {layout}", flush=True)
    M, N, K, gate, fp32, pad, shift = case
    gate = gate and "relu"
    dtype = torch.float32 if fp32 else torch.bfloat16
    parts, blocks, tiles = 2 if gate else 1, -(-K // 128), -(-N // 128)
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    top = 4 if K <= 4200 else 2

    def codes(rows):
        return torch.randint(-1, 2, (rows, K), generator=g, device="cuda").float()

    def scales(*shape):
        return torch.exp2(torch.randint(1 - top, top, shape, generator=g, device="cuda").float())

    x, w, sx, sw = codes(M), codes(parts * N), scales(blocks, M), scales(parts * tiles, blocks)
    bias = torch.randint(-100, 101, (parts * N,), generator=g, device="cuda").float()
    qx, qw = (_strided(t.to(torch.float8_e4m3fn), pad, shift) for t in (x, w))
    got = ops.f8_matmul(qx, sx, qw, sw, bias=bias, gate=gate, dtype=dtype)
    X = x.double() * sx.double().t().repeat_interleave(128, 1)[:, :K]
    out = []
    for i in range(parts):
        s = sw[i * tiles:(i + 1) * tiles].double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
        out.append(X @ (w[i * N:(i + 1) * N].double() * s).t() + bias[i * N:(i + 1) * N].double())
    assert max(float(o.abs().max()) for o in out) < 2 ** 18
    want = out[0] if not gate else torch.relu(out[0]).float() * out[1].float()
    want = want.float().to(dtype)
    wrong = got != want
    assert not bool(wrong.any()), (f"{int(wrong.sum())} of {wrong.numel()} wrong, rows "
                                   f"{wrong.any(1).nonzero()[:4, 0].tolist()}, columns {wrong.any(0).nonzero()[:4, 0].tolist()}")
