"""8-bit floating point codes of more rows, and more tiles, than one launch takes: the same codes and scales as of
the same rows in pieces."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu


def _rows(rows, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.empty(rows, cols, dtype=dtype, device="cuda")
    piece = torch.randn(1_000_003, cols, generator=g, device="cuda").to(dtype)  # (no multiple of a workgroup's rows)
    for at in range(0, rows, piece.shape[0]):
        x[at:at + piece.shape[0]] = piece[:rows - at]
    x[-5] = torch.arange(cols, device="cuda") * 3 + 1
    x[-3, 0] = float("inf")
    return x


# 16 rows a workgroup, of which a launch takes 2^23
@pytest.mark.parametrize("rows,cols,dtype", [(270_000_003, 8, torch.bfloat16), (17_000_001, 130, torch.float32)], ids=str)
def test_rows(rows, cols, dtype):
    print(f"[f8] {rows}x{cols} {dtype}", flush=True)
    x = _rows(rows, cols, dtype)
    q, s = ops.quantize_blocks(x)
    step = 16_000_000  # (pieces of one launch each)
    for at in range(0, rows, step):
        part, scale = ops.quantize_blocks(x[at:at + step])
        assert torch.equal(q.view(torch.uint8)[at:at + step], part.view(torch.uint8))
        assert torch.equal(s[:, at:at + step].nan_to_num(-1.0), scale.nan_to_num(-1.0))
    assert bool(s[0, -3].isnan()) and not q[-3, :8].float().any()


@pytest.mark.parametrize("gated", [False, True])
def test_tiles(gated):
    rows, cols = 1_100_000_000, 9  # 128 rows a workgroup
    print(f"[f8] tiles of {rows}x{cols}", flush=True)
    x = _rows(rows, cols, torch.bfloat16)
    q, s = ops.quantize_tiles(x, gated=gated)
    half = rows // 2 if gated else rows
    assert s.shape == (rows // half * -(-half // 128), 1)
    step = 128 * 500_000
    for first in range(0, rows, half):
        for at in range(0, half, step):
            end = min(at + step, half)
            part, scale = ops.quantize_tiles(x[first + at:first + end])
            assert torch.equal(q.view(torch.uint8)[first + at:first + end], part.view(torch.uint8))
            tile = first // half * -(-half // 128) + at // 128
            assert torch.equal(s[tile:tile + scale.shape[0]].nan_to_num(-1.0), scale.nan_to_num(-1.0))
