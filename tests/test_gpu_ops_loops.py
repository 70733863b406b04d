"""Row kernels whose blocks take several rows one after the other: the norm's gradients, whose blocks are at most 1024,
in every layout, against the formula in 64 bits on the device; the forward kernels and distillation past the 2^20 blocks
of a launch, against the same rows in calls that fit one.

Bounds as in test_gpu_ops_rows.py: u = 2^-24 per fp32 operation and half a bf16 step where a result is rounded."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops, tabpack  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
DTYPES = [torch.bfloat16, torch.float32]
IDS = ["bf16", "fp32"]
GRID = 1 << 20  # blocks of a launch over rows


def _blocks(rows, cols):
    """Blocks of the norm's backward kernel: each has a row of `cols` fp32 sums in the workspace."""
    n = ctypes.c_size_t()
    assert tabpack.load_library().pack_rms_norm_backward_workspace_size(rows, cols, ctypes.byref(n)) == 0
    return n.value // (4 * cols)


def _per_block(cols):
    """Rows that a block of a row kernel takes at a time: 256 threads, 4, 16 or 64 a row; wider rows a block each."""
    return 64 if cols <= 32 else 16 if cols <= 128 else 4 if cols <= 2048 else 1


def _close(got, ref, tol, what):
    off = (got.double() - ref).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst ratio {float((off / tol).max())}"


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("rows,cols", [(66_000, 8), (200_003, 21), (16_500, 64), (50_001, 100), (4_200, 512),
                                       (13_001, 1024), (8_201, 2001), (2_100, 2049), (3_333, 8000), (2_100, 8200),
                                       (3_101, 16_384), (1_100, 20_000)])
def test_norm_backward_over_several_rows_a_block(rows, cols, dtype):
    blocks, per = _blocks(rows, cols), _per_block(cols)
    assert rows > blocks * per, "every block has to go on to a second row"
    print(f"[loops] norm backward {rows}x{cols} {dtype}: {blocks} blocks of {per}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    v, dy, ds = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(3))
    w = 1 + 0.3 * torch.randn(cols, generator=g, device="cuda")
    rstd = (v.double().square().mean(1) + 1e-5).rsqrt().float()
    V, DY, DS, W, R = v.double(), dy.double(), ds.double(), w.double(), rstd.double()[:, None]
    G, N = DY * W, v.double() * R
    mag = (G.abs() + N.abs() / cols * (G * N).abs().sum(1, keepdim=True)) * R
    # a thread's rows one after the other, the block's row groups, its share of the blocks and their 64 streams
    adds = rows / (blocks * per) + 1 + per + blocks / 64 + 64
    for dv in (ds, None):
        dx, dw = ops.rms_norm_backward(dy, v, w, rstd, dv=dv)
        again = ops.rms_norm_backward(dy, v, w, rstd, dv=dv)
        assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
        ref = R * (G - N / cols * (G * N).sum(1, keepdim=True))
        add = torch.zeros_like(V) if dv is None else DS
        ref = ref + add
        _close(dx, ref, ref.abs() * HALF[dtype] + 64 * U * (mag + add.abs()), "dx")
        _close(dw, (DY * N).sum(0), (adds + 8) * U * (DY * N).abs().sum(0), "dweight")


def _pieces(rows, size):
    return [(i, min(i + size, rows)) for i in range(0, rows, size)]


# a row by 4, 16 and 64 threads, several rows a block; by 256 and by 1024, whose rows share a block's barriers
@pytest.mark.parametrize("rows,cols", [((1 << 26) + 77, 8), ((1 << 24) + 77, 40), ((1 << 22) + 77, 136),
                                       ((1 << 20) + 300, 2056), ((1 << 20) + 300, 8200)])
def test_rows_past_one_launch(rows, cols):
    per = _per_block(cols)
    assert rows > GRID * per
    print(f"[loops] rows {rows}x{cols}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = torch.rand(cols, generator=g, device="cuda") + 0.5
    for call in (lambda t: ops.add_rms_norm(t, w, residual=t), lambda t: ops.add_rms_norm_q8(t, w),
                 ops.quantize_rows):
        whole = call(x)
        for lo, hi in _pieces(rows, GRID * per // 2):
            for a, b in zip(whole, call(x[lo:hi])):
                assert torch.equal(a[lo:hi], b), (lo, hi)
        del whole


@pytest.mark.parametrize("rows,classes,k", [((1 << 26) + 77, 8, 2), ((1 << 24) + 77, 40, 3), ((1 << 22) + 77, 136, 5),
                                            ((1 << 20) + 300, 1030, 5), ((1 << 20) + 300, 8200, 9)])
def test_distillation_past_one_launch(rows, classes, k):
    # 4 and 16 threads a row (64 and 16 rows a block), a wave, 256 and 512 threads
    per = 64 if classes <= 32 else 16 if classes <= 128 else 4 if classes <= 1024 else 1
    assert rows > GRID * per
    print(f"[loops] distill {rows}x{classes} k {k}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(classes)
    z = torch.empty(rows, classes, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    idx = torch.randint(-1, classes, (rows, k), generator=g, device="cuda", dtype=torch.int32)
    t = torch.randn(rows, k, generator=g, device="cuda")
    weight = (torch.rand(rows, generator=g, device="cuda") - 0.1).clamp(min=0)
    for grad in (True, False):  # (without the gradient a row has no barrier of its own)
        whole = ops.distill_topk(z, idx, t, temperature=1.5, row_weight=weight, grad=grad)
        for lo, hi in _pieces(rows, GRID * per // 2):
            part = ops.distill_topk(z[lo:hi], idx[lo:hi], t[lo:hi], temperature=1.5, row_weight=weight[lo:hi],
                                    grad=grad)
            assert torch.equal(whole[0][lo:hi], part[0]), (lo, hi)
            assert not grad or torch.equal(whole[1][lo:hi], part[1]), (lo, hi)
        del whole
