"""Lookup in a table and the table's gradient against plain indexing and sums in 64 bits.

Tolerances: a lookup is one product, rounded once.  A gradient's row is a sum of m terms in fp32 by chunks of at most 1024
tokens and joins of at most 2^31 / 1024: off by at most (m + 1) u of the terms' magnitudes, u = 2^-24, then rounded once."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
DTYPES = [torch.bfloat16, torch.float32]
IDS = ["bf16", "fp32"]


def _strided(t, pad, shift):
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=t.dtype, device="cuda")
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v


def _tokens(g, tokens, rows, kind):
    if kind == "one":  # every token the same row
        idx = torch.full((tokens,), rows - 1, device="cuda")
    elif kind == "none":
        idx = torch.full((tokens,), -1, device="cuda")
    elif kind == "few":  # a few rows have nearly all
        idx = (torch.rand(tokens, generator=g, device="cuda") ** 6 * rows).long().clamp(0, rows - 1)
    else:
        idx = torch.randint(0, rows, (tokens,), generator=g, device="cuda")
    if kind == "holes":  # left out, and past the table
        u = torch.rand(tokens, generator=g, device="cuda")
        idx = torch.where(u < 0.2, -1 - idx, torch.where(u > 0.9, rows + idx, idx))
    return idx


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("wide", [torch.int32, torch.int64], ids=["int32", "int64"])
@pytest.mark.parametrize("tokens,rows,cols,pad,shift", [(1, 1, 1, 0, 0), (5, 3, 7, 0, 0), (16, 4000, 32, 0, 0),
                                                        (1000, 77, 301, 3, 1), (333, 50, 1024, 8, 8), (9, 2, 5000, 0, 0)])
def test_lookup(tokens, rows, cols, pad, shift, wide, dtype):
    print(f"[embed] {tokens} of {rows}x{cols} pad {pad} {wide} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(tokens + cols)
    table = _strided(torch.randn(rows, cols, generator=g, device="cuda").to(dtype), pad, shift)
    idx = _tokens(g, tokens, rows, "holes").to(wide)
    there, past = (idx >= 0) & (idx < rows), idx >= rows
    for scale in (1.0, 5.65):
        y = ops.embed(idx, table, scale=scale)
        ref = table.double()[idx.long().clamp(0, rows - 1)] * scale
        assert bool(((y.double() - ref).abs() <= (HALF[dtype] + 2 * U) * ref.abs())[there].all())
        assert bool((y[idx < 0] == 0).all()) and bool(y[past].isnan().all())
        if scale == 1.0:
            assert torch.equal(y[there], table[idx.long()[there]])


def _check_gradient(dy, idx, rows, scale, dtype):
    got = ops.embed_backward(dy, idx, rows, scale=scale)
    assert got.shape == (rows, dy.shape[1]) and got.dtype == dtype
    assert torch.equal(got, ops.embed_backward(dy, idx, rows, scale=scale)), "the same sums each time"
    i = idx.long()
    there = (i >= 0) & (i < rows)
    i, order = torch.sort(i[there])
    ends = torch.searchsorted(i, torch.arange(rows + 1, device="cuda"))
    count = (ends[1:] - ends[:-1]).double()

    def sums(t):  # of each row's tokens, as differences of running sums in 64 bits
        run = torch.cat([torch.zeros(1, t.shape[1], dtype=torch.float64, device="cuda"), t[order].cumsum(0)])
        return run[ends[1:]] - run[ends[:-1]], run[-1] * 2.0 ** -48

    mag, lost = sums(dy.double().abs()[there])
    ref = sums(dy.double()[there])[0] * scale
    tol = ((count[:, None] + 2) * U * mag + lost) * abs(scale) + HALF[dtype] * ref.abs()
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off"
    assert bool((got[count == 0] == 0).all())
    return got


# one workgroup's sort (1024 and 4096 tokens at most) and the long one (blocks of 256, 1024 and 4096), digits of 8
# and of 11 bits, chunks of 16 and more, rows over chunks, one group of columns and several
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["any", "one", "few", "holes", "none"])
@pytest.mark.parametrize("tokens,rows,cols,pad,shift", [
    (1, 1, 1, 0, 0), (17, 300, 5, 0, 0), (1024, 255, 32, 0, 0), (1025, 256, 40, 3, 1), (4097, 70_000, 24, 0, 0),
    (16_384, 3000, 96, 8, 8), (16_385, 2047, 36, 0, 0), (20_000, 2048, 700, 0, 0), (50_001, 66_000, 9, 1, 1),
    (30_000, 2, 1100, 0, 0), (65_536, 70_000, 12, 0, 0), (65_537, 2047, 20, 0, 0), (70_001, 2048, 5, 2, 1)])
def test_gradient(tokens, rows, cols, pad, shift, kind, dtype):
    print(f"[embed] gradient {tokens} of {rows}x{cols} pad {pad} {kind} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(tokens * 7 + cols)
    dy = _strided(torch.randn(tokens, cols, generator=g, device="cuda").to(dtype), pad, shift)
    idx = _tokens(g, tokens, rows, kind).to(torch.int32 if tokens % 2 else torch.int64)
    _check_gradient(dy, idx, rows, 3.0, dtype)


@pytest.mark.parametrize("tokens,rows,cols", [(1_000_000, 1600, 8), (700_001, 5_000_000, 4), (300_000, 2, 8),
                                              (262_145, 40, 130)])
def test_gradient_of_long_lists(tokens, rows, cols):
    print(f"[embed] gradient {tokens} of {rows}x{cols}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(tokens)
    dy = torch.randn(tokens, cols, generator=g, device="cuda")
    _check_gradient(dy, _tokens(g, tokens, rows, "few"), rows, 1.0, torch.float32)


def test_gradient_against_differences():
    g = torch.Generator(device="cuda").manual_seed(2)
    table, dy = torch.randn(6, 5, generator=g, device="cuda"), torch.randn(11, 5, generator=g, device="cuda")
    idx = torch.tensor([0, 3, 3, -1, 5, 0, 0, 2, 5, 3, 0], device="cuda")
    got = ops.embed_backward(dy, idx, 6, scale=2.0)
    for i in range(30):
        d = torch.zeros(30, device="cuda")
        d[i] = 1.0  # (the lookup is linear: a whole step serves)
        up, down = (ops.embed(idx, table + s * d.view(6, 5), scale=2.0).double() for s in (1, -1))
        diff = float(((up - down) / 2 * dy.double()).sum())
        # a few roundings of values up to 8 and 4 terms
        assert abs(diff - float(got.view(-1)[i])) <= 64 * U * 8


def test_no_tokens():
    idx = torch.empty(0, dtype=torch.int32, device="cuda")
    assert ops.embed(idx, torch.ones(3, 4, device="cuda")).shape == (0, 4)
    assert bool((ops.embed_backward(torch.empty(0, 4, device="cuda"), idx, 1000) == 0).all())


def test_captured():
    g = torch.Generator(device="cuda").manual_seed(4)
    dy, idx = torch.randn(20_000, 16, generator=g, device="cuda"), torch.randint(0, 500, (20_000,), generator=g, device="cuda")
    small = idx[:700].clone()
    ops.embed_backward(dy, idx, 500)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        long, short = ops.embed_backward(dy, idx, 500), ops.embed_backward(dy[:700], small, 500)
    for t in range(3):
        dy.copy_(torch.randn(20_000, 16, generator=g, device="cuda"))
        idx.copy_(torch.randint(-5, 500, (20_000,), generator=g, device="cuda"))
        small.copy_(idx[-700:])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(long, ops.embed_backward(dy, idx, 500))
        assert torch.equal(short, ops.embed_backward(dy[:700], small, 500))
