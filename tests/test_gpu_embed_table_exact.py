"""The table's gradient of whole numbers, whose sums are exact in fp32 in any order: each row equals the sum of all of its
tokens, so a token, a chunk or a part that is left out or added twice shows in rows of any length.

Values are whole numbers up to 8 and lists have at most 2,000,000 tokens, so sums stay below 2^24; the scale is a power of two;
results in bf16 are the exact sum, rounded once."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]
IDS = ["bf16", "fp32"]


def _tokens(g, tokens, rows, kind):
    u = torch.rand(tokens, generator=g, device="cuda", dtype=torch.float64)
    if kind == "one":  # the last row has them all
        return torch.full((tokens,), rows - 1, device="cuda")
    if kind == "few":  # the first rows have nearly all
        return (u ** 6 * rows).long()
    if kind == "runs":  # in blocks of equal tokens, with ones of no row between them
        idx = (torch.arange(tokens, device="cuda") // 37 * 7919) % (rows + 2) - 1
        return torch.where(u < 0.01, rows + 5, idx)
    return (u * rows).long()


def _sums(dy, idx, rows, dtype=torch.int64):
    """Of each row's tokens, as differences of running sums: exact in int64, in float64 far below fp32's roundings."""
    there = (idx >= 0) & (idx < rows)
    i, order = torch.sort(idx[there])
    run = torch.cat([torch.zeros(1, dy.shape[1], dtype=dtype, device="cuda"), dy[there][order].to(dtype).cumsum(0)])
    ends = torch.searchsorted(i, torch.arange(rows + 1, device="cuda"))
    return run[ends[1:]] - run[ends[:-1]]


def _check(tokens, rows, cols, kind, dtype, scale=0.5, pad=0):
    g = torch.Generator(device="cuda").manual_seed(tokens + rows + cols)
    dy = torch.full((tokens, cols + pad), float("nan"), dtype=dtype, device="cuda")[:, :cols]
    dy.copy_(torch.randint(-8, 9, (tokens, cols), generator=g, device="cuda"))
    dy[:, 0] = 8  # (a column whose sums grow with the tokens)
    idx = _tokens(g, tokens, rows, kind)
    want = _sums(dy, idx, rows)
    assert int(want.abs().max()) < 1 << 24
    got = ops.embed_backward(dy, idx.int() if tokens % 2 else idx, rows, scale=scale)
    wrong = got != (want.float() * scale).to(dtype)
    assert not bool(wrong.any()), f"{int(wrong.any(1).sum())} rows wrong, the first {wrong.any(1).nonzero()[:4, 0].tolist()}"


# every sort (one workgroup of 1024 and 4096 tokens, blocks of 256, 1024 and 4096, digits of 8 and 11 bits) and every join (256
# and 1024 threads, 1 to 16 chunks a block, rows of a few chunks to thousands, one group of columns and several)
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["any", "one", "few", "runs"])
@pytest.mark.parametrize("tokens,rows,cols", [
    (33, 3, 5), (1024, 255, 32), (1025, 256, 40), (4096, 1, 300), (4097, 70_000, 24), (16_384, 3000, 96), (16_385, 2047, 36),
    (20_000, 2048, 700), (30_000, 2, 1100), (50_001, 66_000, 9), (65_536, 70_000, 12), (65_537, 2047, 20), (70_001, 2048, 5),
    (131_072, 7, 520), (262_145, 40, 130), (300_000, 2, 8), (1_000_000, 1600, 32), (1_000_000, 2, 32), (700_001, 5_000_000, 4),
    (2_000_000, 300, 3), (2_000_000, 1, 16)])
def test_whole_numbers(tokens, rows, cols, kind, dtype):
    print(f"[embed] whole numbers, {tokens} of {rows}x{cols} {kind} {dtype}", flush=True)
    _check(tokens, rows, cols, kind, dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("tokens", [15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_rows_that_end_at_a_chunk(tokens, dtype):
    """Rows of each length about a chunk's, one behind the other: they begin and end on, before and behind chunks' borders."""
    print(f"[embed] rows of {tokens} tokens, {dtype}", flush=True)
    cols = 12
    g = torch.Generator(device="cuda").manual_seed(tokens)
    for lead in (0, 1, 16, 31):  # tokens of row 0 before them
        idx = torch.cat([torch.zeros(lead, dtype=torch.long, device="cuda"),
                         1 + torch.arange(40, device="cuda").repeat_interleave(tokens)])
        dy = torch.randint(-8, 9, (idx.numel(), cols), generator=g, device="cuda").to(dtype)
        want = _sums(dy, idx, 41)
        assert torch.equal(ops.embed_backward(dy, idx, 41, scale=2.0), (want.float() * 2).to(dtype))
        order = torch.randperm(idx.numel(), generator=g, device="cuda")
        assert torch.equal(ops.embed_backward(dy[order], idx[order], 41, scale=2.0), (want.float() * 2).to(dtype))


@pytest.mark.parametrize("tokens,rows,cols,kind", [(1_000_000, 1600, 8, "few"), (262_145, 40, 130, "few"), (300_000, 2, 8, "few"),
                                                   (30_000, 2, 1100, "any")])
def test_real_numbers(tokens, rows, cols, kind):
    """Off by the additions that a term goes through, not by the tokens of its row: a chunk's (1024 at most) and those of the
    join (in these layouts at most tokens / 1024 chunks of a row to a group of threads, and 9 halvings), u = 2^-24 of the
    magnitudes each."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    dy = torch.randn(tokens, cols, generator=g, device="cuda")
    idx = _tokens(g, tokens, rows, kind)
    ref, mag = _sums(dy, idx, rows, torch.float64), _sums(dy.abs(), idx, rows, torch.float64)
    got = ops.embed_backward(dy, idx, rows)
    steps = 1024 + tokens / 1024 + 16
    bad = (got.double() - ref).abs() > steps * 2.0 ** -24 * mag
    assert not bool(bad.any())
    # and in all the sums' own deviation counts: a random walk of roundings, sqrt(steps) u of the magnitudes
    assert float((got.double() - ref).norm()) <= 4 * steps ** 0.5 * 2.0 ** -24 * float(mag.norm())
