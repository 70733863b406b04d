"""Layer norm, dropout, embeddings and 8-bit floating point as users call them: under grad mode, on another stream, two
streams at once, captured and replayed, in place through the C ABI."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops, tabpack  # noqa: E402

pytestmark = pytest.mark.gpu


def _calls(rows=6):
    """(name, call, its floating tensors) of every operator."""
    g = torch.Generator(device="cuda").manual_seed(1)

    def rand(*s):
        return torch.randn(*s, generator=g, device="cuda")

    x, r, w, b, dy, dv = rand(rows, 40), rand(rows, 40), rand(40), rand(40), rand(rows, 40), rand(rows, 40)
    mean, rstd = rand(rows), rand(rows).abs()
    idx = torch.randint(-1, 9, (rows,), generator=g, device="cuda")
    q, s = ops.quantize_blocks(x)
    qw, sw = ops.quantize_tiles(rand(24, 40), gated=True)
    bias = rand(24)
    return [
        ("add_layer_norm", lambda x, w, b, r: ops.add_layer_norm(x, w, b, residual=r), (x, w, b, r)),
        ("layer_norm_backward", lambda dy, v, w, m, rho, dv: ops.layer_norm_backward(dy, v, w, m, rho, dv=dv),
         (dy, x, w, mean, rstd, dv)),
        ("dropout", lambda x, r: ops.dropout(x, 0.5, 1, 2, residual=r), (x, r)),
        ("embed", lambda t: ops.embed(idx, t, 2.0), (x,)),
        ("embed_backward", lambda dy: ops.embed_backward(dy, idx, 9), (dy,)),
        ("quantize_blocks", ops.quantize_blocks, (x,)),
        ("quantize_tiles", ops.quantize_tiles, (x,)),
        ("f8_matmul", lambda s, sw, b: ops.f8_matmul(q, s, qw, sw, bias=b, gate="gelu"), (s, sw, bias))]


def _flat(out):
    return [t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in
            (out if isinstance(out, tuple) else (out,))]


def _same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(_flat(a), _flat(b)))


def test_a_lost_gradient_is_refused():
    for name, call, tensors in _calls():
        want = call(*tensors)
        for i in range(len(tensors)):
            args = [t.detach().clone().requires_grad_(j == i) for j, t in enumerate(tensors)]
            print(f"[grad mode] {name}, tensor {i}", flush=True)
            with pytest.raises(tabpack.PackError, match="no_grad"):
                call(*args)
            with torch.no_grad():
                assert _same(call(*args), want)


def test_another_stream_and_two_at_once():
    calls = _calls(300)
    want = [call(*t) for _, call, t in calls]
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    got = [[], []]
    for k, stream in enumerate((one, two)):
        stream.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = [[], []]
        for (name, call, t) in calls:
            for k, stream in enumerate((one, two)):
                with torch.cuda.stream(stream):
                    got[k].append(call(*t))
        torch.cuda.synchronize()
        for k in range(2):
            for (name, _, _), a, b in zip(calls, got[k], want):
                assert _same(a, b), (k, name)


def test_captured_and_replayed():
    calls = _calls(70)
    eager = [call(*t) for _, call, t in calls]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [call(*t) for _, call, t in calls]
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        again = [call(*t) for _, call, t in calls]  # (eager work between the replays, in the allocator's other blocks)
        for (name, _, _), a, b, c in zip(calls, out, again, eager):
            assert _same(a, b) and _same(b, c), (k, name)


def test_rows_behind_the_last_are_left_alone():
    """Through the C ABI, into buffers longer than the outputs."""
    lib, st = tabpack.load_library(), torch.cuda.current_stream().cuda_stream
    x = torch.randn(5, 33, device="cuda")
    w = torch.ones(33, device="cuda")
    idx = torch.arange(5, dtype=torch.int32, device="cuda")

    def buf(*shape, dtype=torch.float32):
        return torch.full(shape, 77, device="cuda", dtype=dtype)

    y, s, mean, rstd = buf(9, 40), buf(9, 40), buf(9), buf(9)
    assert lib.pack_add_layer_norm(x.data_ptr(), 33, None, 0, w.data_ptr(), None, 1, 5, 33, 1e-5, s.data_ptr(), 40,
                                   y.data_ptr(), 40, mean.data_ptr(), rstd.data_ptr(), st) == 0
    z, e, q, qs = buf(9, 40), buf(9, 40), buf(9, 40, dtype=torch.uint8), buf(9)
    assert lib.pack_dropout(x.data_ptr(), 33, None, 0, 1, 5, 33, 0.5, 1, 1, None, 0, z.data_ptr(), 40, st) == 0
    assert lib.pack_embed(idx.data_ptr(), 0, x.data_ptr(), 33, 1, 5, 5, 33, 1.0, e.data_ptr(), 40, st) == 0
    assert lib.pack_quantize_blocks(x.data_ptr(), 33, 1, 5, 33, q.data_ptr(), 40, qs.data_ptr(), st) == 0
    torch.cuda.synchronize()
    for t in (y, s, z, e, q):
        assert bool((t[5:] == 77).all()) and bool((t[:, 33:] == 77).all())
    for t in (mean, rstd, qs):
        assert bool((t[5:] == 77).all())
    assert torch.equal(s[:5, :33], x) and torch.equal(e[:5, :33], x)


@pytest.mark.parametrize("cols", [33, 1024, 9000, 20_000])
def test_in_place(cols):
    """Outputs that may be inputs: the norm's sum, its gradient and dropout."""
    lib, st = tabpack.load_library(), torch.cuda.current_stream().cuda_stream
    g = torch.Generator(device="cuda").manual_seed(cols)
    x, r, dy, dv = (torch.randn(70, cols, generator=g, device="cuda") for _ in range(4))
    w = torch.randn(cols, generator=g, device="cuda")
    y, v, mean, rstd = ops.add_layer_norm(x, w, residual=r)
    for which in (0, 1):
        a, b, out = x.clone(), r.clone(), torch.empty_like(x)
        assert lib.pack_add_layer_norm(a.data_ptr(), cols, b.data_ptr(), cols, w.data_ptr(), None, 1, 70, cols, 1e-5,
                                       (a, b)[which].data_ptr(), cols, out.data_ptr(), cols, None, None, st) == 0
        assert torch.equal((a, b)[which], v) and torch.equal(out, y)
    want = ops.layer_norm_backward(dy, v, w, mean, rstd, dv=dv)
    work = torch.empty(ops._bytes("pack_layer_norm_backward_workspace_size", 70, cols), dtype=torch.uint8, device="cuda")
    for which in (0, 1):
        a, b, sums = dy.clone(), dv.clone(), torch.empty(2, cols, device="cuda")
        assert lib.pack_layer_norm_backward(a.data_ptr(), cols, v.data_ptr(), cols, w.data_ptr(), mean.data_ptr(),
                                            rstd.data_ptr(), b.data_ptr(), cols, 1, 70, cols, (a, b)[which].data_ptr(),
                                            cols, sums[0].data_ptr(), sums[1].data_ptr(), work.data_ptr(), work.numel(),
                                            st) == 0
        assert torch.equal((a, b)[which], want[0]) and torch.equal(sums[0], want[1]) and torch.equal(sums[1], want[2])
    want = ops.dropout(x, 0.3, 4, 5, residual=r)
    for which in (0, 1):
        a, b = x.clone(), r.clone()
        assert lib.pack_dropout(a.data_ptr(), cols, b.data_ptr(), cols, 1, 70, cols, 0.3, 4, 5, None, 0,
                                (a, b)[which].data_ptr(), cols, st) == 0
        assert torch.equal((a, b)[which], want)


def test_offsets_past_32_bits():
    """A table of 5 GB and a batch of 5 GB: elements past 2^31 and bytes past 2^32."""
    rows, cols = 2_600_001, 1024
    table = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    idx = torch.tensor([rows - 1, 5, rows - 2, 2_100_000], device="cuda")
    table[idx] = torch.randn(4, cols, device="cuda").bfloat16()
    assert torch.equal(ops.embed(idx, table), table[idx])
    y = ops.dropout(table, 0.0, 1, 1)
    assert torch.equal(y[idx], table[idx])
    y = ops.dropout(table, 0.25, 3, 4)
    some = torch.where(y[idx] != 0, table[idx].float() / 0.75, 0.0)
    assert float((y[idx].float() - some).abs().max()) <= 2.0 ** -8 * float(some.abs().max())
    assert 0.72 < float((y[idx] != 0).float().mean()) < 0.78
    dy = table[-4:].contiguous()
    got = ops.embed_backward(dy, idx, rows)
    assert torch.equal(got[idx], dy) and not bool(got[:5].any()) and not bool(got[6:2_000_000].any())
    w = torch.ones(cols, device="cuda")
    n, _, mean, rstd = ops.add_layer_norm(table, w)
    assert torch.equal(n[idx], ops.add_layer_norm(table[idx].contiguous(), w)[0])
    q, s = ops.quantize_blocks(table)
    qs, ss = ops.quantize_blocks(table[idx].contiguous())
    assert torch.equal(q.view(torch.uint8)[idx], qs.view(torch.uint8)) and torch.equal(s[:, idx], ss)
    qw, sw = ops.quantize_tiles(torch.randn(16, cols, device="cuda"))
    z = ops.f8_matmul(q, s, qw, sw)
    ref = ops.f8_matmul(qs, ss, qw, sw, dtype=torch.float32)
    assert float((z[idx].float() - ref).abs().max()) <= 2.0 ** -7 * float(ref.abs().max())


def _draws(rows, cols, seed, step, site):
    """The 16-bit draws of the given rows' first columns, from the oracle's generator."""
    import numpy as np
    from oracle.philox import philox4x32_10
    c, r = np.meshgrid(np.arange(-(-cols // 8), dtype=np.uint64), np.asarray(rows, dtype=np.uint64))
    w = np.stack([np.asarray(x, dtype=np.uint64) for x in philox4x32_10(
        c, r, np.uint64(site), np.uint64(step), seed & 0xFFFFFFFF, (seed >> 32) ^ (4 << 28))], -1)
    return np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(len(rows), -1)[:, :cols]


def test_more_vectors_than_32_bits_count():
    """2.2e9 vectors: the kernels' other division, and rows near 2^31."""
    rows, cols = 1_100_000_000, 9
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    at = [0, 1, 500_000_000, rows - 2, rows - 1]
    y = ops.dropout(x, 0.5, 9, 8, site=7)
    keep = torch.from_numpy(_draws(at, cols, 9, 8, 7) >= 32768).cuda()
    assert torch.equal(y[at] != 0, keep) and bool((y[at][keep] == 2).all())
    del y
    x[:3] = torch.randn(3, cols, device="cuda").bfloat16()
    idx = torch.zeros(rows, dtype=torch.int32, device="cuda")
    idx[at] = torch.tensor([2, 1, -1, 1, rows - 1], dtype=torch.int32, device="cuda")
    y = ops.embed(idx, x)
    assert torch.equal(y[at], torch.stack([x[2], x[1], torch.zeros_like(x[0]), x[1], x[-1]]))
    assert torch.equal(y[700_000_000:700_000_100], x[0].expand(100, cols))


def test_more_rows_than_a_launch_has_blocks():
    """2^20 blocks of 4 rows: each goes on to rows past the grid."""
    rows, cols = 4_300_000, 300
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(rows, cols, generator=g, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(cols, generator=g, device="cuda")
    y, _, mean, rstd = ops.add_layer_norm(x, w, w)
    half = rows // 2
    for part in (slice(0, half), slice(half, rows)):
        z, _, m, r = ops.add_layer_norm(x[part], w, w)
        assert torch.equal(y[part], z) and torch.equal(mean[part], m) and torch.equal(rstd[part], r)
