"""The student with categorical columns, layer norm and dropout: its logits and gradients against the same network in
64 bits, its predictions in 8-bit floating point, and a training step captured into a graph."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops, student  # noqa: E402

pytestmark = pytest.mark.gpu

SIZES = (3, 11, 2)


def _data(rows, d_in, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, d_in, generator=g, device="cuda")
    columns = torch.stack([torch.randint(-1, n + 1, (rows,), generator=g, device="cuda") for n in SIZES], 1)
    return x, columns  # (-1 and n are classes that a column does not have)


def _reference(s, x, columns, step):
    """Logits of the network in 64 bits on the host, differentiable in the parameters."""
    params = [p.detach().double().cpu().requires_grad_() for p in s.params]
    c, at = columns.cpu(), 0
    parts = [x.double().cpu()]
    for j, n in enumerate(SIZES):
        there = (c[:, j] >= 0) & (c[:, j] < n)
        parts.append(params[-1][at + c[:, j].clamp(0, n - 1)] * there[:, None])
        at += n
    v = torch.cat(parts, 1)

    def norm(i, v):
        if not s.layer:
            return v / torch.sqrt((v ** 2).mean(1, keepdim=True) + s.eps) * params[3 * i]
        m = v.mean(1, keepdim=True)
        return (v - m) / torch.sqrt(((v - m) ** 2).mean(1, keepdim=True) + s.eps) * params[3 * i] + params[s.head + 1 + i]

    for b in range(s.blocks):
        gate, up = (norm(b, v) @ params[3 * b + 1].t()).chunk(2, 1)
        y = (torch.nn.functional.silu(gate) * up) @ params[3 * b + 2].t()
        if step is not None and s.p:
            keep = ops.dropout(torch.ones_like(v, dtype=torch.float32, device="cuda"), s.p, s.seed, step, site=b) > 0
            y = y * keep.cpu() / (1 - s.p)
        v = v + y
    return norm(s.blocks, v) @ params[s.head].t(), params


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_gradients_fp32(norm, p):
    rows, d_in = 70, 13
    s = student.Student(d_in, 5, blocks=2, hidden=40, dtype=torch.float32, seed=1, norm=norm, dropout=p, columns=SIZES,
                        d_column=4)
    for q in s.params:
        if q.dim() == 1:
            q.add_(0.2 * torch.randn_like(q))
    s._copies()
    x, columns = _data(rows, d_in, 3)
    idx, teacher = student.teacher_entries(torch.softmax(2 * torch.randn(rows, 5, device="cuda"), 1), 3)
    weight = torch.full((rows,), 1.0 / rows, device="cuda")
    logits, kept = s.forward(x, columns, 7)
    loss, dz = ops.distill_topk(logits, idx, teacher, 2.0, weight)
    grads = s.backward(dz, kept)
    ref, params = _reference(s, x, columns, 7)
    # some ten fp32 operations deep over sums of at most 40 terms of order 1: 1e-5 of the largest value is 100 u of
    # slack on each
    assert (logits.double().cpu() - ref).abs().max() <= 1e-5 * ref.abs().max()
    q = torch.softmax(teacher.double().cpu() / 2, 1)
    lq = torch.log_softmax(ref / 2, 1).gather(1, idx.long().cpu())
    total = (4 * q * (torch.log(q) - lq)).sum() / rows
    assert abs(float(loss.double().sum()) - float(total.detach())) <= 1e-5 * abs(float(total.detach()))
    for got, want in zip(grads, torch.autograd.grad(total, params)):
        assert got.shape == want.shape
        assert (got.double().cpu() - want).norm() <= 1e-4 * want.norm()
    # without a step there is no dropout
    ref, _ = _reference(s, x, columns, None)
    assert (s.forward(x, columns)[0].double().cpu() - ref).abs().max() <= 1e-5 * ref.abs().max()


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_served_in_8_bits(norm, codes):
    s = student.Student(52, 10, blocks=2, hidden=128, seed=2, norm=norm, dropout=0.2, columns=SIZES, d_column=4)
    x, columns = _data(500, 52, 4)
    ref = torch.softmax(_reference(s, x, columns, None)[0], 1)
    out = s.quantize(codes).predict(x, columns).double().cpu()
    # 5 quantised stages deep; a code is off by half a step of 1 / 127 of its row's largest value, or of 2^-3 of its own
    part = 0.5 / 127 if codes == "int8" else 2.0 ** -4
    assert (out - ref).abs().mean() <= 5 * part and (out - ref).abs().max() <= 0.15
    assert torch.equal(s.predict(x[:1], columns[:1]), s.predict(x[:1], columns[:1]))


def test_fit_runs_and_predicts():
    x, columns = _data(600, 20, 5)
    idx, teacher = student.teacher_entries(torch.softmax(torch.randn(600, 4, device="cuda"), 1), 3)
    s = student.Student(20, 4, blocks=2, hidden=64, seed=5, norm="layer", dropout=0.1, columns=SIZES)
    before = [p.clone() for p in s.params]
    loss = s.fit(x, idx, teacher, steps=5, batch=128, columns=columns)
    assert loss.shape == (5,) and bool(loss.isfinite().all())
    assert all(not torch.equal(p, q) for p, q in zip(s.params, before))
    assert s.quantize("e4m3").predict(x, columns).shape == (600, 4)


def test_captured_steps_draw_their_own_masks():
    """A forward and backward pass in a graph whose step counter lies on the device, replayed among eager passes."""
    s = student.Student(20, 4, blocks=2, hidden=64, seed=5, norm="layer", dropout=0.4, columns=SIZES)
    x, columns = _data(128, 20, 6)
    dz = torch.randn(128, 4, device="cuda") / 128
    step = torch.zeros((), dtype=torch.int64, device="cuda")

    def both(step):
        logits, kept = s.forward(x, columns, step)
        return [logits] + s.backward(dz, kept)

    both(0)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both(step)
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(step)
        step += 1
    seen = []
    for t in range(3):
        graph.replay()
        torch.cuda.synchronize()
        want = both(t)
        assert all(torch.equal(a, b) for a, b in zip(out, want)), t
        seen.append(out[0].clone())
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])
