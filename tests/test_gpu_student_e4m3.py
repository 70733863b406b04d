"""A student served in 8-bit floating point, stage by stage: each call of a prediction gets what the ones before it gave, with
the weights of its own block, and gives what the formulas in 64 bits make of that.

Bounds: codes of a block's values are exact (test_gpu_f8.py); a weight's are off by half a step, 2^-4 of the value, or half of
2^-9 of the scale where that is more; a product in bf16 by its rounding, at most 2^-8 of each, and what the instructions cut off,
which is less in norm.  Through the network: rounding to e4m3 is off by at most 2^-4 of each element, in mean square by a third of
that square at most, so a product of two rounded operands by (2 / 3)^(1/2) 2^-4 = 0.051 of its norm; the five products of two
blocks and the head add up to 0.26 at most."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops, student  # noqa: E402
from test_gpu_f8 import _block_values  # noqa: E402
from test_gpu_student_columns import SIZES, _data, _reference  # noqa: E402

pytestmark = pytest.mark.gpu

CALLS = ("embed", "add_rms_norm", "add_layer_norm", "quantize_blocks", "f8_matmul")


def _recorded(monkeypatch, run):
    calls = []

    def recorder(name, fn):
        def call(*args, **kw):
            out = fn(*args, **kw)
            calls.append((name, args, kw, out))
            return out
        return call

    with monkeypatch.context() as m:
        for name in CALLS:
            m.setattr(ops, name, recorder(name, getattr(ops, name)))
        out = run()
    return out, calls


def _weights(q, scale, parts):
    rows = q.shape[0] // parts
    s = scale.double().view(parts, -1, scale.shape[1]).repeat_interleave(128, 1)[:, :rows].repeat_interleave(128, 2)
    s = s[:, :, :q.shape[1]].reshape(q.shape)
    return q.double() * s, s


@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_stages(norm, monkeypatch):
    # widths and hidden units that are no multiples of 128
    s = student.Student(152, 10, blocks=2, hidden=200, seed=2, norm=norm, act="gelu", columns=SIZES, d_column=4)
    for p in s.params:
        if p.dim() == 1:
            p.add_(0.2 * torch.randn_like(p))
    s._copies()
    x, columns = _data(300, 152, 4)
    s.quantize("e4m3")
    out, calls = _recorded(monkeypatch, lambda: s.predict(x, columns))
    # after the lookup: a block is norm, codes, gated product, codes, product; then norm, codes, head
    stage = ["add_layer_norm" if norm == "layer" else "add_rms_norm", "quantize_blocks", "f8_matmul"]
    assert [c[0] for c in calls] == ["embed"] + 2 * (stage + stage[1:]) + stage
    branch, stream = None, s._input(x, columns, torch.bfloat16, s.served_table)[0]
    it = iter(calls[1:])
    for b in range(3):
        _, args, kw, (n, v, *_) = next(it)
        new, w = args[0], args[1]
        residual = args[-2]
        if branch is None:
            assert residual is None and torch.equal(new, stream)
            total = new.double()
        else:
            assert new is branch and residual is stream
            total = new.double() + residual.double()
        assert torch.equal(w, s.params[3 * b])
        if norm == "layer":
            total_n = (total - total.mean(1, keepdim=True))
            total_n = total_n * (total_n.square().mean(1, keepdim=True) + s.eps).rsqrt() * w.double() + args[2].double()
            assert torch.equal(args[2], s.params[s.head + 1 + b])
        else:
            total_n = total * (total.square().mean(1, keepdim=True) + s.eps).rsqrt() * w.double()
        assert float((n.double() - total_n).norm()) <= 2.0 ** -8 * float(total_n.norm())
        stream, h = v, n
        for k in (1, 2) if b < 2 else (1,):
            _, (given,), _, (q, scale) = next(it)
            assert given is h
            codes, blocks = _block_values(given, 1)
            assert torch.equal(q.double(), codes) and torch.equal(scale, blocks.t())
            _, (mq, ms, w, ws), kw, h = next(it)
            assert mq is q and ms is scale
            gated = b < 2 and k == 1
            assert kw.get("gate") == ("gelu" if gated else None)
            W, step = _weights(w, ws, 2 if gated else 1)
            master = s.params[3 * b + k].double()
            assert bool(((W - master).abs() <= torch.maximum(master.abs() * 2.0 ** -4, step * 2.0 ** -10) * (1 + 1e-5)).all())
            ref = (q.double() * scale.double().t().repeat_interleave(128, 1)[:, :q.shape[1]]) @ W.t()
            if gated:
                gate, up = ref.chunk(2, 1)
                ref = torch.nn.functional.gelu(gate) * up
            assert h.dtype == (torch.float32 if b == 2 else torch.bfloat16)
            assert float((h.double() - ref).norm()) <= (1e-5 if b == 2 else 2.0 ** -8) * float(ref.norm())
        branch = h
    assert torch.equal(out, torch.softmax(h, 1))


def _centred(p):
    z = p.double().cpu().clamp(min=1e-300).log()
    return z - z.mean(1, keepdim=True)


@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_whole_network(norm):
    s = student.Student(52, 10, blocks=2, hidden=128, seed=2, norm=norm, columns=SIZES, d_column=4)
    x, columns = _data(500, 52, 4)
    ref = _reference(s, x, columns, None)[0].detach()
    ref = ref - ref.mean(1, keepdim=True)
    got = _centred(s.quantize("e4m3").predict(x, columns))
    assert float((got - ref).norm()) <= 0.26 * float(ref.norm())
    # one row alone, by the kernels of few rows: every bf16 value at most a step of 2^-8 apart, so that one code in 16 may be its
    # neighbour, 2^-3 away: 2^-5 of an operand's norm, five times
    for i in range(0, 500, 50):
        one = _centred(s.predict(x[i:i + 1], columns[i:i + 1]))
        assert float((one - got[i:i + 1]).norm()) <= 5 * 2.0 ** -5 * float(got[i:i + 1].norm())
