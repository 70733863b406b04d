"""Students that are trained in several calls, and what a prediction does once a student is laid out to serve."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import student  # noqa: E402

pytestmark = pytest.mark.gpu


def _task(rows, d_in, classes):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, d_in, generator=g, device="cuda")
    return (x, *student.teacher_entries(torch.softmax(torch.randn(rows, classes, generator=g, device="cuda"), 1), 3))


def test_a_second_fit_goes_on_with_the_masks():
    x, idx, teacher = _task(300, 12, 4)
    s = student.Student(12, 4, blocks=1, hidden=32, dropout=0.5)
    steps, forward = [], s.forward
    s.forward = lambda x, columns=None, step=None: (steps.append(step), forward(x, columns, step))[1]
    s.fit(x, idx, teacher, steps=3, batch=64)
    s.fit(x, idx, teacher, steps=2, batch=64)
    assert steps == [0, 1, 2, 3, 4]
    # a call of no steps changes nothing
    s.fit(x, idx, teacher, steps=0, batch=64)
    s.fit(x, idx, teacher, steps=1, batch=64)
    assert steps[-1] == 5


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_a_prediction_rounds_no_table(dtype):
    """The table is laid out with the other weights, not in each prediction (its rows are many, a request's few)."""
    from torch.utils._python_dispatch import TorchDispatchMode

    class Copies(TorchDispatchMode):
        largest = 0

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            out = func(*args, **(kwargs or {}))
            if isinstance(out, torch.Tensor):
                Copies.largest = max(Copies.largest, out.numel())
            return out

    sizes = (5000, 3000)
    s = student.Student(12, 4, blocks=1, hidden=32, dtype=dtype, columns=sizes, d_column=16)
    x = torch.randn(7, 12, device="cuda")
    columns = torch.stack([torch.arange(7, device="cuda") * 700, 2999 - torch.arange(7, device="cuda")], 1)
    columns[2, 1] = -1
    s.quantize()
    with Copies():
        out = s.predict(x, columns)
    assert 0 < Copies.largest < sum(sizes)
    # the embeddings are those of the masters, rounded once
    at = torch.where(columns < 0, 0, columns + torch.tensor([0, sizes[0]], device="cuda"))
    rows = (s.params[-1][at] * (columns >= 0)[:, :, None]).bfloat16()
    v, _ = s._input(x, columns, torch.bfloat16, s.served_table)
    assert torch.equal(v, torch.cat([x.bfloat16(), rows.reshape(7, -1)], 1))
    # another fit's weights serve after it
    idx, teacher = student.teacher_entries(torch.softmax(torch.randn(7, 4, device="cuda"), 1), 3)
    s.fit(x, idx, teacher, steps=1, batch=16, columns=columns)
    assert not torch.equal(s.predict(x, columns), out)
    assert torch.equal(s.served_table, s.params[-1].bfloat16())
