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
