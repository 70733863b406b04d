"""What a student network refuses to be built of (CPU)."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import student, tabpack  # noqa: E402


@pytest.mark.parametrize("kw,part", [(dict(blocks=0), "blocks"), (dict(blocks=-1), "blocks"), (dict(hidden=0), "hidden"),
                                     (dict(d_in=0), "d_in"), (dict(classes=0), "classes"),
                                     (dict(act="tanh"), "tanh"), (dict(dtype=torch.float16), "float16")])
def test_student_refuses(kw, part):
    a = dict(d_in=8, classes=3, blocks=1, hidden=4, device="cpu")
    a.update(kw)
    with pytest.raises(tabpack.PackError, match=part):
        student.Student(**a)


def test_student_is_built():
    s = student.Student(8, 3, blocks=1, hidden=4, device="cpu")
    assert [tuple(p.shape) for p in s.params] == [(8,), (8, 8), (8, 4), (8,), (3, 8)]
