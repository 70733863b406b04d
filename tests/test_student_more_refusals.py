"""What a student with categorical columns, layer norm and dropout refuses to be built of, and its parameters (CPU)."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import student, tabpack  # noqa: E402


@pytest.mark.parametrize("kw,part", [(dict(norm="batch"), "batch"), (dict(dropout=1.0), "dropout"),
                                     (dict(dropout=-0.1), "dropout"), (dict(dropout=float("nan")), "dropout"),
                                     (dict(columns=(3, 0)), "columns"), (dict(d_column=0), "d_column")])
def test_student_refuses(kw, part):
    with pytest.raises(tabpack.PackError, match=part):
        student.Student(**dict(dict(d_in=8, classes=3, blocks=1, hidden=4, device="cpu"), **kw))


def test_unknown_codes():
    with pytest.raises(tabpack.PackError, match="int4"):
        student.Student(8, 3, blocks=1, hidden=4, device="cpu").quantize("int4")


def test_missing_columns():
    s = student.Student(8, 3, blocks=1, hidden=4, device="cpu", columns=(5, 6))
    for columns in (None, torch.zeros(2, 1), torch.zeros(3, 2)):
        with pytest.raises(tabpack.PackError, match="columns"):
            s.forward(torch.zeros(2, 8), columns)


def test_parameters():
    s = student.Student(8, 3, blocks=1, hidden=4, device="cpu", norm="layer", columns=(5, 6), d_column=2)
    assert [tuple(p.shape) for p in s.params] == [(12,), (8, 12), (12, 4), (12,), (3, 12), (12,), (12,), (11, 2)]
    # the first ones do not depend on what was added
    a, b = (student.Student(8, 3, blocks=2, hidden=4, device="cpu", norm=n) for n in ("rms", "layer"))
    assert all(torch.equal(p, q) for p, q in zip(a.params, b.params))
