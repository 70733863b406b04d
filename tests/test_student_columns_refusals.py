"""A student refuses categorical columns that it was not built for (CPU)."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import student, tabpack  # noqa: E402


def test_columns_of_a_student_without():
    s = student.Student(8, 3, blocks=1, hidden=4, device="cpu")
    for columns in (torch.zeros(2, 1, dtype=torch.int64), torch.zeros(2, 0, dtype=torch.int64)):
        with pytest.raises(tabpack.PackError, match="without columns"):
            s.forward(torch.zeros(2, 8), columns)
        with pytest.raises(tabpack.PackError, match="without columns"):
            s.served = []  # (laid out already)
            s.predict(torch.zeros(2, 8), columns)
