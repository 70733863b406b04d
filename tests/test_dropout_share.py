"""Dropout's draws have 16 bits: a p whose share of kept elements would differ from 1 - p by more than one part in 256 is
refused, by the call and where a student is built (CPU: the checks run on the host, and calls without rows end there)."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import student, tabpack  # noqa: E402

TAKEN = [0.0, 1e-9, 1e-6, 0.1, 0.5, 0.9, 0.99, 1 - 2.0 ** -8, 1 - 2.0 ** -12, 1 - 2.0 ** -16, 1 - 1.002 * 2.0 ** -8]
REFUSED = [1 - 1e-6, 1 - 2.0 ** -17, 1 - 1.5 * 2.0 ** -16, 0.9999, 1 - 2.0 ** -53, 0.999]


def _call(p):
    return tabpack.load_library().pack_dropout(None, 8, None, 0, 1, 0, 8, p, 1, 2, None, 0, None, 8, None)


@pytest.mark.parametrize("p", TAKEN)
def test_taken(p):
    share = 1 - math.floor(p * 65536) / 65536
    assert 1 - p <= share <= (1 - p) * (1 + 1 / 256)
    assert _call(p) == 0
    student.Student(4, 2, blocks=1, hidden=4, device="cpu", dropout=p)


@pytest.mark.parametrize("p", REFUSED)
def test_refused(p):
    assert 1 - math.floor(p * 65536) / 65536 > (1 - p) * (1 + 1 / 256)
    assert _call(p) == -1 and "16 bits" in tabpack.load_library().pack_last_error().decode()
    with pytest.raises(tabpack.PackError, match="16 bits"):
        student.Student(4, 2, blocks=1, hidden=4, device="cpu", dropout=p)


def test_every_p_below_is_taken():
    """Up to 1 - 2^-8 whatever p is: the share is past 1 - p by at most 2^-16."""
    g = torch.Generator().manual_seed(0)
    for p in torch.rand(2000, generator=g, dtype=torch.float64).tolist():
        assert _call(p * (1 - 2.0 ** -8)) == 0
