"""More teacher entries than 32 bits count are refused, and not taken for what is left of their number in 32 bits."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_05380_amd import ops, tabpack  # noqa: E402

pytestmark = pytest.mark.gpu


def test_teacher_entries_past_32_bits():
    k = (1 << 32) + 3
    z = torch.randn(1, 10, device="cuda")
    idx = torch.empty(1, k, dtype=torch.int32, device="cuda")  # (17 GB each; only the first entries are given values)
    teacher = torch.empty(1, k, device="cuda")
    idx[:, :8], teacher[:, :8] = 0, 0.0
    with pytest.raises(tabpack.PackError, match="4294967299"):
        ops.distill_topk(z, idx, teacher)
