"""The summary of kernel times and HBM bytes by case, on small hand-written CSV files (CPU)."""
import csv
import types

import pytest

from paper_2607_05380_amd import profiles_summary as ps

NORM = "_ZN7tabpack12_GLOBAL__N_117layer_norm_kernelIDF16bLi64ELi16EEEvNS_13LayerNormArgsE"
COPY = "void tabpack::(anonymous namespace)::stream_copy_kernel(...)"


def _write(path, rows):
    path.parent.mkdir(parents=True, exist_ok=True)
    with open(path, "w", newline="") as f:
        w = csv.DictWriter(f, fieldnames=list(rows[0]))
        w.writeheader()
        w.writerows(rows)


def _run(tmp_path, copies=True):
    for case, ns, kib in (("a", 10_000, 1000), ("b", 20_000, 4000)):
        _write(tmp_path / "s" / case / "run_kernel_stats.csv", [
            dict(Name=NORM, Calls=4, TotalDurationNs=4 * ns), dict(Name=COPY, Calls=2, TotalDurationNs=99),
            dict(Name="void at::native::fill(...)", Calls=9, TotalDurationNs=9)])
        for counter, factor in (("FETCH_SIZE", 0.5), ("WRITE_SIZE", 1.0)):
            rows = [dict(Dispatch_Id=i, Kernel_Name=NORM, Counter_Name=counter, Counter_Value=kib * factor) for i in (1, 2)]
            if copies:
                rows.append(dict(Dispatch_Id=3, Kernel_Name=COPY, Counter_Name=counter,
                                 Counter_Value=ps.COPY_BYTES / 1024 * factor))
            _write(tmp_path / counter / case / "run_counter_collection.csv", rows)
    out = tmp_path / "out.md"
    ps.cases(types.SimpleNamespace(stats=str(tmp_path / "s"), fetch=str(tmp_path / "FETCH_SIZE"),
                                   write=str(tmp_path / "WRITE_SIZE"), out=str(out), command="cmd"))
    return out.read_text()


def test_times_and_scaled_bytes(tmp_path):
    text = _run(tmp_path)
    # 1000 KiB each way in 10 us, 4000 in 20
    assert "| a | layer_norm | 4 | 10.0 | 1.02 | 1.02 | 0.20 |" in text
    assert "| b | layer_norm | 4 | 20.0 | 4.10 | 4.10 | 0.41 |" in text
    assert "stream_copy |" not in text


def test_a_run_without_copies(tmp_path):
    with pytest.raises(SystemExit, match="calibration"):
        _run(tmp_path, copies=False)
