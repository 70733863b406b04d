"""Profile summaries tell the tile sizes of one kernel apart (CPU)."""
import re
import subprocess

import pytest

from paper_2607_05380_amd import profiles_summary as ps
from paper_2607_05380_amd import tabpack


@pytest.mark.parametrize("kernel,name", [
    ("_ZN7tabpack12_GLOBAL__N_112small_kernelIaLb0ELb0ELi3ELb1ELi1ELi4EEEvNS_6MmArgsE", "mm_small_i8_kk_q8"),
    ("_ZN7tabpack12_GLOBAL__N_112small_kernelIaLb0ELb0ELi3ELb1ELi2ELi2EEEvNS_6MmArgsE", "mm_small_i8_kk_q8_128"),
    ("_ZN7tabpack12_GLOBAL__N_112small_kernelIDF16bLb0ELb1ELi2ELb0ELi2ELi2EEEvNS_6MmArgsE",
     "mm_small_bf16_kr_gate_bwd_128"),
    ("_ZN7tabpack12_GLOBAL__N_117small_pair_kernelIfLi0ELb1ELi1ELi4EEEvNS0_6MmPairE", "mm_small_pair_f32_plain"),
    ("_ZN7tabpack12_GLOBAL__N_117small_pair_kernelIfLi0ELb1ELi2ELi2EEEvNS0_6MmPairE", "mm_small_pair_f32_plain_128")])
def test_short_name_of_tiles(kernel, name):
    assert ps.short_name(kernel) == name


def test_names_of_the_library_as_built():
    """Every instance of the two kernels in the built library has the name of its tile size."""
    out = subprocess.run(["nm", tabpack.LIB_PATH], capture_output=True, text=True, check=True).stdout
    names = set(re.findall(r"(_ZN7tabpack12_GLOBAL__N_1\d+(?:small|small_pair)_kernelI\w+)", out))
    assert names
    for n in names:
        nb = re.search(r"Lb[01]ELi([12])ELi[24]EEE", n).group(1)
        assert ps.short_name(n).endswith("_128") == (nb == "2"), n
