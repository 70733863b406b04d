"""Names of the student's kernels in the profile summaries (CPU)."""
import pytest

from paper_2607_05380_amd import profiles_summary as ps


@pytest.mark.parametrize("kernel,name", [
    ("_ZN7tabpack12_GLOBAL__N_111huge_kernelIDF16bLb0ELb0ELi1EEEvNS_6MmArgsE", "mm_huge_bf16_kk_gate"),
    ("_ZN7tabpack12_GLOBAL__N_111huge_kernelIaLb0ELb0ELi4EEEvNS_6MmArgsE", "mm_huge_i8_kk_q8_gate"),
    ("_ZN7tabpack12_GLOBAL__N_112small_kernelIfLb1ELb1ELi0ELb0ELi1ELi2EEEvNS_6MmArgsE", "mm_small_f32_rr_plain"),
    ("_ZN7tabpack12_GLOBAL__N_117small_pair_kernelIDF16bLi2ELb1ELi1ELi4EEEvNS0_6MmPairE", "mm_small_pair_bf16_gate_bwd"),
    ("_ZN7tabpack12_GLOBAL__N_111thin_kernelIaLi4ELi4EEEvNS_6MmArgsE", "mm_thin_i8_q8_gate"),
    ("_ZN7tabpack12_GLOBAL__N_111join_kernelILi0EDF16bEEvNS_6MmArgsE", "mm_join_bf16_plain"),
    ("_ZN7tabpack12_GLOBAL__N_116join_pair_kernelILi2EfEEvNS0_6MmPairE", "mm_join_pair_f32_gate_bwd"),
    ("_ZN7tabpack12_GLOBAL__N_111rows_kernelIDF16bLi64ELi16ELi1EEEvNS_7RowArgsE", "rows_bf16_norm_q8"),
    ("_ZN7tabpack12_GLOBAL__N_115norm_bwd_kernelIDF16bLi64ELi16EEEvNS_11NormBwdArgsE", "norm_bwd"),
    ("_ZN7tabpack12_GLOBAL__N_114distill_kernelIDF16bLi512ELi64ELb0EEEvNS_11DistillArgsE", "distill"),
    ("_ZN7tabpack12_GLOBAL__N_116copy_rows_kernelENS0_8CopyArgsE", "copy_rows"),
    ("_ZN7tabpack12_GLOBAL__N_119rows_to_bf16_kernelEPKfPDF16bllll", "rows_to_bf16")])
def test_short_name_of_operators(kernel, name):
    assert ps.short_name(kernel) == name
