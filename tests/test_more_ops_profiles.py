"""Names of layer norm's, dropout's, the embeddings' and the 8-bit floating point kernels in the profile summaries (CPU)."""
import pytest

from paper_2607_05380_amd import profiles_summary as ps


@pytest.mark.parametrize("kernel,name", [
    ("_ZN7tabpack12_GLOBAL__N_111huge_kernelIhLb0ELb0ELi6EEEvNS_6MmArgsE", "mm_huge_f8_kk_gate"),
    ("_ZN7tabpack12_GLOBAL__N_112small_kernelIcLb0ELb0ELi5ELb1ELi2ELi2EEEvNS_6MmArgsE", "mm_small_f8_widened_kk_plain_128"),
    ("_ZN7tabpack12_GLOBAL__N_111thin_kernelIhLi6ELi4EEEvNS_6MmArgsE", "mm_thin_f8_gate"),
    ("_ZN7tabpack12_GLOBAL__N_111join_kernelILi5EhEEvNS_6MmArgsE", "mm_join_f8_plain"),
    ("_ZN7tabpack12_GLOBAL__N_117layer_norm_kernelIDF16bLi64ELi16EEEvNS_13LayerNormArgsE", "layer_norm"),
    ("_ZN7tabpack12_GLOBAL__N_121layer_norm_bwd_kernelIfLi64ELi16ELb1EEEvNS_16LayerNormBwdArgsE", "layer_norm_bwd"),
    ("_ZN7tabpack12_GLOBAL__N_114dropout_kernelIDF16bjEEvNS_11DropoutArgsET0_S3_", "dropout"),
    ("_ZN7tabpack12_GLOBAL__N_115run_join_kernelIfEEvNS_12EmbedBwdArgsENS0_7SumArgsE", "run_join"),
    ("_ZN7tabpack12_GLOBAL__N_112embed_kernelIfjEEvNS_9EmbedArgsET0_S3_", "embed")])
def test_short_name(kernel, name):
    assert ps.short_name(kernel) == name
