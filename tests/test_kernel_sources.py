"""Rules that the kernels' sources keep (CPU)."""
import glob
import os
import re

from paper_2607_05380_amd import build


def test_wave_barriers_order_memory():
    """A wave barrier only keeps the lanes together: what one lane wrote to LDS before it and another reads after it is
    ordered by a wavefront fence, so every wave barrier stands directly behind one."""
    found = 0
    for path in sorted(glob.glob(os.path.join(build.HERE, "csrc", "*"))):
        with open(path) as fh:
            text = re.sub(r"//[^\n]*", "", fh.read())
        for m in re.finditer(r"__builtin_amdgcn_wave_barrier\(\)", text):
            found += 1
            before = text[:m.start()].rstrip().rstrip("{").rstrip()
            assert re.search(r'__builtin_amdgcn_fence\(__ATOMIC_(ACQ_REL|RELEASE), "wavefront"\);$', before), \
                f"{os.path.basename(path)}:{text[:m.start()].count(chr(10)) + 1}"
    assert found > 0
