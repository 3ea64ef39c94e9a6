"""Lanes of a wavefront exchange results through shared memory without a barrier of the workgroup in the products of sdl_orthogonalize.hip: in the compiler's own output every block of
results has the marks that keep the writes of some lanes and the reads of others in their order (CPU only, a build of this source to assembly)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2501_18512_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="needs hipcc")
def test_every_exchange_is_marked(tmp_path):
    out = str(tmp_path / "orthogonalize.s")
    source = next(s for s in build.SOURCES if s.endswith("sdl_orthogonalize.hip"))
    subprocess.run([HIPCC, *[f for f in build.FLAGS if f != "-shared"], "--cuda-device-only", "-S", source, "-o", out], check=True, capture_output=True)
    marks, name = {}, None
    with open(out) as f:
        for line in f:
            start = re.match(r"_ZN\S*product_kernelILi(\d+)ELb\dELi(\d)ELi(\d)E\S*:", line)
            if start:
                name = start[0]
                marks[name] = [*map(int, start.groups()), 0]
            elif name and "wave barrier" in line:
                marks[name][3] += 1
            elif name and "s_endpgm" in line:
                name = None
    assert len(marks) == 37
    for name, (tile, mode, how, n) in marks.items():
        blocks = max(1, tile // 2 // 64) ** 2
        # behind the writes, behind the reads, and the same for what is turned; a slice's sums go to memory without an exchange
        assert n >= (0 if how == 1 else 4 * blocks), name
