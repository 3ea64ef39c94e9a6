"""The copies into shared memory that are written as assembly, of which the compiler does not know what they need (CPU only: compiled, not run).

A vector memory instruction may read a scalar register five wait states after a vector instruction wrote it at the earliest; an instruction takes one, s_nop n
takes n + 1.  The addresses come from lanes (readlane), so the wait has to stand in the same piece of assembly, wherever the compiler puts it.  And m0, which
is written there, has to be no one else's."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2501_18512_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SOURCE = """#include "sdl_attention.h"
using namespace sdl_device;
__global__ void both(const uint64_t* bases, const float* words, float* out)
{
    __shared__ __attribute__((aligned(16))) char tile[2][1024];
    const uint64_t mine = bases[threadIdx.x];
    const uint64_t base = (uint32_t)__builtin_amdgcn_readlane((int)mine, 5) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), 5) << 32;
    copy_piece<false>((const char*)base, threadIdx.x * 16, lds_offset(tile[0]));
    copy_piece<true>((const char*)base, threadIdx.x * 16, lds_offset(tile[1]));
    copy_word(words + threadIdx.x, lds_offset(tile[0]));
    own_loads_done();
    out[threadIdx.x] = *(float*)(tile[0] + threadIdx.x * 4) + *(float*)(tile[1] + threadIdx.x * 4);
}
"""


FLAGS = [f for f in build.FLAGS if f != "-shared"]


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="needs hipcc")
def test_copies_wait_for_scalar_registers_that_vector_instructions_write(tmp_path):
    src, out = tmp_path / "copies.hip", tmp_path / "copies.s"
    src.write_text(SOURCE)
    subprocess.run([HIPCC, *FLAGS, "-I", os.path.join(build.HERE, "csrc"), "--cuda-device-only", "-S", str(src), "-o", str(out)], check=True, capture_output=True)
    copies = [b for b in re.findall(r"#ASMSTART(.*?)#ASMEND", out.read_text(), re.S) if "global_load_lds" in b]
    assert len(copies) == 3
    for b in copies:
        lines = [line.split(";")[0].strip() for line in b.splitlines()]
        lines = [line for line in lines if line]
        load = next(i for i, line in enumerate(lines) if line.startswith("global_load_lds"))
        waits = sum(int(line.split()[1], 0) + 1 if line.startswith("s_nop") else 1 for line in lines[:load])
        assert waits >= (5 if re.search(r"\bs\[", lines[load]) else 2), b          # m0 itself: one behind the instruction that writes it


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="needs hipcc")
def test_nothing_but_the_copies_uses_m0(tmp_path):
    names = [s for s in build.SOURCES if "sdl_attention" in s]
    running = [subprocess.Popen([HIPCC, *FLAGS, "--cuda-device-only", "-S", s, "-o", str(tmp_path / os.path.basename(s))], stderr=subprocess.DEVNULL) for s in names]
    assert [p.wait() for p in running] == [0, 0]
    for s in names:
        text = (tmp_path / os.path.basename(s)).read_text()
        assert text.count("global_load_lds") > 100
        code = "\n".join(line.split(";")[0] for line in re.sub(r"#ASMSTART.*?#ASMEND", "", text, flags=re.S).splitlines())
        assert not re.search(r"\bm0\b", code), s
