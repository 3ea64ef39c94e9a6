"""What surrounds the kernels at the decoder's two ends and of its matrices' update, on the CPU: the extension module that converts their arguments under AddressSanitizer and
UndefinedBehaviorSanitizer, and the compiler's own report on the kernels whose copies into shared memory are waited for by count, so that a register spilled inside
a loop would wait for them."""
import os
import re
import shutil
import subprocess
import sys
import sysconfig

import pytest

from paper_2501_18512_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_arguments_under_sanitizers(tmp_path):
    def run(cmd):
        return subprocess.run(cmd, check=True, capture_output=True, text=True).stdout.strip()
    fuzz, ext, lib = os.path.join(ROOT, "tests", "host_fuzz"), str(tmp_path / "_training.so"), str(tmp_path / "standins.so")
    runtime = run(["gcc", "-print-file-name=libasan.so"])
    if not os.path.isabs(runtime):
        pytest.skip("needs libasan")
    flags = ["-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer", "-shared", "-fPIC", "-I",
             os.path.join(ROOT, "include")]
    run(["gcc", *flags, "-I", sysconfig.get_paths()["include"], os.path.join(ROOT, "paper_2501_18512_amd", "csrc", "sdl_training.c"), "-o", ext])
    run(["gcc", *flags, os.path.join(fuzz, "training_standins.c"), "-o", lib])
    # every object an allocation of its own, so that a use after it was freed is seen
    env = dict(os.environ, LD_PRELOAD=" ".join([runtime, *os.environ.get("LD_PRELOAD", "").split()]), ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0",
               PYTHONMALLOC="malloc")
    res = subprocess.run([sys.executable, os.path.join(fuzz, "training_fuzz.py"), ext, lib], capture_output=True, text=True, env=env, timeout=600)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
    _, calls, _, refused = res.stdout.split()
    assert int(calls) > 10000 and int(refused) > 5000, res.stdout


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="needs hipcc")
def test_kernels_use_no_scratch(tmp_path):
    flags = [f for f in build.FLAGS if f != "-shared"]
    running = [subprocess.Popen([HIPCC, *flags, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-c", next(s for s in build.SOURCES if s.endswith(name)), "-o",
                                 str(tmp_path / (name + ".o"))], stderr=subprocess.PIPE, text=True) for name in ("sdl_orthogonalize.hip", "sdl_cross_entropy.hip", "sdl_embedding.hip")]
    reports = [p.communicate()[1] for p in running]
    assert [p.returncode for p in running] == [0, 0, 0], reports
    scratch = dict(re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+)", "".join(reports), re.S))
    # one image or two; tiles of 256, and of 128 and 64 with sums in slices; updates of two images with results in bf16 too
    assert len([k for k in scratch if "product_kernel" in k]) == 2 * (3 + 2 * 7) + 3
    assert {k: int(x) for k, x in scratch.items() if int(x)} == {}
