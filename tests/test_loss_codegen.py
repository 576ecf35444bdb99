"""CPU check of the loss's generated device code: where wavefronts meet behind requests that the memory unit writes to LDS by itself, the wait for them is the
source's own (between the compiler's marks of inline assembly), not one that the compiler may or may not add to a barrier."""
import os
import re
import subprocess

import pytest

from paper_2410_05589_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "ps_loss.s")
    cmd = [build.hipcc_path(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fno-gpu-rdc", "-fvisibility=hidden",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-mllvm", "-instcombine-max-copied-from-constant-users=10000",
           "-I", os.path.join(ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-S", "-o", out, os.path.join(build.CSRC, "ps_loss.hip")]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-2000:]
    lines, found, name = open(out).read().splitlines(), {}, None
    for line in lines:
        m = re.match(r"^(_Z\w+):", line)
        if m:
            name = m.group(1)
            found[name] = []
        if name:
            found[name].append(line.strip())
    return found


# places: the pipeline's end, behind which its buffers get other contents; the targets' rows, which other wavefronts read
@pytest.mark.parametrize("kernel,places", [("vl_score_wide_kernel", 1), ("vl_grad_wide_kernelILb0", 1), ("vl_grad_wide_kernelILb1", 2)])
def test_waits_for_what_is_on_its_way_to_the_lds_are_written_out(kernels, kernel, places):
    (name,) = [n for n in kernels if kernel in n]
    lines, own, inside = kernels[name], set(), False         # own: lines of the source's own assembly
    for i, l in enumerate(lines):
        inside = l.startswith(";;#ASMSTART") or (inside and not l.startswith(";;#ASMEND"))
        if inside:
            own.add(i)
    waits = [i for i in sorted(own) if re.match(r"s_waitcnt vmcnt\(0\) lgkmcnt\(0\)", lines[i])]
    met = [i for i in waits if any(l.startswith("s_barrier") for l in lines[i:i + 6])]
    assert len(met) == places, [lines[i:i + 6] for i in waits]
