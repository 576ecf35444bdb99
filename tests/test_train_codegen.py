"""CPU check of the training operators' generated device code: blocks of matrix instructions hold no scratch access (a spilled register in such a
loop costs more than the loop's loads), and no packed float32 arithmetic is selected anywhere.  In the loops over stages of the attention's
gradients nothing waits for memory before the last products: their operands stand in LDS, and what is on its way is the next stage."""
import os
import re
import subprocess

import pytest

from paper_2410_05589_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _blocks(text):
    """(kernel, lines) of every stretch without labels and branches."""
    kernel, lines = None, []
    for line in text.splitlines():
        m = re.match(r"^(_Z\w+):", line)
        if m or re.match(r"^\.LBB\d+_\d+:", line):
            if kernel:
                yield kernel, lines
            kernel, lines = m.group(1) if m else kernel, []
        else:
            lines.append(line)
            if kernel and "s_cbranch" in line:
                yield kernel, lines
                lines = []
    if kernel:
        yield kernel, lines


@pytest.mark.parametrize("source,kernels", [("ps_train_grad", ("gb_dq_kernel", "gb_dkv_kernel")),
                                            ("ps_loss", ("vl_score_wide_kernel", "vl_grad_wide_kernel", "vl_score_kernel", "vl_grad_kernel"))])
def test_products_do_not_spill(tmp_path, source, kernels):
    out = str(tmp_path / (source + ".s"))
    cmd = [build.hipcc_path(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fno-gpu-rdc", "-fvisibility=hidden",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-mllvm", "-instcombine-max-copied-from-constant-users=10000",
           "-I", os.path.join(ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-S", "-o", out, os.path.join(build.CSRC, source + ".hip")]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-2000:]
    text = open(out).read()
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)
    seen, loops = set(), 0
    for kernel, lines in _blocks(text):
        if sum("v_mfma" in l for l in lines) >= 8:
            seen.update(k for k in kernels if k in kernel)
            assert not any("scratch_" in l for l in lines), kernel
        if source == "ps_train_grad" and sum("v_mfma" in l for l in lines) >= 24 and any("s_barrier" in l for l in lines):
            last = max(n for n, l in enumerate(lines) if "s_barrier" in l)
            if any("v_mfma" in l for l in lines[last:]):     # (a barrier before the products: the [MASK] keys' own tiles)
                continue
            loops += 1
            seen_mfma, total = 0, sum("v_mfma" in l for l in lines)
            for l in lines:
                seen_mfma += "v_mfma" in l
                assert "vmcnt" not in l or seen_mfma >= total - 4, (kernel, seen_mfma, l)
    assert seen == set(kernels) and (loops > 0 or source != "ps_train_grad")
