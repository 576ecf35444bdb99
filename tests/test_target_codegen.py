"""CPU check of the generated device code of the target's operators: no registers spilled, and in the attention that stages blocks in LDS the waits for what the
memory unit writes there are the source's own, for as many requests as a step makes."""
import os
import re
import subprocess

import pytest

from paper_2410_05589_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
UNITS = ("ps_cache", "ps_tree_attn", "ps_probs")


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    folder, jobs, found = tmp_path_factory.mktemp("asm"), [], {}
    for unit in UNITS:
        out = str(folder / (unit + ".s"))
        jobs.append((unit, out, subprocess.Popen(
            [build.hipcc_path(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fno-gpu-rdc", "-fvisibility=hidden",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-mllvm", "-instcombine-max-copied-from-constant-users=10000",
             "-I", os.path.join(ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-S", "-o", out, os.path.join(build.CSRC, unit + ".hip")],
            stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for unit, out, job in jobs:
        text = job.communicate()[0]
        assert job.returncode == 0, text[-2000:]
        found[unit] = open(out).read()
    return found


@pytest.mark.parametrize("unit,kernels", [("ps_cache", 11), ("ps_tree_attn", 18), ("ps_probs", 18)])
def test_no_registers_are_spilled(listings, unit, kernels):      # (two of each are the headers')
    text = listings[unit]
    assert len(re.findall(r"\.vgpr_spill_count:", text)) == kernels
    assert not re.search(r"\.vgpr_spill_count: +[1-9]", text) and not re.search(r"\.private_segment_fixed_size: +[1-9]", text)


@pytest.mark.parametrize("dims,requests", [(128, 5), (64, 3)])
def test_staged_blocks_are_waited_for(listings, dims, requests):
    (start,) = re.findall(r"^(_ZN\w+tree_attn_kernelI6bf16_tLi%dELi4E\w+):" % dims, listings["ps_tree_attn"], re.M)
    lines = [l.strip() for l in listings["ps_tree_attn"].split("\n" + start + ":", 1)[1].split(".Lfunc_end")[0].splitlines()]
    own, inside = set(), False
    for i, l in enumerate(lines):
        inside = l.startswith(";;#ASMSTART") or (inside and not l.startswith(";;#ASMEND"))
        if inside:
            own.add(i)
    is_request = lambda l: l.startswith("buffer_load") and l.endswith("lds")
    waits = [i for i in sorted(own) if re.match(r"s_waitcnt vmcnt\(%d\) lgkmcnt\(0\)" % requests, lines[i])]
    assert len(waits) == 3                                   # one per buffer
    for i in waits:
        near = lines[i + 1:i + 6]
        assert any(l.startswith("s_barrier") for l in near) and not any(is_request(l) for l in near), near
        # the step's own requests, all between this wait and the next
        following = [j for j in range(i, len(lines)) if is_request(lines[j])][:requests]
        assert len(following) == requests
        assert not any(i < w < following[-1] for w in waits)
    # (two steps are asked for in front of the loop)
    assert sum(is_request(l) for l in lines) == 5 * requests
    assert any(re.match(r"s_waitcnt vmcnt\(0\) lgkmcnt\(0\)", lines[i]) for i in own)   # (behind the loop)
