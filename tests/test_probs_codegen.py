"""CPU check of the generated device code of the target's distributions: what a workgroup's wavefronts decide by is not written again before a barrier.

A count in LDS that every wavefront reads to choose its branch may be reset only behind a barrier that they all reach after the read: else a late one reads the reset
count, takes the other branch, and the workgroup's barriers meet out of step.  Followed here over the control flow of every kernel of the unit."""
import re

import pytest

from tests.test_target_codegen import listings  # noqa: F401


def kernels(text):
    for m in re.finditer(r"^(_ZN\S*kernel\S*):\s*; @", text, re.M):
        yield m.group(1), text[m.end():].split(".Lfunc_end", 1)[0].splitlines()


def unguarded(lines, reads, writes):
    """Pairs of a read and a write that is reachable from it without a barrier; the numbers of reads and writes."""
    at, code = {}, []
    for line in lines:
        line = line.split(";", 1)[0].strip()
        label = re.match(r"(\.LBB\w+):", line)
        if label:
            at[label.group(1)] = len(code)
        elif line and not line.startswith("."):
            code.append(line)
    assert not any(c.startswith(("s_setpc", "s_swappc", "s_call")) for c in code)

    def following(i):
        branch = re.match(r"s_(c?)branch\S* (\.LBB\w+)", code[i])
        if branch:
            return [at[branch.group(2)]] + ([i + 1] if branch.group(1) else [])
        return [] if code[i].startswith("s_endpgm") else [i + 1]

    bad = []
    for i, first in enumerate(code):
        if not reads(first):
            continue
        seen, todo = set(), following(i)
        while todo:
            j = todo.pop()
            if j in seen or j >= len(code) or code[j].startswith("s_barrier"):
                continue
            seen.add(j)
            if writes(code[j]):
                bad.append((i, first, j, code[j]))
            todo += following(j)
    return bad, sum(map(reads, code)), sum(map(writes, code))


# struct Shared: 2 KiB of table, 32 KiB of histogram or cells, 16 KiB of list, two arrays of sixteen sums, found_before, found_at, sixteen words, found, n_list
FIELDS = {"red": 51200, "red2": 51328, "found_before": 51456, "found_at": 51464, "red32": 51472, "found": 51536, "n_list": 51540}


@pytest.mark.parametrize("field", FIELDS)
def test_what_is_decided_by_is_reset_behind_a_barrier(listings, field):  # noqa: F811
    offset, reads, writes = FIELDS[field], 0, 0
    for name, lines in kernels(listings["ps_probs"]):
        bad, r, w = unguarded(lines, lambda c: re.match(r"ds_read\S* .*offset:%d\b" % offset, c) is not None,
                              lambda c: re.match(r"ds_write\S* .*offset:%d\b" % offset, c) is not None)
        assert not bad, (name, bad[:3])
        reads, writes = reads + r, writes + w
    if field in ("n_list", "found"):                         # (the layout is still the one that is looked at)
        assert reads >= 8 and writes >= 8


def test_a_read_without_a_barrier_behind_it_is_found():
    code = """
	ds_read_b32 v1, v0 offset:8
	s_cbranch_scc1 .LBB0_2
	s_barrier
	s_branch .LBB0_3
.LBB0_2:
	ds_write_b32 v0, v0 offset:8
.LBB0_3:
	s_endpgm"""
    read, write = (lambda c: c.startswith("ds_read")), (lambda c: c.startswith("ds_write"))
    assert len(unguarded(code.splitlines(), read, write)[0]) == 1
    assert not unguarded(code.replace(".LBB0_2:", ".LBB0_2:\n\ts_barrier").splitlines(), read, write)[0]
