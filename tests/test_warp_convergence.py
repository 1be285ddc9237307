"""Instructions that a whole, converged warp has to issue together, in the sources of the kernels that have them behind code in which lanes part: between the two
stands something that brings the lanes together again.  (Without it nothing but the compiler's habit does, and what comes then is undefined: a cluster barrier may
never complete.)  A walk over the text: loop bodies are gone through twice, so that the end of one round is followed by the start of the next."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_28418_b200", "csrc")
TOGETHER = re.compile(r"__syncwarp|__syncthreads|_sync\(|mbar_wait\w*_warp\(|\bmeet\(\)")
MAYBE = re.compile(r"if \(.*&& !?\(ok = ")             # a wait that only some rounds come to
WHOLE = re.compile(r"\b(tmem_ld_\w+|tmem_st_32x16|store_transposed|umma_\w+_(?:elect|pair)|cluster_arrive)\(")
LANE = re.compile(r"\b(lane|tid|key|bad|channel|to|f)\b")                  # names whose values differ between the lanes of a warp
LOOP = re.compile(r"^\s*(for|while) \(|\} while \(")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return [re.sub(r"//.*", "", line) for line in f]


def parts(line):
    """Whether a condition in this line depends on the lane."""
    for m in re.finditer(r"\b(?:if|for|while|if constexpr) \(", line):
        depth, at = 1, m.end()
        while at < len(line) and depth:
            depth += {"(": 1, ")": -1}.get(line[at], 0)
            at += 1
        if LANE.search(line[m.end():at]):
            return True
    return False


def block_end(lines, i):
    """The line behind the statement that starts at line i: its block, or itself."""
    depth = 0
    for j in range(i, len(lines)):
        depth += lines[j].count("{") - lines[j].count("}")
        if depth <= 0 and (";" in lines[j] or "}" in lines[j]):
            return j + 1
    return len(lines)


def walk(lines, start, end, parted, found, meets):
    i = start
    while i < end:
        line = lines[i]
        loop = LOOP.search(line) and "{" in line
        if TOGETHER.search(line) and not MAYBE.search(line):
            parted = False
        hit = WHOLE.search(line)
        if hit and parted and not line.startswith("__device__") and not (hit.group(1) == "cluster_arrive" and meets):
            found.append((i + 1, line.strip()))
        if parts(line):
            parted = True
        if loop:
            stop = block_end(lines, i)
            for _ in range(2):
                parted = walk(lines, i + 1, stop - 1, parted, found, meets)
            parted = parted or parts(line)
            i = stop
        else:
            i += 1
    return parted


@pytest.mark.parametrize("name", ["linear.cu", "attn_tree.cu"])
def test_lanes_meet_before_whole_warp_instructions(name):
    lines = source(name)
    text = "".join(lines)
    meets = re.search(r"void cluster_arrive\(\) \{[^}]*__syncwarp\(\);", text) is not None     # then every call of it does
    first = next(i for i, line in enumerate(lines) if "__global__" in line)
    found = []
    walk(lines, first, len(lines), False, found, meets)
    assert not sorted(set(found))


@pytest.mark.parametrize("name,kernels", [("linear.cu", 2), ("attn_tree.cu", 1)])
def test_a_wait_given_up_is_seen_behind_the_last_barrier(name, kernels):
    """Copies may be in flight when any role of a kernel gives a wait up.  Whether one did is known behind the barrier that all roles come to, and not before it: a role that
    is done early would find nothing."""
    text = "".join(source(name))
    assert len(re.findall(r"__syncthreads\(\);\s*if \(\*abort_flag\) let_copies_land\(\);", text)) == kernels
    assert text.count("let_copies_land") == kernels and "__nanosleep" not in text
