"""Rules of the kernels' sources that no run can be relied on to show."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_24840_b200", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")))
ALIGNED_BARRIER = re.compile(r'asm volatile\(\s*"(bar\.(sync|arrive)\b|barrier\.cluster\.(arrive|wait)\S*\.aligned|'
                             r'tcgen05\.(alloc|dealloc|relinquish_alloc_permit)\b)')


def _code(path):
    return re.sub(r"//[^\n]*", "", open(path).read())


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_aligned_barriers_follow_a_warp_barrier(path):
    """The aligned barriers, and the allocation of tensor memory, are undefined in a warp that is not converged: each is issued directly
    behind a __syncwarp()."""
    code = _code(path)
    for m in ALIGNED_BARRIER.finditer(code):
        assert code[:m.start()].rstrip().endswith("__syncwarp();"), "%s: %s" % (os.path.basename(path), code[m.start():m.start() + 80])


def test_the_rule_finds_the_barriers():
    assert sum(len(ALIGNED_BARRIER.findall(_code(p))) for p in SOURCES) >= 10


def _kernels(code):
    """(name, body) of every __global__ function."""
    for m in re.finditer(r"__global__", code):
        bounds = re.compile(r"__launch_bounds__\([^)]*\)").search(code, m.end(), m.end() + 80)
        head = re.compile(r"(\w+)\s*\(").search(code, bounds.end() if bounds else m.end())
        at = code.index("{", head.end())
        depth, i = 0, at
        while True:
            depth += {"{": 1, "}": -1}.get(code[i], 0)
            if depth == 0:
                break
            i += 1
        yield head.group(1), code[at + 1:i]


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_kernels_wait_for_their_asynchronous_copies_on_every_way_out(path):
    """A block's shared memory is another block's once it has left: where a kernel issues asynchronous copies, the wait for them stands at
    the outermost level behind the last of them, and nothing returns in between."""
    for name, body in _kernels(_code(path)):
        if "cp_async_16(" not in body:
            continue
        depth, waits = 0, []
        for m in re.finditer(r"[{}]|cp_async_wait_all\(\)", body):
            depth += {"{": 1, "}": -1}.get(m.group(), 0)
            if depth == 0 and m.group().startswith("cp_async"):
                waits.append(m.start())
        assert waits and waits[-1] > body.rindex("cp_async_16("), name
        assert not re.search(r"\breturn;", body[body.index("cp_async_16("):waits[-1]]), name


def test_the_rule_finds_the_kernels():
    found = {name for p in SOURCES for name, _ in _kernels(_code(p))}
    assert {"combine_splits_kernel", "token_logprob_kernel", "prune_fused_kernel", "column_sum_kernel"} <= found


@pytest.mark.parametrize("name", ["attention.cu", "attention_backward.cu"])
def test_a_scanned_stage_is_waited_for_behind_its_filling(name):
    """A wait for a phase knows only its parity, so a phase that is two ahead passes for one that is over.  A stage is filled again only once the scanner
    has handed it back, so whoever waits for the scanner waits for the filling first, whatever else it has waited for."""
    code = _code(os.path.join(CSRC, name))
    roles = re.split(r"\n    (?:\} else )?if \([^\n]*warp [=>]=? ?\d", code)
    waits = 0
    for role in roles:
        for m in re.finditer(r"mbar_wait\w*\(&\w+\.scanned\[(\w+)\]", role):
            waits += 1
            loop = role.rindex(" while (" if name == "attention.cu" else " for (int b = 0;", 0, m.start())
            assert re.search(r"mbar_wait\w*\(&\w+\.full\[%s\]" % m.group(1), role[loop:m.start()]), name
    assert waits == 1
    if name == "attention.cu":       # where S runs ahead the wait is for the keys, whose stage the scanner hands back with the values
        assert "if (!C::AHEAD && !mbar_wait_warp(&sm.full[st], parity" in code
        assert "if (C::AHEAD) mbar_arrive(&sm.empty[(pos - 1) % C::STAGES]);" in code
        assert "mbar_init(&sm.empty[i], C::AHEAD ? 3 : 1 + (i & 1));" in code


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_kernels_that_start_early_wait_before_they_touch_what_others_wrote(path):
    """Only a grid that waits itself is promised what the grids before it wrote; that the one in between has waited does not do.  So the wait is every
    thread's, at the outermost level, and comes before anything that is asked for through pdl_acquire() or added to."""
    for name, body in _kernels(_code(path)):
        if "pdl_wait()" not in body:
            continue
        depth, wait = 0, 0
        for m in re.finditer(r"[{}]|\bpdl_wait\(\)", body):
            depth += {"{": 1, "}": -1}.get(m.group(), 0)
            if m.group().startswith("pdl_wait"):
                wait = m.start()
                break
        assert depth == 0, name
        assert re.search(r"[;{}]\s*$", body[:wait]), "%s: the wait stands under a condition" % name
        assert not re.search(r"\b(pdl_acquire|atomic\w+)\(", body[:wait]), name


def test_stages_read_by_warps_are_handed_back_behind_a_proxy_fence():
    """Reads of shared memory by instructions and the copies that refill it belong to different proxies, and an arrival orders nothing between them: a warp that has
    read a stage through ldmatrix fences before it arrives, every lane, and the lanes meet before the one arrives for all."""
    found = 0
    for path in SOURCES:
        code = re.sub(r"\s+", " ", _code(path))
        if "ldmatrix_x4" not in code or "mbar_arrive" not in code:
            continue
        for m in re.finditer(r"if \(lane == 0\) mbar_arrive\w*\(&sm\.empty\[", code):
            found += 1
            assert code[:m.start()].endswith("fence_proxy_async_smem(); __syncwarp(); "), os.path.basename(path)
    assert found == 1
