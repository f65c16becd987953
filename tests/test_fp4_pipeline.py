"""The 4-bit product's stages, read from the source on the CPU: who reads with ordinary loads what a copy has
left waits with an acquiring poll, its reads are fenced before the stage goes back to the copies, and
nothing is written to a stage but by copies."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_30846_gb300", "csrc")
SOURCE = open(os.path.join(CSRC, "ip_fp4_kernels.cuh")).read()
SHARED = open(os.path.join(CSRC, "ip_ptx.cuh")).read()


def function(name):
    """Body of a device function of this file, else of the shared helpers."""
    for text in (SOURCE, SHARED):
        m = re.search(rf"__device__ __forceinline__ \w+ {name}\(", text)
        if m:
            return text[m.start():text.index("\n}\n", m.start())]
    raise AssertionError(name)


def scale_warps():
    at = SOURCE.index("// Scales to TMEM")
    return SOURCE[at:SOURCE.index("} else {", at)]


def test_the_scale_warps_wait_before_they_read():
    body = scale_warps()
    wait, read = body.index("warp_wait_or_dead(scales(s)"), body.index("lds128(")
    assert wait < read
    polls = set(re.findall(r"\b(\w*try_wait)\(", function("wait_or_dead")))
    assert len(polls) == 1
    poll = function(polls.pop())
    assert "mbarrier.try_wait.parity" in poll and "relaxed" not in poll and '"memory"' in poll


def test_reads_of_a_stage_are_fenced_before_its_refill():
    body = scale_warps()
    last = max(body.rindex("lds128("), body.rindex("tcgen05.wait::st"))
    assert last < body.index("fence.proxy.async.shared::cta") < body.index("__syncwarp()", last) < body.index("arrive_first<PAIR>(ready(s))")


def test_nothing_but_copies_writes_a_stage():
    for call in re.findall(r"sts\d+\([^;]*;", SOURCE):
        assert "STAGES_AT" not in call, call
    # the sums of a tile's parts, which other CTAs read, lie apart from the stages too
    joined = SOURCE[SOURCE.index("const int row = part * ROWS"):SOURCE.index("no CTA ends while another one reads its sums")]
    assert "STAGES_AT" not in joined and "OUT_AT" in joined


def test_a_part_s_sums_have_places_of_their_own():
    # sum_at, as the source has it: a permutation of the 128 x 64 floats, pairs of columns side by side
    assert "4u * static_cast<uint32_t>(row * BN + (col ^ (row & 7) << 3))" in function("sum_at")
    at = [[4 * (row * 64 + (col ^ (row & 7) << 3)) for col in range(64)] for row in range(128)]
    assert sorted(a for row in at for a in row) == list(range(0, 4 * 128 * 64, 4))
    assert all(row[c + 1] == row[c] + 4 and row[c] % 8 == 0 for row in at for c in range(0, 64, 2))
    # the lanes of a store (eight rows, four pairs of columns) fall on all banks, half a warp at a time
    for c in range(0, 64, 8):
        for r in range(0, 128, 4):
            assert len({at[r + i][c + 2 * j] // 8 % 16 for i in range(4) for j in range(4)}) == 16
