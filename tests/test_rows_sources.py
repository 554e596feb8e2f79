"""Rules of the memory model that no run shows reliably, looked up in the kernels' sources."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1708_04801_b200", "csrc")


def kernels():
    """(file, name, body without comments) of every __global__ function."""
    for f in sorted(os.listdir(CSRC)):
        if not f.endswith((".cu", ".cuh")):
            continue
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, f)).read())
        for m in re.finditer(r"__global__\s+void", text):
            start = text.index("{", m.end())
            depth, end = 1, start + 1
            while depth:
                depth += {"{": 1, "}": -1}.get(text[end], 0)
                end += 1
            yield f, re.search(r"(\w*kernel\w*)\s*\(", text[m.end():start]).group(1), text[start:end]


REMOTE = [(f, name, body) for f, name, body in kernels() if "mapa." in body]


def test_kernels_that_reach_other_blocks_shared_memory_are_found():
    assert {name for _, name, _ in REMOTE} >= {"clip_small_kernel", "margins_kernel"}


@pytest.mark.parametrize("name,body", [(name, body) for _, name, body in REMOTE], ids=[name for _, name, _ in REMOTE])
def test_no_block_reaches_anothers_shared_memory_before_all_of_the_cluster_run(name, body):
    # a block's shared memory exists from its start on: a barrier of the cluster lies before the first access
    before = body[:body.index("mapa.")]
    assert re.search(r"barrier\.cluster\.wait|cluster_sync_any\(\)|cluster_barrier\(\)|cluster_wait\(\)", before)


def test_gradients_that_a_kernel_scales_in_place_are_not_read_past_the_coherent_caches():
    # ld.global.nc is for memory that nothing writes while the kernel runs; clip_small_kernel reads and writes the same gradients
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "clip.cuh")).read())
    assert "chunk_squares" in text and not re.search(r"__ldg|ld\.global\.nc|ld_stream16", text)


def test_waits_of_whole_warps_end_alike_in_all_lanes():
    # a bounded wait can run out in one lane and not in the next; what follows has barriers of the warp, so the outcome is put to a vote
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "gradient.cuh")).read())
    loop = text[text.index("gradient_rows_kernel(const"):text.index("evaluate();\n\n")]
    waits = [loop[max(0, m.start() - 40):m.start()] for m in re.finditer(r"mbar_wait_bounded\(&full\[cur\]", loop)]
    assert waits and all("__all_sync(0xffffffffu, " in w for w in waits)


def test_products_are_issued_and_committed_by_the_same_thread():
    # tcgen05.commit covers the products of the thread that executes it, and which lane elect.sync chooses is not specified
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "margins.cuh")).read())
    kernel = text[text.index("margins_kernel("):]
    uses = [m.start() for m in re.finditer(r"mma_commit\(|mma_e4m3\(", kernel)]
    assert len(uses) == 4
    for at in uses:
        last = max(kernel.rfind("elect_one()", 0, at), kernel.rfind("lane == 0", 0, at))
        assert kernel.startswith("elect_one()", last)


def test_what_is_in_flight_is_waited_for_whatever_the_limit_of_the_other_waits():
    # "spin_limit" may be 1: a block that gave up after one poll still has to let its copies and products end before its memory passes on
    for f, kernel, drains in (("gradient.cuh", "gradient_rows_kernel(const", 1), ("margins.cuh", "margins_kernel(const", 2)):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, f)).read())
        text = text[text.index(kernel):]
        after = text[text.index("dead_flag) {" if f == "margins.cuh" else "if (dead >= 0 && lane == 0"):]
        waits = re.findall(r"mbar_wait_bounded\((.*?), (\S+)\);", after)
        assert len(waits) == drains and all(limit == "DRAIN_LIMIT" for _, limit in waits)
