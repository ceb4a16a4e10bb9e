"""Properties of the kernels' source that no run can be made to show without a GPU fault."""

import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_15039_gb300", "csrc")


def test_every_drain_arrival_is_waited_for():
    """A tcgen05.commit arrives on its barrier some time later: where a kernel commits to its drain barrier it waits
    for it under the same condition, before the CTA leaves its shared memory to another."""
    found = 0
    for name in ("gemm_tc.cu", "gemm_pair.cuh", "gemm_f64.cuh"):
        with open(os.path.join(CSRC, name)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for m in re.finditer(r"pdl_trigger\(\);\s*if \((leader|!ok)\) \{(.*?)mbar_wait\(drain_bar", text, re.S):
            body = m.group(2)
            assert len(re.findall(r"mma_commit(?:_pair)?\(drain_bar\)", body)) == 1
            guarded = re.search(r"if \(!ok\)\s*$", body) is not None  # the wait alone is conditional
            assert not guarded, name
            found += 1
        assert len(re.findall(r"mma_commit(?:_pair)?\(drain_bar\)", text)) == len(
            re.findall(r"mbar_wait\(drain_bar", text)), name
    assert found == 4


def test_what_an_overlapping_kernel_writes_is_not_read_as_read_only():
    """A kernel that begins beside the one before it reads what that one writes by plain loads: the read-only path is for what
    nobody writes while the kernel lives, and its loads may be moved above the wait."""
    for name, kernels, written in (
            ("evict.cu", ("evict_move_kernel", "keep_path_kernel", "move_path"), r"(?:a\.)?(?:list|plan|path|accepted)\b"),
            ("weigh.cu", ("weigh_sum_kernel",), r"(?:w\.)?(?:parts|s)\b|scores_of"),
            ("weigh_tc.cu", ("struct Kernel", "weigh_join_rows_kernel"), r"(?:a\.)?(?:rows|parts|sums|plan|first|arrived)\b"),
            ("attention_tc.cu", ("attention_join_kernel",), r"(?:a\.)?(?:slots|divided|counters)\b")):
        with open(os.path.join(CSRC, name)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for kernel in kernels:
            assert kernel in text, kernel
        assert not re.findall(r"__ldg\(\s*(?:reinterpret_cast<[^>]*>\()?\s*(?:" + written + ")", text), name
    with open(os.path.join(CSRC, "evict.cu")) as f:
        path = re.search(r"void move_path\(.*?\n}\n.*?void __launch_bounds__\(kPathThreads\) keep_path_kernel\(.*?\n}\n", f.read(), re.S).group(0)
    # (it may begin beside any kernel that writes the lengths or the table)
    assert not re.findall(r"__ldg|paged_(?:seq|page)\(", path)
