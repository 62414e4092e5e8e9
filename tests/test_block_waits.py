"""Waits of the block GEMM (csrc/gws_tc.cuh): those that depend on another warp's success have a limit."""
import os
import re

from paper_2505_11170_b200 import _build


def _instructions(name):
    """The inline PTX of a source file."""
    text = open(os.path.join(_build.CSRC, name)).read()
    text = re.sub(r"//[^\n]*", "", text)
    return re.findall(r'asm(?: volatile)?\(\s*((?:"(?:[^"\\]|\\.)*"\s*)+)', text)


def test_no_warp_waits_for_another_at_a_named_barrier():
    # bar.sync and barrier.cta have no limit: a warp that left its loop after a failed wait would keep its partner there for good
    for name in ("gws_tc.cuh", "gws_act8.cuh"):
        ptx = _instructions(name)
        assert ptx
        assert not [p for p in ptx if re.search(r"\bbar(rier)?(\.cta)?\.(sync|arrive|red)\b", p)], name


def test_every_loop_on_an_mbarrier_reads_the_clock():
    text = open(os.path.join(_build.CSRC, "gws_tc.cuh")).read()
    loops = re.findall(r"for \(;;\) \{(.*?)\n  \}", text, re.S)
    assert loops and all("clock64()" in body for body in loops)


def test_a_kernel_lets_the_next_one_in_only_after_its_own_wait():
    # otherwise a third kernel of a stream becomes resident behind two that have not ended
    files = [name for name in sorted(os.listdir(_build.CSRC)) if any("griddepcontrol" in p for p in _instructions(name))]
    assert "gws_act8.cuh" in files and "gws_kernels.cuh" in files
    for name in files:
        order = re.findall(r"griddepcontrol\.(\w+)", " ".join(_instructions(name)))
        assert order == ["wait", "launch_dependents"] * (len(order) // 2), name
