"""Waits of whole warps in the 8-bit product, read from its source: one that runs out must end for all lanes of a warp or for none, or the lanes that go on reach
aligned instructions without the others.  (Shown by reading: a wait that runs out cannot be made on a GPU without a kernel that is wrong.)"""
import os
import re

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_07244_b200", "csrc")


def test_waits_of_whole_warps_end_for_all_lanes_together():
    text = re.sub(r"//[^\n]*", "", open(os.path.join(SRC, "mrl_score.cu")).read())
    lines = [line for line in text.split("\n") if re.search(r"\bmbar_wait\w*\(", line)]
    by_one_lane = [line for line in lines if "empty_bar(stage), phase ^ 1u" in line]       # the copying lane alone
    assert len(by_one_lane) == 2 and text.count("if (lane == 0) {\n      int stage = 0;") == 2
    issue = [line for line in lines if "mbar_wait2(tempty_bar" in line]                     # nothing aligned up to the end of these loops
    for after in text.split("mbar_wait2(tempty_bar")[1:]:
        loop = after.split("} else")[0]
        assert "sync" not in loop and "tc_ld" not in loop
    others = [line for line in lines if line not in by_one_lane + issue]
    assert len(issue) == 2 and len(others) == 3
    for line in others:
        assert "mbar_wait_warp(" in line, line
    assert "ready = __all_sync(0xffffffffu, mbar_test(tfull_bar(acc), acc_phase));" in text and text.count("mbar_test(") == 1


def test_the_vote_is_of_all_lanes():
    text = open(os.path.join(SRC, "mrl_tensor.cuh")).read()
    body = text.split("bool mbar_wait_warp(")[1].split("}")[0]
    assert "return __all_sync(0xffffffffu, mbar_wait(" in body
