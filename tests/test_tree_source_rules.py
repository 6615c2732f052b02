"""Rules of tree attention's source that no run on a healthy device can show broken."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2503_01586_b200", "csrc")


def test_a_units_words_are_given_back_with_release():
    """The first block's claiming warp writes the next unit over the words of one that all readers of both blocks have given
    back.  The readers' loads are ordered before that by the release of their arrival (and the acquire of its wait); a relaxed
    arrival orders nothing.  Relaxed ones are left to the accumulator's barrier, whose reads tcgen05.wait::ld has waited for."""
    with open(os.path.join(CSRC, "tree_tc.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    body = re.search(r"auto release_unit = \[&\]\(\) \{(.*?)\};", text, flags=re.S).group(1)
    assert "q_empty" in body and "mbar_arrive_cluster(" in body and "mbar_arrive(" in body
    assert re.search(r"warp_wait_cluster\(smem_u32\(&bars->q_empty", text)
    relaxed = [m.start() for m in re.finditer(r"mbar_arrive_cluster_relaxed\(", text)]
    assert relaxed
    for at in relaxed:
        assert "acc_empty" in text[text.rfind("smem_u32(", 0, at):at]
