"""The bounded waits of attention over sequences, read from the kernel sources (a wait that gives up is not provoked inside
a kernel on a GPU; the give-up itself is what mnmt_wait_timeout_selftest shows).

What follows a wait of a whole warp is executed by whole warps only (tcgen05.ld, st and wait, votes, __syncwarp), so its
lanes must agree whether the wait gave up; a wait of one lane, under a branch on the lane, must not vote."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2306_04235_gb300", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def body(text, head):
    """The brace-matched body after the first occurrence of `head`."""
    i = text.index("{", text.index(head))
    depth = 0
    for j in range(i, len(text)):
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        if depth == 0:
            return text[i + 1:j]
    raise AssertionError(head)


def test_a_warp_gives_up_as_one():
    text = source("seq_tile.cuh")
    waits = body(text, "struct SqWaits")
    warp, one = body(waits, "operator()"), body(waits, "bool one(")
    assert "vote.sync.all.pred" in body(text, "bool sq_try_all(")
    assert re.sub(r"\s+", " ", warp).strip() == "return sq_try_all(bar, parity) || sq_wait_warp(failed, status, bar, parity);"
    assert not re.search(r"sync|_all\(|vote", one)
    slow = body(text, "sq_wait_warp(")
    # both ways out are votes of all lanes
    assert re.search(r"if \(sq_try_all\(bar, parity\)\) return true;", slow)
    assert re.search(r"__any_sync\(0xFFFFFFFFu, \*failed \|\| [^)]*\) - t0 > MNMT_WAIT_NS\)", slow)
    assert slow.count("return") == 2, "a way out that is no vote"


@pytest.mark.parametrize("name,kernel,warp", [("seq_attn.cu", "seq_attn_forward_kernel(", "if (warp == 4)"), ("seq_attn_backward.cu", "seq_attn_dq_kernel(", "if (warp == 8)")])
def test_producers_of_one_lane(name, kernel, warp):
    text = source(name)
    part = body(text[text.index(kernel):], warp)
    assert "lane == 0" in part and "wait.one(" in part and not re.search(r"\bwait\(", part)


@pytest.mark.parametrize("name,kernel,warp", [("seq_attn.cu", "seq_attn_forward_kernel(", "} else if (warp == 5)"), ("seq_attn_backward.cu", "seq_attn_dq_kernel(", "} else if (warp == 9)"),
                                              ("seq_attn_backward.cu", "seq_attn_dkv_kernel(", "} else if (warp == 9)"), ("seq_attn_backward.cu", "seq_attn_dkv_kernel(", "if (warp == 8)")])
def test_whole_warps(name, kernel, warp):
    """The MMA warps, and the producer that all lanes of a warp are: no wait of one lane, no branch on `failed` by the lane."""
    text = source(name)
    part = body(text[text.index(kernel):], warp)
    assert re.search(r"\bwait\(", part) and "wait.one(" not in part and not re.search(r"if \(failed\)", part)
