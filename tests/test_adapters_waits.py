"""How the adapters' kernels leave when a wait runs out, read off their source: no ordinary call gets there, and nothing here runs a kernel.

A wait's outcome may differ between threads (one sees the phase end, the next that another has given up), so it must be made one before
anything that several threads do together: an instruction of a whole warp, a barrier of several warps, memory of another block."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_40093_b200", "csrc")


def _block(text, at):
    """From the brace that opens at or behind `at` to the one that closes it."""
    begin = text.index("{", at)
    depth = 0
    for i in range(begin, len(text)):
        depth += (text[i] == "{") - (text[i] == "}")
        if depth == 0:
            return text[begin:i + 1]
    raise AssertionError("unbalanced")


def _kernel(name, source="ep_adapters.cu"):
    with open(os.path.join(CSRC, source)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    text = re.sub(r'"(\\.|[^"\\])*"', '""', text)                       # braces of inline assembly
    return _block(text, text.index(name + "("))


def _of_warps(body):
    """A kernel's text without what a single thread does."""
    for found in reversed(list(re.finditer(r"if \([^{;]*elect_one\(\)\)", body))):
        block = _block(body, found.end())
        at = body.index(block, found.end())
        body = body[:at] + body[at + len(block):]
    return body


@pytest.mark.parametrize("kernel", ["rank_kernel", "adapter_grad_kernel"])
def test_a_warps_lanes_take_one_answer_from_a_wait(kernel):
    text = _of_warps(_kernel(kernel))
    assert "warp_wait" in text
    for found in re.finditer(r"\bbar_wait\b[^;]*;", text):
        drains = "&none" in found.group()                                # its outcome decides nothing
        chosen = re.search(r"warp_wide \? warp_wait\(([^()]*)\) : bar_wait\(\1\)", text[:found.end()].rsplit("\n", 1)[-1])
        assert drains or chosen, found.group()


def test_the_warps_that_empty_an_accumulator_leave_together():
    text = _kernel("adapter_grad_kernel")
    loop = _block(text, text.index("for (;;)", text.index("const auto agreed")))
    vote = re.search(r"if \(!agreed\(\w+\)\) break;", loop)
    assert vote and "together()" not in loop[:vote.start()]
    assert not re.search(r"_wait\(|next\(|\bbreak;|\breturn\b", re.sub(r"if \(c0 [^;]*\) break;", "", loop[vote.end():]))
    assert text.count("together();") == loop.count("together();")


def test_a_block_of_a_cluster_leaves_when_all_are_done():
    """What is left of a block that has exited cannot be written to; one that gave up does not know whether the others still will."""
    text = _kernel("rank_kernel")
    end = text[text.rindex("__syncthreads();"):]
    assert "if (split > 1) cluster_sync();" in end and "return;" not in text[text.index("cluster_arrive();"):]


@pytest.mark.parametrize("kernel,flag,copies", [("rank_kernel", "tab.gave_up", ["land(full0, stages, s, phase, sent);", "land(unit_full0, units, u, uphase, usent);"]),
                                                ("adapter_grad_kernel", "gave_up_", ["if (boxes) bar_wait(boxes, boxes_phase, &none);"])])
def test_nothing_is_under_way_when_a_block_exits(kernel, flag, copies):
    """Copies into a block's memory and products that read it are waited for whoever gave up, which the thread that issued them may not know
    before all have met."""
    text = _kernel(kernel)
    at = text.index("if (%s) {" % flag)
    block = _block(text, at)
    assert re.search(r"__syncthreads\(\);\s*$", text[:at]) and re.search(r"__syncthreads\(\);\s*}$", block)
    assert all(c in block for c in copies) and "mma_commit" in block and at < text.index("tmem_free")
    assert "&none" not in text[:at]                                      # no thread decides that for itself
