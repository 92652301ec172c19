"""How the experts' products leave when a wait runs out, read off their source, as test_adapters_waits.py does for the adapters' kernels."""
import re

from test_adapters_waits import _block, _kernel, _of_warps


def test_a_warps_lanes_take_one_answer_from_a_wait():
    text = _of_warps(_kernel("product_kernel", "ep_experts.cu"))
    assert "warp_wait" in text
    assert all("&none" in found for found in re.findall(r"\bbar_wait\b[^;]*;", text))       # those decide nothing


def test_nothing_is_under_way_when_a_block_exits():
    text = _kernel("product_kernel", "ep_experts.cu")
    at = text.index("if (gave_up_) {")
    block = _block(text, at)
    assert re.search(r"__syncthreads\(\);\s*$", text[:at]) and re.search(r"__syncthreads\(\);\s*}$", block)
    assert "in_flight > 0" in block and "mma_commit<CG>" in block and "&none" not in text[:at]
    assert at < text.rindex("cluster_sync();") < text.index("tmem_free")
