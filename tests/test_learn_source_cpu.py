"""What the learning pass's kernels owe to the order of their instructions and no run shows for certain, checked on their source."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_18719_gb300", "csrc")


def source(path):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, path)).read())


def between(text, first, second):
    """The text from `first` up to the next `second`; both have to be there."""
    at = text.index(first)
    return text[at:text.index(second, at)]


def test_a_row_stored_by_its_lane_is_complete_before_other_lanes_write_it():
    part = between(source("prompt_attn.cu"), "store_tile<", "attend_row<")
    assert part.index("p.a.lse[") < part.index("__syncwarp()")  # (a ballot orders no memory)


def test_lanes_meet_before_each_load_from_tensor_memory():
    loop = between(source("prompt_items.cuh"), "store_tile(uint32_t", "return bad")
    loop = loop[loop.index("for (int b = 0"):]
    assert 0 <= loop.index("__syncwarp()") < loop.index("tmem_ld32(")
    assert "continue" not in loop


def test_kernels_that_start_early_order_earlier_stores_before_their_bulk_reads():
    norm = between(source("block_norm.cu"), "block_norm_grad_kernel(const", "request(blockIdx.x, 0)")
    assert "pdl_wait_async();" in norm and not re.search(r"pdl_wait\(\);", norm.replace("else pdl_wait();", ""))
    grad = source("prompt_grad.cu")
    start = between(grad, "    prompt_grad_kernel(const", "if (warp == 0)")
    assert start.index("pdl_wait_async();") < start.index("pdl_launch_dependents();") and "pdl_wait();" not in start
    # the kernel of d_q begins without a wait of its own
    assert re.match(r"if \(warp == 0\) \{\s*if \(!KEYS\) fence_async_global\(\);", between(grad, "if (warp == 0) {", "tma_load_2d("))
    assert "fence.proxy.async.global" in between(source("tc_tiles.cuh"), "fence_async_global()", "}")
    # the forward kernel is no programmatic dependent
    assert re.search(r"launch_at\(Start::kInOrder, kern\b", source("prompt_attn.cu")) and "kEarly" not in source("prompt_attn.cu")


def test_a_wait_is_as_long_as_the_work_it_waits_for():
    waits = between(source("tc_tiles.cuh"), "bool warp_waits(", "return true;")
    assert "now != work" in waits and waits.index("t0 = globaltimer();") < waits.index("> limit")
    assert "atomicAdd(work, 1)" in between(source("prompt_rows.cuh"), "attend_row(", "store_lane<")
    for path in ("prompt_attn.cu", "prompt_grad.cu"):  # (the count begins as the flag does)
        assert "abort_flag[0] = abort_flag[1] = 0;" in source(path)


def test_every_wait_gives_up():
    kernels = {p: source(p) for p in ("prompt_attn.cu", "prompt_grad.cu", "block_norm.cu")}
    for path, text in kernels.items():
        # all waits of the kernels are these helpers' (a try stands before one of them, as its first question), and there are some
        waits = re.findall(r"\b(warp_waits|wait_drain|wait_drain_reported)\(", text)
        assert len(waits) >= 1, path
        for m in re.finditer(r"mbar_try_wait\(", text):
            assert "wait_drain_reported(" in text[m.start():m.start() + 200], path
        for m in re.finditer(r"\bwhile\s*\(", text):  # no loop of its own around a barrier
            assert "mbar" not in text[m.start():text.index("\n", m.start())], path
    assert "warp_waits(" in kernels["prompt_attn.cu"] and "warp_waits(" in kernels["prompt_grad.cu"]
    helpers = {"tc_tiles.cuh": ["warp_waits"], "ptx.cuh": ["wait_bounded", "wait_drain", "wait_drain_reported", "wait_cluster_data"]}
    for path, names in helpers.items():
        text = source(path)
        for name in names:
            body = between(text, f" {name}(", "\n}\n")
            assert len(re.findall(r"try_wait", body)) >= 1 and re.search(r"globaltimer\(\) - t0 > limit", body), name
        # and no other function of the file tries in a loop
        loops = len(re.findall(r"(?:while|for) \([^{;]*(?:;[^{]*)?mbar_try_wait", text))
        assert loops == {"tc_tiles.cuh": 1, "ptx.cuh": 2}[path], (path, loops)


def test_dependents_start_where_they_may():
    grad, attn = source("prompt_grad.cu"), source("prompt_attn.cu")
    assert grad.count("pdl_launch_dependents()") == 1 and attn.count("pdl_launch_dependents()") == 0
    # the only one stands behind the allocation of tensor memory and the wait for the kernel of D
    order = [grad.index(x, grad.index("    prompt_grad_kernel(const")) for x in ("tmem_take(", "tc_fence_after();", "pdl_wait_async();", "pdl_launch_dependents();")]
    assert order == sorted(order)
