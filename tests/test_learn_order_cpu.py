"""Orders inside the learning pass's tensor-core kernels that a run shows only by hanging or racing, checked on their source."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_18719_gb300", "csrc")


def body(path, name):
    text = open(os.path.join(CSRC, path)).read()
    at = re.search(r"__global__[^;{]*?\b" + name + r"\s*\([^;{]*\{\n", text).end()
    return text[at:text.index("\n}\n", at)]


def test_dependents_start_after_the_tensor_memory_is_held():
    # a dependent's CTA that shares the SM could otherwise allocate first and then wait for this kernel
    for path, name in (("prompt_attn.cu", "prompt_attn_kernel"), ("prompt_grad.cu", "prompt_grad_kernel")):
        b = body(path, name)
        held = b.index("tc_fence_after()", b.index("tmem_take("))
        for m in re.finditer(r"pdl_launch_dependents\(\)", b):
            assert m.start() > held, name
        assert b.rindex("tmem_give(") > b.rindex("__syncthreads()")


def test_the_kernel_that_starts_early_ends_after_the_one_before():
    b = body("prompt_grad.cu", "prompt_grad_kernel")
    assert b.rstrip().endswith("if (!KEYS) pdl_wait();")


def test_waits_are_bounded():
    for path in ("prompt_attn.cu", "prompt_grad.cu", "block_norm.cu"):
        text = open(os.path.join(CSRC, path)).read()
        # every try_wait stands in a helper that gives up, or before one
        for m in re.finditer(r"mbar_try_wait\(", text):
            assert "wait_drain_reported" in text[m.start():m.start() + 200], path
