"""What the prompts' windowed attention kernel has to keep for the kernels beside it: tensor memory goes back before the CTA waits for its
cluster, no grid behind it is let go early, and every wait is bounded."""
import os
import re

from tests.test_tc_plan import ROOT

CSRC = os.path.join(ROOT, "paper_2604_18396_b200", "csrc")


def kernel():
    s = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "window_attn_prompt.cuh")).read())
    i = re.search(r"\bwindow_attn_prompt_kernel\(", s).start()
    return s, s[i:s.index("\n}\n", i)]


def test_tensor_memory():
    _, b = kernel()
    assert b.count("tc_alloc(") == 1 and b.count("tc_dealloc(") == 1
    assert b.index("tc_alloc(") < b.index("__syncthreads();") < b.index("tc_dealloc(") < b.index("cluster.sync();")
    assert "pdl_launch" not in b and "pdl_wait" not in b


def test_waits_are_bounded():
    s, b = kernel()
    assert "mbar_try_wait" not in b  # (only through the bounded wait)
    w = s[s.index("void wp_wait("):]
    w = w[:w.index("\n}\n")]
    assert "kWaitLimit" in w and "abort_flag" in w


def test_shared_memory_fits():
    s, b = kernel()
    n = re.search(r"return (\d+) \+ (\d+) \* (\d+) \* (\d+) \* (\d+);", s)
    dynamic = int(n[1]) + int(n[2]) * int(n[3]) * int(n[4]) * int(n[5])
    assert dynamic + 1024 <= 227 * 1024  # (and what the kernel declares, some 200 bytes)
