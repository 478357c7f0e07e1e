"""What the kernels for requests that share prefixes have to keep: tensor memory goes back, every wait is bounded, shared memory and registers fit."""
import os
import re

from tests.test_tc_plan import ROOT

CSRC = os.path.join(ROOT, "paper_2604_18396_b200", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def kernel(name, of):
    s = source(of)
    i = re.search(rf"\b{name}\(", s).start()
    return s[i:s.index("\n}\n", i)]


def test_tensor_memory():
    b = kernel("prefix_tiles_kernel", "prefix_attn_tiles.cuh")
    assert b.count("tc_alloc(") == 1 and b.count("tc_dealloc(") == 1
    assert b.index("tc_alloc(") < b.index("__syncthreads();") < b.index("tc_dealloc(")
    assert not re.search(r"\breturn;", b)  # (nobody leaves before it goes back)


def test_waits_are_bounded():
    for name in ("prefix_attn_tiles.cuh", "prefix_attn_own.cuh", "prefix_units.cuh", "pages_batch.cu", "pages_scan.cuh"):
        s = source(name)
        assert "mbar_try_wait" not in s and "while (true)" not in s and "while (1)" not in s and "for (;;)" not in s, name
        assert len(re.findall(r"wp_wait\(", s)) == len(re.findall(r"wp_wait\(.*abortp, a\.polls\);", s)), name


def test_register_split():
    """Four warps of few registers and eight of many: together no more than the launch has."""
    b = kernel("prefix_tiles_kernel", "prefix_attn_tiles.cuh")
    dec, inc = (int(re.search(rf"setmaxnreg.{d}.sync.aligned.u32 (\d+)", b)[1]) for d in ("dec", "inc"))
    assert 4 * dec + 8 * inc <= 65536 // 384 // 8 * 8 * 12


def test_no_cluster_multicast():
    for name in ("prefix_attn_tiles.cuh", "prefix_attn_own.cuh", "prefix_attn.cu"):
        assert "multicast" not in source(name)
