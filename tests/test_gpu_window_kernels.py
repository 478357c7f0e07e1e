"""Which kernel takes a call of window_attention, over the rule's sides, and each of them against the 64-bit statement (needs a B200)."""
import os
import subprocess
import sys

import pytest
import torch
from torch.profiler import ProfilerActivity, profile

from paper_2604_18396_b200 import window_attention
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16
CASES = [
    ([1] * 3, [500, 20, 90], 8, 2, 128, 16, 100, 4, BF, "step"),
    ([4], [3000], 8, 8, 64, 16, 2048, 4, F16, "step"),
    ([1] * 64, [2100] * 64, 32, 1, 128, 16, 2048, 4, BF, "prompt"),  # single tokens of 32 heads: query tiles of 32 rows
    ([64], [3000], 8, 2, 128, 16, 2048, 4, BF, "prompt split"),
    ([120], [3000], 12, 1, 64, 32, 2900, 30, F16, "prompt split"),
    ([1000, 333], [0, 700], 16, 8, 128, 16, 300, 4, BF, "prompt whole"),
    ([1100], [40], 16, 16, 64, 64, 2000, 4, F16, "prompt whole"),
]


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(new, hist, hq, hkv, dh, page, window, sinks, dtype):
    lens = [a + b for a, b in zip(new, hist)]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    pool, table, lens_t = ref.cache(lens, page, hkv, dh, dtype, 7)
    q = (torch.randn(sum(new), hq, dh, generator=torch.Generator().manual_seed(8)) * 2).to(dtype).cuda()
    out, status = torch.full_like(q, float("nan")), i32([0])

    def call():
        window_attention(q, out, i32(starts), pool, 1, table, lens_t, window=window, sinks=sinks, max_q=max(new), status=status)
        return out, status

    return call, lambda: ref.attention(q, starts, pool, 1, table, lens, window, sinks, dh ** -0.5)


@pytest.mark.parametrize("case", CASES)
def test_results(case):
    call, statement = prepare(*case[:-1])
    out, status = call()
    want, tol = statement()
    assert status.item() == 0
    assert ((out.double() - want).abs() <= tol).all()


def test_which_kernel_runs():
    """In a process of its own: captures of single calls come back empty late in a long one."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    got = subprocess.run([sys.executable, "-m", "tests.test_gpu_window_kernels"], cwd=root, capture_output=True, text=True, timeout=300)
    lines = [x for x in got.stdout.splitlines() if x.startswith("ran: ")]
    assert got.returncode == 0 and len(lines) == len(CASES), got.stderr[-2000:]
    for case, line in zip(CASES, lines):
        assert line[5:].startswith(case[-1]), (case, line)


def tell_kernels():
    for case in CASES:
        call, _ = prepare(*case[:-1])
        call()
        torch.cuda.synchronize()
        with profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA]) as prof:
            call()
            torch.cuda.synchronize()
        names = [e.name for e in prof.events() if e.device_type == torch.autograd.DeviceType.CUDA and "window_attn" in e.name]
        assert len(names) == 1, names
        print("ran:", "step" if "window_attn_step" in names[0] else "prompt split" if "true" in names[0] or "(bool)1" in names[0] else "prompt whole", flush=True)


@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0])
@pytest.mark.parametrize("new,hist", [([1, 1], [200, 5]), ([150, 40], [200, 5])])
def test_any_softmax_scale(new, hist, scale):
    """None at all (every position the same), a negative one, one that makes single positions count."""
    lens = [a + b for a, b in zip(new, hist)]
    starts = [0, new[0], sum(new)]
    pool, table, lens_t = ref.cache(lens, 16, 2, 64, BF, 5)
    q = torch.randn(sum(new), 4, 64, generator=torch.Generator().manual_seed(8)).to(BF).cuda()
    out = torch.full_like(q, float("nan"))
    window_attention(q, out, i32(starts), pool, 1, table, lens_t, window=64, sinks=3, max_q=max(new), softmax_scale=scale)
    want, tol = ref.attention(q, starts, pool, 1, table, lens, 64, 3, scale)
    assert ((out.double() - want).abs() <= tol).all()


def test_rising_scores_over_many_tiles():
    """Keys whose scores grow along the sequence: every tile of keys moves the running maximum, by more than it may lag."""
    n, dh = 1500, 128
    pool, table, lens = ref.cache([n], 16, 1, dh, BF, 5)
    j = torch.arange(n, device="cuda")
    page = table[0].long()[j // 16]
    pool[0, page, 0, 0, j % 16] = (torch.ones(n, dh, device="cuda") * (j[:, None] / 50.0)).to(BF)
    for new in (1, 300):
        q = torch.full((new, 2, dh), 0.5, dtype=BF, device="cuda")
        q[:, 1] = -0.5
        out = torch.full_like(q, float("nan"))
        window_attention(q, out, i32([0, new]), pool, 1, table, lens, window=n, sinks=0, max_q=new)
        want, tol = ref.attention(q, [0, new], pool, 1, table, [n], n, 0, dh ** -0.5)
        assert ((out.double() - want).abs() <= tol).all()


if __name__ == "__main__":
    tell_kernels()
