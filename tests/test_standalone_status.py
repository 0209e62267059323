"""Waits that give up in calls without a handle are reported."""
import os
import subprocess
import sys

import pytest

gpu = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_limits_outside_their_range_are_refused():
    from paper_2405_10951_b200 import binding as Bd
    for limit in (0, 999, 100_000_001):
        with pytest.raises(Bd.BsrError) as e:
            Bd._check(Bd.lib().bsr_selftest_wait_expiry(None, limit, None))
        assert e.value.status == -1 and "limit_ns" in str(e.value)


@gpu
def test_an_expired_wait_is_reported_once_and_calls_go_on():
    import torch
    from paper_2405_10951_b200 import binding as Bd
    x, w = torch.randn((40, 256), device="cuda"), torch.randn((72, 256), device="cuda")
    q = Bd.bsr_quantize_e4m3_rows128(x) + Bd.bsr_quantize_e4m3_blocks128(w)
    want = Bd.bsr_linear_forward_e4m3_block128(*q)
    Bd.bsr_standalone_status()
    side = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(stream):
            Bd.bsr_selftest_wait_expiry(1_000_000)
            with pytest.raises(Bd.BsrError) as e:
                Bd.bsr_standalone_status()
            assert e.value.status == -5 and "wait expired" in str(e.value)
            Bd.bsr_standalone_status()
            assert torch.equal(Bd.bsr_linear_forward_e4m3_block128(*q), want)
            Bd.bsr_standalone_status()


FIRST_UNDER_CAPTURE = """
import torch
from paper_2405_10951_b200 import binding as Bd
x, w = torch.randn((40, 256), device="cuda"), torch.randn((72, 256), device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    y = Bd.bsr_linear_forward_e4m3_block128(*Bd.bsr_quantize_e4m3_rows128(x), *Bd.bsr_quantize_e4m3_blocks128(w))
    Bd.bsr_selftest_wait_expiry(100_000)
    try:
        Bd.bsr_standalone_status()
    except Bd.BsrError as e:
        assert e.status == -1 and "captured" in str(e), e
    else:
        raise AssertionError("read under capture")
Bd.bsr_standalone_status()
graph.replay()
want = Bd.bsr_linear_forward_e4m3_block128(*Bd.bsr_quantize_e4m3_rows128(x), *Bd.bsr_quantize_e4m3_blocks128(w))
try:
    Bd.bsr_standalone_status()
except Bd.BsrError as e:
    assert e.status == -5, e
else:
    raise AssertionError("not reported")
assert torch.equal(y, want)
print("fine")
"""


@gpu
def test_the_first_call_of_a_process_may_be_captured():
    run = subprocess.run([sys.executable, "-c", FIRST_UNDER_CAPTURE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "fine" in run.stdout, run.stdout + run.stderr
