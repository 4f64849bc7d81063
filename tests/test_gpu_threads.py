"""Threads beside a call whose launch waits: the device's queue is kept full by a kernel that counts clock cycles for a while, and the interpreter
goes on meanwhile.  (A thread that the queue waits for could otherwise never get there.)"""
import threading
import time

import pytest
import torch

from paper_2608_25683_b200.workloads import Workload

from util import build_plan

pytestmark = pytest.mark.gpu
bf = torch.bfloat16


def calls(lib):
    r = lambda *s: torch.randn(*s, device="cuda").to(bf)
    x, w, g, q = r(8, 256), r(256, 256), r(256), r(8, 2, 128)
    rope = lib.Rope(128, sections=[24, 20, 20])
    pos = torch.zeros(3, 8, device="cuda", dtype=torch.int32)
    plan = build_plan(lib, Workload("t", [-1], [8], [16], 2, 1, 128, "bf16"))
    pools = [r(1, plan.oracle["pool_slots"], 128) for _ in range(2)]
    return {
        "rms_norm_fwd": lambda: lib.psrl_rms_norm_fwd(x, g, residual=x, want_codes=True),
        "rms_norm_bwd": lambda: lib.psrl_rms_norm_bwd(x, g, x),
        "linear_fwd": lambda: lib.psrl_linear_fwd(x, w, activation="silu", want_z=True),
        "linear_bwd": lambda: lib.psrl_linear_bwd(x, w, x, z=x, activation="silu"),
        "rope_axes_rows": lambda: lib.psrl_rope_axes_rows(rope, q, pos),
        "rope_axes_qkv_fwd": lambda: lib.psrl_rope_axes_qkv_fwd(plan, rope, pos, q, q[:, :1], q[:, 1:], *pools),
        "rope_axes_qkv_bwd": lambda: lib.psrl_rope_axes_qkv_bwd(plan, rope, pos, q, *pools),
    }


@pytest.mark.parametrize("name", ["rms_norm_fwd", "rms_norm_bwd", "linear_fwd", "linear_bwd", "rope_axes_rows", "rope_axes_qkv_fwd", "rope_axes_qkv_bwd"])
def test_a_launch_that_waits_holds_nobody_up(lib, name):
    call = calls(lib)[name]
    call()
    torch.cuda.synchronize()
    ticks, stop = [], threading.Event()

    def clock():
        while not stop.is_set():
            ticks.append(time.perf_counter())
            time.sleep(0.002)

    other = threading.Thread(target=clock)
    other.start()
    end = torch.cuda.Event()
    torch.cuda._sleep(1_900_000_000)            # cycles: a second or so
    start = time.perf_counter()
    for _ in range(3000):                       # more launches than the queue holds
        call()
    queued = time.perf_counter() - start
    end.record()
    stop.set()
    other.join()
    end.synchronize()
    gap = max(b - a for a, b in zip(ticks, ticks[1:]))
    assert queued > 0.5, "the queue was never full"
    assert gap < 0.25 * queued, (gap, queued)
