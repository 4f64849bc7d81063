"""Workspaces a caller can look into: whether a wait inside the kernels gave up is seen from Python.  (No wait gives up here: the
status word is written by the test, the kernels' part of it is read by test_barrier_protocol and test_move_order.)"""
import pytest
import torch

from test_gpu_kv_move import bits, plain, pools
from test_gpu_logprob import make

pytestmark = pytest.mark.gpu
TIMEOUT = 10   # PSRL_ERR_TIMEOUT


def set_word(ws, value):
    at = ws.ptr - ws._buf.data_ptr()
    ws._buf[at:at + 4].view(torch.int32).fill_(value)
    torch.cuda.synchronize()


@pytest.mark.parametrize("slots,stream", [(500, False), (500, True), (30000, False), (30000, True)])
def test_a_move_says_how_it_ended(lib, slots, stream):
    k, v = pools(1, 8, slots + 100, 128, "bf16")
    e = [[60, 7, slots]]
    want = plain(e, k, k)
    side = torch.cuda.Stream() if stream else None
    torch.cuda.synchronize()
    ws = lib.psrl_kv_move(e, k, v, stream=side)
    assert ws.status() == lib.psrl_device_status(ws) == lib.PSRL_OK
    assert torch.equal(bits(k).cpu(), want)
    set_word(ws, TIMEOUT)
    assert ws.status() == TIMEOUT and lib.STATUS_NAMES[ws.status()] == "PSRL_ERR_TIMEOUT"
    assert lib.psrl_kv_move(e, k, v, stream=side, workspace=ws) is ws and ws.status() == lib.PSRL_OK   # the next call starts anew
    assert lib.psrl_kv_move([], k, v).status() == lib.PSRL_OK


@pytest.mark.parametrize("n,dtype", [(2, torch.bfloat16), (40, torch.bfloat16), (300, torch.bfloat16), (40, torch.float32)])
def test_log_probabilities_with_a_workspace_of_the_callers(lib, n, dtype):
    hidden, weight, targets, g = make(n, 64, 1000, n, dtype=dtype)
    name = "f32" if dtype == torch.float32 else "bf16"
    ws = lib.Workspace(max(lib.psrl_token_logprob_workspace_bytes(n, 64, 1000, n, b, name) for b in (False, True)))
    with pytest.raises(RuntimeError):
        ws.status()
    want = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    want_grads = lib.psrl_token_logprob_bwd(hidden, weight, targets, *want, g)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, side):
        set_word(ws, TIMEOUT)
        got = lib.psrl_token_logprob_fwd(hidden, weight, targets, workspace=ws, stream=stream)
        assert ws.status() == lib.PSRL_OK
        set_word(ws, TIMEOUT)
        grads = lib.psrl_token_logprob_bwd(hidden, weight, targets, *got, g, workspace=ws, stream=stream)
        assert ws.status() == lib.PSRL_OK
        assert all(torch.equal(a, b) for a, b in zip(got + grads, want + want_grads))
    small = lib.Workspace(256)
    with pytest.raises(lib.PsrlError) as e:
        lib.psrl_token_logprob_bwd(hidden, weight, targets, *want, g, workspace=small)
    assert e.value.name == "PSRL_ERR_WORKSPACE"
    with pytest.raises(ValueError):
        lib.psrl_kv_move([], *pools(1, 1, 4, 128, "bf16"), workspace=(1, 2, 3))


def test_captured_calls_with_workspaces_of_their_own(lib):
    """Two graphs, each with its workspace, replayed on streams of their own; the status of a replay is that stream's."""
    k0, v0 = pools(3, 4, 9000, 128, "bf16")
    e = [[100, 20, 8800]]
    want = plain(e, k0, k0), plain(e, v0, v0)
    hidden, weight, targets, g = make(300, 64, 1000, 4)
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    grads = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g)
    jobs = []
    for _ in range(2):
        k, v = k0.clone(), v0.clone()
        move, loss = lib.Workspace(256), lib.Workspace(lib.psrl_token_logprob_workspace_bytes(300, 64, 1000, 300, True))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lib.psrl_kv_move(e, k, v, workspace=move)
            out = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g, workspace=loss)
        jobs.append((graph, k, v, move, loss, out, torch.cuda.Stream()))
    for _ in range(3):
        for graph, k, v, *_ in jobs:
            k.copy_(k0), v.copy_(v0)
        torch.cuda.synchronize()
        for graph, k, v, move, loss, out, stream in jobs:
            with torch.cuda.stream(stream):
                graph.replay()
        for graph, k, v, move, loss, out, stream in jobs:
            assert move.status(stream) == loss.status(stream) == lib.psrl_device_status(loss, stream=stream) == lib.PSRL_OK
            assert torch.equal(bits(k).cpu(), want[0]) and torch.equal(bits(v).cpu(), want[1])
            assert all(torch.equal(a, b) for a, b in zip(out, grads))
