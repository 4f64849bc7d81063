"""Products through the C entry points with NULL for a workspace, which the header allows where psrl_linear_workspace_bytes says 256 (fp32:
where the depth is not cut): the bits of the call that has one."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def p(t):
    return None if t is None else t.data_ptr()


# sizes whose depth is not cut: shallow ones, and one with as many tiles as there are SMs
@pytest.mark.parametrize("m,k,n", [(1, 8, 1), (5, 64, 72), (300, 120, 264), (2048, 256, 2048)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_without_workspace(lib, dtype, m, k, n):
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    code = 0 if dtype == "f32" else 1
    assert lib.psrl_linear_workspace_bytes(m, k, n, False, dtype) == 256
    x, w, pitch = torch.randn(m, k, device="cuda").to(t), torch.randn(n, k, device="cuda").to(t), -(-n // 8) * 8
    res = torch.randn(m, pitch, device="cuda").to(t)
    bias = torch.randn(n, device="cuda").to(t)
    stream = torch.cuda.current_stream().cuda_stream
    out = []
    for ws in (lib.Workspace(256), None):
        y, z = torch.zeros(m, pitch, device="cuda", dtype=t), torch.zeros(m, pitch, device="cuda", dtype=t)
        st = lib.lib().psrl_linear_fwd(code, m, k, n, p(x), k, None, p(w), k, None, p(bias), 2, None, 0, p(res), pitch, p(y), pitch, p(z), pitch,
                                       ws and ws.ptr, ws.nbytes if ws else 0, stream)
        assert st == 0
        torch.cuda.synchronize()
        out.append((y, z))
    assert out[0][0].any() and all(torch.equal(a, b) for a, b in zip(*out))
    assert torch.equal(out[0][0][:, :n], lib.psrl_linear_fwd(x, w, bias=bias, activation="silu", residual=res[:, :n])[0])


@pytest.mark.parametrize("m,k,n", [(1, 8, 8), (64, 72, 120), (120, 264, 120)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_without_workspace(lib, dtype, m, k, n):
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    code = 0 if dtype == "f32" else 1
    x, w, dy = torch.randn(m, k, device="cuda").to(t), torch.randn(n, k, device="cuda").to(t), torch.randn(m, n, device="cuda").to(t)
    stream = torch.cuda.current_stream().cuda_stream
    out = []
    for ws in (lib.Workspace(lib.psrl_linear_workspace_bytes(m, k, n, True, dtype)), None):
        dx, dw = torch.zeros(m, k, device="cuda", dtype=t), torch.zeros(n, k, device="cuda", dtype=t)
        st = lib.lib().psrl_linear_bwd(code, m, k, n, p(x), k, p(w), k, None, 0, 0, None, 0, p(dy), n, p(dx), k, p(dw), k, None, None, 0, ws and ws.ptr,
                                       ws.nbytes if ws else 0, stream)
        assert st == 0
        torch.cuda.synchronize()
        out.append((dx, dw))
    assert out[0][0].any() and out[0][1].any() and all(torch.equal(a, b) for a, b in zip(*out))
    want = lib.psrl_linear_bwd(x, w, dy)
    assert torch.equal(out[0][0], want[0]) and torch.equal(out[0][1], want[1])
