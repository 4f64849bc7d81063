"""The status word of a call that takes several kernels: the first of them clears it, and what one of them records stays for the caller.  A
backward's kernels are captured, and the graph launched with its first kernel alone, or without it, on a word that holds an error."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


def nodes_of(graph):
    cu = ctypes.CDLL("libcuda.so.1")
    n = ctypes.c_size_t()
    found = []
    for f in (cu.cuGraphGetRootNodes, cu.cuGraphGetNodes):
        assert f(ctypes.c_void_p(graph), None, ctypes.byref(n)) == 0
        nodes = (ctypes.c_void_p * n.value)()
        assert f(ctypes.c_void_p(graph), nodes, ctypes.byref(n)) == 0
        found.append(list(nodes))
    return cu, found[0], found[1]


# dtype, rows, in_dim, out_dim, activation, kernels of the call
@pytest.mark.parametrize("dtype,m,k,n,activation,kernels", [("bf16", 8, 256, 8192, None, 2),          # d_x shared out over its depth, then d_weight
                                                            ("bf16", 8, 256, 8192, "silu", 4),        # dz and d_bias before those
                                                            ("bf16", 300, 264, 520, "silu", 3),       # dz, d_bias, both gradients
                                                            ("f32", 40, 264, 72, None, 2), ("f32", 40, 264, 72, "silu", 4)])
def test_an_error_stays(lib, dtype, m, k, n, activation, kernels):
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    x, w, dy, z = (torch.randn(*s, device="cuda").to(t) for s in ((m, k), (n, k), (m, n), (m, n)))
    ws = lib.Workspace(lib.psrl_linear_workspace_bytes(m, k, n, True, dtype))
    out = dict(d_x=torch.empty_like(x), d_weight=torch.empty_like(w), d_bias=torch.empty(n, device="cuda", dtype=t) if activation else None)
    call = lambda: lib.psrl_linear_bwd(x, w, dy, z=z, activation=activation, want_bias=activation is not None, workspace=ws, **out)
    call()
    assert ws.status() == 0
    word = ws._buf[ws.ptr - ws._buf.data_ptr():][:4].view(torch.int32)
    for keep_first, want in ((True, 0), (False, 10)):
        graph = torch.cuda.CUDAGraph(keep_graph=True)
        with torch.cuda.graph(graph):
            call()
        cu, roots, nodes = nodes_of(graph.raw_cuda_graph())
        assert len(roots) == 1 and len(nodes) == kernels
        for node in nodes:
            if (node in roots) != keep_first:
                assert cu.cuGraphDestroyNode(ctypes.c_void_p(node)) == 0
        graph.instantiate()
        word.fill_(10)
        graph.replay()
        torch.cuda.synchronize()
        assert int(word) == want, keep_first
    call()
    assert ws.status() == 0
