"""Products over depths that take a tile a second: the waits for it go by the depth, and nothing of it is left out.  Operands are zeros but for
small whole numbers here and there (the first and last of the depth among them), so that every sum is exact."""
import pytest
import torch

pytestmark = pytest.mark.gpu
bf = torch.bfloat16


def places(depth):
    return [0, 1, 63, 64, 12345, depth // 3, depth // 2 - 1, depth // 2, depth - 130, depth - 65, depth - 2, depth - 1]


def test_gradient_of_a_weight_over_many_rows(lib):
    m = 1 << 28
    x, dy = torch.zeros(m, 8, device="cuda", dtype=bf), torch.zeros(m, 8, device="cuda", dtype=bf)
    want = torch.zeros(8, 8)
    for i, r in enumerate(places(m)):
        x[r], dy[r] = torch.arange(8.0) - i, torch.arange(8.0) * (i % 3 - 1) + 1
        want += torch.outer(dy[r].float().cpu(), x[r].float().cpu())
    ws = lib.Workspace(256)
    d_weight = lib.psrl_linear_bwd(x, torch.zeros(8, 8, device="cuda", dtype=bf), dy, want_x=False, workspace=ws)[1]
    assert ws.status() == 0 and torch.equal(d_weight.float().cpu(), want)


def test_a_row_of_a_great_many_elements(lib):
    k = 1 << 29
    x, w = torch.zeros(1, k, device="cuda", dtype=bf), torch.zeros(2, k, device="cuda", dtype=bf)
    want = torch.zeros(2)
    for i, c in enumerate(places(k)):
        x[0, c], w[0, c], w[1, c] = i + 1, 3 - i, i % 4
        want += (i + 1) * torch.tensor([3.0 - i, i % 4])
    ws = lib.Workspace(256)
    y = lib.psrl_linear_fwd(x, w, workspace=ws)[0]
    assert ws.status() == 0 and torch.equal(y.float().cpu()[0], want.to(bf).float())
