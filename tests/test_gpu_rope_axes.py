"""Rotary positions with several axes on the GPU against the fp64 oracle.

Tolerance as for one axis, relative to s (|x1| + |x2|): 2^-21 for an angle that is exact but for the rounding of its fraction to
24 bits, cos, sin, products and a sum (8 x 2^-24); the axis in the fraction's two lowest bits shifts an angle by at most
3 x 2^-64 x 2^31 turns = 2 pi 3 x 2^-33 < 2^-28, covered by counting 2^-20 for far positions (with the oracle's own
2^31 2^-53).  A bf16 result adds half a step, 2^-8 |y|."""
import numpy as np
import pytest
import torch

from oracle.layer import oracle_axes, oracle_rope_axes
from paper_2608_25683_b200.workloads import Workload

from util import build_plan, to_np

pytestmark = pytest.mark.gpu


def close(got, x, pos, axis, rope, layout, inverse=False, far=False):
    want = oracle_rope_axes(x, pos, axis, rope.freq, rope.scale, layout, inverse)
    n = len(rope.freq)
    i = np.arange(n)
    a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    size = np.zeros_like(want)
    size[..., a] = size[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * rope.scale
    tol = 2.0 ** (-20 if far else -21) * size + (2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8) if got.dtype == torch.bfloat16 else 0.0)
    err = np.abs(to_np(got) - want) - tol
    assert err.max() <= 0, float(err.max())
    assert np.array_equal(to_np(got)[..., 2 * n:], x[..., 2 * n:])


CASES = [
    # dtype, d, rotary, layout, Hq, Hkv, sections, order, rope arguments
    ("bf16", 128, 128, "half", 4, 2, [16, 24, 24], "blocks", {}),
    ("bf16", 128, 128, "interleaved", 7, 1, [24, 20, 20], "cyclic", dict(scaling="linear", factor=4.0)),
    ("bf16", 128, 64, "half", 3, 3, [10, 0, 12, 10], "blocks", dict(scaling="yarn", factor=4.0, original_positions=4096)),
    ("bf16", 128, 96, "interleaved", 4, 2, [24, 24], "cyclic", {}),
    ("bf16", 128, 10, "half", 4, 2, [1, 2, 2], "blocks", {}),          # not whole vectors: element by element
    ("f32", 64, 64, "half", 2, 2, [12, 10, 10], "cyclic", {}),
    ("f32", 64, 24, "interleaved", 5, 1, [4, 4, 4], "blocks", dict(scaling="banded", factor=8.0, original_positions=8192)),
    ("f32", 128, 128, "half", 4, 2, [64], "blocks", dict(attention_scale=0.5)),     # one axis at positions of its own
    ("f32", 64, 62, "interleaved", 4, 2, [11, 10, 10], "cyclic", {}),
]


@pytest.mark.parametrize("dtype,d,rotary,layout,Hq,Hkv,sections,order,kw", CASES)
def test_qkv_forward_and_backward(lib, dtype, d, rotary, layout, Hq, Hkv, sections, order, kw):
    w = Workload("r", [-1, 0, 0, 2, -1, 4, 4], [333, 1, 45, 17, 130, 64, 9], [64, 16], Hq, Hkv, d, dtype, seg_flags=[0, 3, 3, 3, 1, 3, 3],
                 free_extents=[(2048, 512), (0, 192), (512, 1024), (4096, 1024)])
    plan = build_plan(lib, w)
    V = plan.oracle
    T, cap, heads = V["T_q"], V["pool_slots"] + 48, Hq + 2 * Hkv
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(d + rotary + Hq)
    rope = lib.Rope(d, rotary, layout=layout, base=10000.0, sections=sections, order=order, **kw)
    axis = oracle_axes(sections, order)
    slot = np.concatenate([V["tok_slot"][V["seg_tok_off"][c]:V["seg_tok_off"][c] + V["seg_len"][c]] for c in range(V["n_seg"]) if V["seg_q_off"][c] >= 0])
    slots = torch.as_tensor(slot, device="cuda").long()
    wide = torch.randint(-50, 5000, (len(sections), T + 7), device="cuda", generator=g, dtype=torch.int32)
    positions = wide[:, 3:3 + T]                                       # a slice: axes further apart than the rows are many
    pos = positions.cpu().numpy()
    x = torch.randn(T, heads, d, device="cuda", generator=g).to(tdt)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    pools = [torch.full((Hkv, cap, d), float("nan"), device="cuda", dtype=tdt) for _ in range(2)]
    q_out = lib.psrl_rope_axes_qkv_fwd(plan, rope, positions, q, k, v, *pools)
    torch.cuda.synchronize()
    close(q_out, to_np(q), pos, axis, rope, layout)
    close(pools[0][:, slots].transpose(0, 1), to_np(k), pos, axis, rope, layout)
    assert torch.equal(pools[1][:, slots].transpose(0, 1), v)
    rest = torch.ones(cap, dtype=torch.bool, device="cuda")
    rest[slots] = False
    assert torch.isnan(pools[0][:, rest]).all() and torch.isnan(pools[1][:, rest]).all()
    q2 = q.contiguous()
    assert lib.psrl_rope_axes_qkv_fwd(plan, rope, positions, q2, k, v, *pools, q_out=q2) is q2 and torch.equal(q2, q_out)

    dq = torch.randn(T, Hq, d, device="cuda", generator=g).to(tdt)
    dpools = [torch.randn(Hkv, cap, d, device="cuda", generator=g).to(tdt) for _ in range(2)]
    out = torch.full((T, heads, d), float("nan"), device="cuda", dtype=tdt)
    got = lib.psrl_rope_axes_qkv_bwd(plan, rope, positions, dq, *dpools, dq_out=out[:, :Hq], dk_out=out[:, Hq:Hq + Hkv], dv_out=out[:, Hq + Hkv:])
    torch.cuda.synchronize()
    close(got[0], to_np(dq), pos, axis, rope, layout, inverse=True)
    close(got[1], to_np(dpools[0][:, slots].transpose(0, 1)), pos, axis, rope, layout, inverse=True)
    assert torch.equal(got[2], dpools[1][:, slots].transpose(0, 1))
    if dtype == "f32":   # differences of a linear map are the map itself
        up, down = (lib.psrl_rope_axes_qkv_fwd(plan, rope, positions, (q + h * dq).contiguous(), k, v, *pools) for h in (0.5, -0.5))
        slope = ((to_np(up) - to_np(down)) * to_np(dq)).sum()
        direct = (to_np(got[0]) * to_np(dq)).sum()
        assert abs(slope - direct) <= 2.0 ** -18 * (np.abs(to_np(dq)) * (np.abs(to_np(up)) + np.abs(to_np(down)))).sum()


@pytest.mark.parametrize("dtype,d,rotary,layout", [("bf16", 128, 128, "half"), ("bf16", 64, 32, "interleaved"), ("f32", 256, 256, "half"),
                                                   ("f32", 40, 20, "half"), ("bf16", 24, 6, "interleaved")])
@pytest.mark.parametrize("rows,heads", [(1, 1), (1, 40), (5, 3), (333, 5), (1000, 1)])
def test_rows_at_any_position(lib, dtype, d, rotary, layout, rows, heads):
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(rows * heads + d)
    n = rotary // 2
    sections = [n - 2 * (n // 3), n // 3, n // 3]
    rope, axis = lib.Rope(d, rotary, base=500000.0, layout=layout, sections=sections, order="cyclic"), oracle_axes(sections, "cyclic")
    x = torch.randn(rows, heads, d, device="cuda", generator=g).to(tdt)
    pos = torch.randint(-2 ** 31, 2 ** 31, (3, rows), device="cuda", generator=g).to(torch.int32)
    pos[1, 0], pos[2, 0] = 2 ** 31 - 1, -2 ** 31
    for inverse in (False, True):
        y = lib.psrl_rope_axes_rows(rope, x, pos, inverse=inverse)
        torch.cuda.synchronize()
        close(y, to_np(x), pos.cpu().numpy(), axis, rope, layout, inverse, far=True)
    same = x.clone()
    assert lib.psrl_rope_axes_rows(rope, same, pos, y=same, inverse=True) is same and torch.equal(same, y)
    assert lib.psrl_rope_axes_rows(rope, x[:0], pos[:, :0]).shape == (0, heads, d)


def test_text_is_the_one_axis_form(lib):
    """The same position on every axis; the entry points without axes take such a rope as it is."""
    w = Workload("t", [-1, 0, 0], [100, 33, 7], [16], 4, 2, 128, "bf16")
    plan = build_plan(lib, w)
    V = plan.oracle
    one, three = lib.Rope(128), lib.Rope(128, sections=[22, 21, 21], order="cyclic")
    x = torch.randn(V["T_q"], 8, 128, device="cuda").to(torch.bfloat16)
    pos = torch.as_tensor(np.concatenate([V["seg_anc_tokens"][c] + np.arange(V["seg_len"][c]) for c in range(3)]), dtype=torch.int32, device="cuda")
    pools = lambda: [torch.zeros(2, V["pool_slots"], 128, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    split = x[:, :4], x[:, 4:6], x[:, 6:]
    a, b, c = pools(), pools(), pools()
    want = lib.psrl_rope_qkv_fwd(plan, one, *split, *a)
    for got, p in ((lib.psrl_rope_qkv_fwd(plan, three, *split, *b), b), (lib.psrl_rope_axes_qkv_fwd(plan, three, pos.expand(3, -1).contiguous(), *split, *c), c)):
        assert torch.equal(got, want) and torch.equal(p[0], a[0]) and torch.equal(p[1], a[1])
    assert torch.equal(lib.psrl_rope_rows(three, x, pos), lib.psrl_rope_rows(one, x, pos))


def test_stream_graph_and_refusals(lib):
    plan = build_plan(lib, Workload("x", [-1, 0], [20, 5], [16], 2, 1, 128, "bf16"))
    rope = lib.Rope(128, sections=[24, 20, 20], order="cyclic")
    t = lambda *s: torch.randn(*s, device="cuda").to(torch.bfloat16)
    pos = torch.randint(0, 99, (3, 25), device="cuda", dtype=torch.int32)
    good = dict(q=t(25, 2, 128), k=t(25, 1, 128), v=t(25, 1, 128), k_pool=t(1, 48, 128), v_pool=t(1, 48, 128))
    want = lib.psrl_rope_axes_qkv_fwd(plan, rope, pos, **good)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lib.psrl_rope_axes_qkv_fwd(plan, rope, pos, **good, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out, graph = torch.empty_like(want), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.psrl_rope_axes_qkv_fwd(plan, rope, pos, **good, q_out=out)
    pos.add_(7)
    want = lib.psrl_rope_axes_qkv_fwd(plan, rope, pos, **good)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    for bad in (pos[:2], pos[:, :24], pos.long(), pos.T.contiguous().T, pos.float()):
        with pytest.raises(ValueError):
            lib.psrl_rope_axes_qkv_fwd(plan, rope, bad, **good)
        with pytest.raises(ValueError):
            lib.psrl_rope_axes_rows(rope, good["q"], bad)
    with pytest.raises(RuntimeError):
        lib.psrl_rope_axes_qkv_fwd(plan, rope, pos, **{**good, "q": good["q"].cpu()})
    with pytest.raises(ValueError):
        lib.psrl_rope_axes_qkv_fwd(plan, rope, pos.cpu(), **good)
