"""Rotary positions on the GPU against the fp64 oracle, with the plan built by the oracle.

Tolerance of one rotated element y = s (x1 c - x2 t), relative to s (|x1| + |x2|): cos and sin of an angle that is exact
but for the rounding of its fraction to 24 bits (pi 2^-25), their own error (2 steps of 2^-24 each), their product with s
(2^-24), two products and a sum (2 x 2^-24): below 8 x 2^-24 = 2^-21 in all.  A bf16 result adds half a step, 2^-8 |y|."""
import numpy as np
import pytest
import torch

from oracle.rope import oracle_rope, oracle_rope_frequencies
from paper_2608_25683_b200.workloads import Workload, make_workload

from util import build_plan, to_np

pytestmark = pytest.mark.gpu


def close(got, x, pos, rope, layout, inverse=False):
    want = oracle_rope(x, pos, rope.freq, rope.scale, layout, inverse)
    n = len(rope.freq)
    i = np.arange(n)
    a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    size = np.zeros_like(want)
    size[..., a] = size[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * rope.scale
    tol = 2.0 ** -21 * size + (2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8) if got.dtype == torch.bfloat16 else 0.0)
    err = np.abs(to_np(got) - want) - tol
    assert err.max() <= 0, float(err.max())
    assert np.array_equal(to_np(got)[..., 2 * n:], x[..., 2 * n:])   # what is not rotated passes through exactly


def rows_of(V):
    pos, slot = np.zeros(V["T_q"], dtype=np.int64), np.zeros(V["T_q"], dtype=np.int64)
    for c in range(V["n_seg"]):
        r, t, n = int(V["seg_q_off"][c]), int(V["seg_tok_off"][c]), int(V["seg_len"][c])
        if r >= 0:
            pos[r:r + n] = V["seg_anc_tokens"][c] + np.arange(n)
            slot[r:r + n] = V["tok_slot"][t:t + n]
    return pos, slot


CASES = [
    # dtype, d, rotary, layout, Hq, Hkv, rope arguments
    ("bf16", 128, 128, "half", 4, 2, {}),
    ("bf16", 128, 128, "interleaved", 7, 1, dict(scaling="linear", factor=4.0)),
    ("bf16", 128, 48, "half", 3, 3, dict(scaling="ntk", factor=8.0)),
    ("bf16", 128, 64, "interleaved", 4, 2, dict(scaling="yarn", factor=4.0, original_positions=4096)),
    ("bf16", 128, 10, "half", 4, 2, {}),              # not whole vectors: element by element
    ("bf16", 128, 2, "interleaved", 4, 2, {}),
    ("f32", 64, 64, "half", 2, 2, {}),
    ("f32", 64, 24, "interleaved", 5, 1, dict(scaling="banded", factor=8.0, original_positions=8192)),
    ("f32", 128, 128, "half", 4, 2, dict(attention_scale=0.5)),
    ("f32", 128, 12, "half", 4, 2, {}),
    ("f32", 64, 62, "interleaved", 4, 2, {}),
]


@pytest.mark.parametrize("dtype,d,rotary,layout,Hq,Hkv,kw", CASES)
@pytest.mark.parametrize("cached", [False, True])
def test_qkv_forward_and_backward(lib, dtype, d, rotary, layout, Hq, Hkv, kw, cached):
    """One projection output [T_q, (Hq + 2 Hkv) d], read and written as slices; fragmented pool, short segments, and with
    `cached` a prefix whose rows are not there and whose slots keep what they hold."""
    flags = [0, 3, 3, 3, 1, 3, 3] if cached else [1, 3, 3, 3, 1, 3, 3]
    w = Workload("r", [-1, 0, 0, 2, -1, 4, 4], [333, 1, 45, 17, 130, 64, 9], [64, 16], Hq, Hkv, d, dtype, seg_flags=flags,
                 free_extents=[(2048, 512), (0, 192), (512, 1024), (4096, 1024)])
    plan = build_plan(lib, w)
    V = plan.oracle
    T, cap, heads = V["T_q"], V["pool_slots"] + 48, Hq + 2 * Hkv
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(d + rotary + Hq)
    rope = lib.Rope(d, rotary, layout=layout, base=10000.0, **kw)
    pos, slot = rows_of(V)
    slots = torch.as_tensor(slot, device="cuda")
    x = torch.randn(T, heads, d, device="cuda", generator=g).to(tdt)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    pools = [torch.full((Hkv, cap, d), float("nan"), device="cuda", dtype=tdt) for _ in range(2)]
    q_out = lib.psrl_rope_qkv_fwd(plan, rope, q, k, v, *pools)
    torch.cuda.synchronize()
    close(q_out, to_np(q), pos, rope, layout)
    close(pools[0][:, slots].transpose(0, 1), to_np(k), pos, rope, layout)
    assert torch.equal(pools[1][:, slots].transpose(0, 1), v)
    rest = torch.ones(cap, dtype=torch.bool, device="cuda")
    rest[slots] = False
    assert torch.isnan(pools[0][:, rest]).all() and torch.isnan(pools[1][:, rest]).all()
    # in place on a contiguous Q, bit for bit the same
    q2 = q.contiguous()
    lib.psrl_rope_qkv_fwd(plan, rope, q2, k, v, *pools, q_out=q2)
    assert torch.equal(q2, q_out)

    dq = torch.randn(T, Hq, d, device="cuda", generator=g).to(tdt)
    dpools = [torch.randn(Hkv, cap, d, device="cuda", generator=g).to(tdt) for _ in range(2)]
    for p in dpools:
        p[:, rest] = float("nan")
    out = torch.full((T, heads, d), float("nan"), device="cuda", dtype=tdt)
    got = lib.psrl_rope_qkv_bwd(plan, rope, dq, *dpools, dq_out=out[:, :Hq], dk_out=out[:, Hq:Hq + Hkv], dv_out=out[:, Hq + Hkv:])
    torch.cuda.synchronize()
    assert not torch.isnan(out).any()
    close(got[0], to_np(dq), pos, rope, layout, inverse=True)
    close(got[1], to_np(dpools[0][:, slots].transpose(0, 1)), pos, rope, layout, inverse=True)
    assert torch.equal(got[2], dpools[1][:, slots].transpose(0, 1))
    for a, b in zip(got, lib.psrl_rope_qkv_bwd(plan, rope, dq, *dpools)):
        assert torch.equal(a, b)
    # the backward is the transpose of the forward: <dq, R q> = <R^T dq, q>; differences of a linear map are the map itself
    if dtype == "f32":
        a, b = (to_np(dq) * to_np(q_out)).sum(), (to_np(got[0]) * to_np(q)).sum()
        assert abs(a - b) <= 2.0 ** -20 * (np.abs(to_np(dq)) * np.abs(to_np(q_out))).sum() * 2
        h = 0.5
        up = lib.psrl_rope_qkv_fwd(plan, rope, (q + h * dq).contiguous(), k, v, *pools)
        down = lib.psrl_rope_qkv_fwd(plan, rope, (q - h * dq).contiguous(), k, v, *pools)
        slope = ((to_np(up) - to_np(down)) / (2 * h) * to_np(dq)).sum()
        direct = (to_np(got[0]) * to_np(dq)).sum()
        assert abs(slope - direct) <= 2.0 ** -18 * (np.abs(to_np(dq)) * (np.abs(to_np(up)) + np.abs(to_np(down)))).sum()


@pytest.mark.parametrize("dtype,d,rotary,layout", [("bf16", 128, 128, "half"), ("bf16", 64, 32, "interleaved"),
                                                   ("f32", 256, 256, "half"), ("f32", 40, 20, "half"), ("bf16", 8, 8, "half"),
                                                   ("bf16", 24, 6, "interleaved")])
@pytest.mark.parametrize("rows,heads", [(1, 1), (1, 40), (5, 3), (333, 5), (1000, 1)])
def test_rows_at_any_position(lib, dtype, d, rotary, layout, rows, heads):
    """Far and negative positions lose nothing: the oracle multiplies in fp64, whose own error at 2^31 is 2^31 2^-53."""
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(rows * heads + d)
    rope = lib.Rope(d, rotary, base=500000.0, layout=layout)
    wide = torch.randn(rows, heads + 2, d, device="cuda", generator=g).to(tdt)
    x = wide[:, 1:1 + heads]
    pos = torch.randint(-2 ** 31, 2 ** 31, (rows,), device="cuda", generator=g).to(torch.int32)
    pos[0] = 2 ** 31 - 1
    if (d * (heads + 2) * x.element_size()) % 16 or (d * x.element_size()) % 16:
        x = x.contiguous()
    for inverse in (False, True):
        y = lib.psrl_rope_rows(rope, x, pos, inverse=inverse)
        torch.cuda.synchronize()
        want = oracle_rope(to_np(x), pos.cpu().numpy(), rope.freq, rope.scale, layout, inverse)
        size = np.abs(to_np(x)).max()
        tol = 2.0 ** -20 * size + 2.0 ** -21 * size + (2.0 ** -8 * np.abs(want) * 1.01 if dtype == "bf16" else 0)
        assert (np.abs(to_np(y) - want) <= tol).all()
    same = x.clone()
    assert lib.psrl_rope_rows(rope, same, pos, y=same, inverse=True) is same and torch.equal(same, y)
    assert lib.psrl_rope_rows(rope, x[:0], pos[:0]).shape == (0, heads, d)


def test_streams_graphs_and_no_query_rows(lib):
    w = make_workload("c2s", 4)
    plan = build_plan(lib, w)
    V = plan.oracle
    rope = lib.Rope(128)
    g = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda: torch.randn(V["T_q"], 48, 128, device="cuda", generator=g).to(torch.bfloat16)
    x = draw()
    pools = [torch.zeros(8, V["pool_slots"], 128, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    split = lambda t: (t[:, :32], t[:, 32:40], t[:, 40:])
    want = lib.psrl_rope_qkv_fwd(plan, rope, *split(x), *pools)
    want_pools = [p.clone() for p in pools]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for p in pools:
        p.zero_()
    side.wait_stream(torch.cuda.current_stream())
    got = lib.psrl_rope_qkv_fwd(plan, rope, *split(x), *pools, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(pools, want_pools))
    # captured, then replayed on new inputs in the same buffers
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.psrl_rope_qkv_fwd(plan, rope, *split(x), *pools, q_out=out)
    y = draw()
    want = lib.psrl_rope_qkv_fwd(plan, rope, *split(y), *pools)
    want_pools = [p.clone() for p in pools]
    x.copy_(y)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(pools, want_pools))
    # a plan without query rows: nothing to do
    w = Workload("nq", [-1, 0], [200, 70], [64], 4, 2, 128, "bf16", seg_flags=[0, 2])
    plan = build_plan(lib, w)
    empty = lambda h: torch.empty(0, h, 128, device="cuda", dtype=torch.bfloat16)
    pools = [torch.full((2, plan.oracle["pool_slots"], 128), 3.0, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    assert lib.psrl_rope_qkv_fwd(plan, rope, empty(4), empty(2), empty(2), *pools).shape == (0, 4, 128)
    assert all((p == 3.0).all() for p in pools)


def test_wrapper_refusals(lib):
    w = Workload("x", [-1, 0], [20, 5], [16], 2, 1, 128, "bf16")
    plan, rope = build_plan(lib, w), lib.Rope(128)
    t = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.bfloat16)
    good = dict(q=t(25, 2, 128), k=t(25, 1, 128), v=t(25, 1, 128), k_pool=t(1, 48, 128), v_pool=t(1, 48, 128))
    lib.psrl_rope_qkv_fwd(plan, rope, **good)
    for bad in (dict(q=t(24, 2, 128)), dict(k=t(25, 2, 128)), dict(q=t(25, 128, 2).transpose(1, 2)), dict(v_pool=t(1, 64, 128)),
                dict(k_pool=t(2, 48, 128)), dict(q_out=t(25, 3, 128)[:, :2])):
        with pytest.raises(ValueError):
            lib.psrl_rope_qkv_fwd(plan, rope, **{**good, **bad})
    for bad in (dict(q=good["q"].float()), dict(k=good["k"].half())):
        with pytest.raises(TypeError):
            lib.psrl_rope_qkv_fwd(plan, rope, **{**good, **bad})
    with pytest.raises(RuntimeError):
        lib.psrl_rope_qkv_fwd(plan, rope, **{**good, "q": good["q"].cpu()})
    with pytest.raises(ValueError):
        lib.psrl_rope_rows(rope, good["q"], torch.zeros(24, device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError):
        lib.psrl_rope_rows(rope, good["q"], torch.zeros(25, device="cuda", dtype=torch.int64))
    with pytest.raises(TypeError):
        lib.psrl_rope_rows(rope, good["q"].half(), torch.zeros(25, device="cuda", dtype=torch.int32))
    with pytest.raises(lib.PsrlError) as e:      # a slice that starts off a 16-byte boundary
        lib.psrl_rope_qkv_fwd(plan, rope, **{**good, "q": t(25 * 256 + 8)[3:3 + 25 * 256].view(25, 2, 128)})
    assert e.value.name == "PSRL_ERR_INVALID_ARG"
