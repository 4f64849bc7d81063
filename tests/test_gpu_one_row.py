"""Calls on one row that is a slice of a larger tensor (the next token of one rollout): the bits of that row in the whole call, whether the call
takes its one-step way or, with a stream given, the wrapper's."""
import numpy as np
import pytest
import torch

from oracle.layer import oracle_axes, oracle_rope_axes
from paper_2608_25683_b200.workloads import Workload

from util import build_plan, to_np

pytestmark = pytest.mark.gpu


def same(a, b):
    return a.shape == b.shape and a.dtype == b.dtype and torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def rope_of(lib, sections, d):
    return lib.Rope(d, base=10000.0, sections=sections, order="cyclic")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sections", [[24, 20, 20], [32, 32], [16, 16, 16, 16]])
def test_rows_at_a_slice_of_positions(lib, dtype, sections):
    """The last column, too: behind it there is nothing of the last axis."""
    rope, axes, T = rope_of(lib, sections, 128), len(sections), 9
    x = torch.randn(T, 3, 128, device="cuda").to(dtype)
    pos = torch.randint(0, 5000, (axes, T), device="cuda", dtype=torch.int32)
    here = torch.cuda.current_stream()
    for inverse in (False, True):
        whole = lib.psrl_rope_axes_rows(rope, x, pos, inverse=inverse)
        for t in (0, 3, T - 1):
            one = lib.psrl_rope_axes_rows(rope, x[t:t + 1], pos[:, t:t + 1], inverse=inverse)
            other = lib.psrl_rope_axes_rows(rope, x[t:t + 1], pos[:, t:t + 1], inverse=inverse, stream=here)
            torch.cuda.synchronize()
            assert same(one, whole[t:t + 1]) and same(other, one), t
            # angles within 2^-21 and products within 8 x 2^-24 of |x1| + |x2| <= 2 max|x|; a bf16 result half a step, 2^-8, besides
            want = oracle_rope_axes(to_np(x[t:t + 1]), pos[:, t:t + 1].cpu().numpy(), oracle_axes(sections, "cyclic"), rope.freq, 1.0, inverse=inverse)
            tol = 2.0 ** -20 * 2 * float(x.abs().max()) + (2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8) if dtype == torch.bfloat16 else 0.0)
            assert (np.abs(to_np(one) - want) <= tol).all()
    # one position for all axes has its axes no distance apart: refused on both ways
    for kw in ({}, {"stream": here}):
        with pytest.raises(lib.PsrlError) as e:
            lib.psrl_rope_axes_rows(rope, x[:1], pos[:1, :1].expand(axes, 1), **kw)
        assert e.value.name == "PSRL_ERR_SHAPE"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_plan_of_one_query_row(lib, dtype):
    """A tree whose prefix is cached and whose one branch has a single new token."""
    Hq, Hkv, D = 4, 2, 128
    sections = [24, 20, 20]
    plan = build_plan(lib, Workload("o", [-1, 0], [40, 1], [16], Hq, Hkv, D, dtype, seg_flags=[0, 3]))
    V = plan.oracle
    assert V["T_q"] == 1
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rope, here = rope_of(lib, sections, D), torch.cuda.current_stream()
    wide = torch.randint(0, 5000, (3, 11), device="cuda", dtype=torch.int32)
    x = torch.randn(1, Hq + 2 * Hkv, D, device="cuda").to(t)
    split = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    pools = lambda: [torch.zeros(Hkv, V["pool_slots"], D, device="cuda", dtype=t) for _ in range(2)]
    for at in (0, 5, 10):
        pos = wide[:, at:at + 1]
        turned = lib.psrl_rope_axes_rows(rope, x, pos.contiguous())
        for kw in ({}, {"stream": here}):
            p = pools()
            q = lib.psrl_rope_axes_qkv_fwd(plan, rope, pos, *split, *p, **kw)
            torch.cuda.synchronize()
            assert same(q, turned[:, :Hq])
            slot = int(V["tok_slot"][V["seg_tok_off"][1]])
            assert same(p[0][:, slot], turned[0, Hq:Hq + Hkv]) and same(p[1][:, slot], x[0, Hq + Hkv:])
            back = lib.psrl_rope_axes_qkv_bwd(plan, rope, pos, q, *p, **kw)
            torch.cuda.synchronize()
            assert same(back[0], lib.psrl_rope_axes_rows(rope, q, pos.contiguous(), inverse=True))
            assert same(back[1], lib.psrl_rope_axes_rows(rope, p[0][:, slot][None].contiguous(), pos.contiguous(), inverse=True))
            assert same(back[2], split[2])


def test_one_row_slices_of_every_operand(lib):
    """Each row of the operands of norms and products as a slice of one row, at pitches of their own, by both ways: the same bits, and
    the oracle's rows by the tests of many rows."""
    H, F, T = 512, 264, 7
    g = torch.Generator(device="cuda").manual_seed(1)
    bf = torch.bfloat16
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).to(bf)
    here = torch.cuda.current_stream()
    x, dy, ds, wide, d = rnd(T, H + 24), rnd(T, H + 8), rnd(T, H), rnd(T, 3 * F), rnd(T, F + 16)
    gain, w, bias, head = rnd(H), rnd(F, H), rnd(F), rnd(1, H)
    codes, scales = lib.psrl_quantize_rows(x[:, 8:8 + H])
    wc, ws = lib.psrl_quantize_rows(w)
    heads = rnd(T, 6, 128)
    for t in (0, 3, T - 1):
        r = slice(t, t + 1)
        xs, mul, res, z = x[r, 8:8 + H], wide[r, :F], wide[r, F:2 * F], wide[r, 2 * F:]
        calls = [
            (lib.psrl_rms_norm_fwd, (xs, gain), dict(residual=ds[r], want_codes=True)),
            (lib.psrl_rms_norm_fwd, (heads[r, 1:5], None), dict(want_codes=True)),
            (lib.psrl_rms_norm_bwd, (xs, gain, dy[r, :H]), dict(d_summed=ds[r])),
            (lib.psrl_rms_norm_bwd, (heads[r, 1:5], heads[0, 0].contiguous(), heads[r, 2:6]), dict()),
            (lib.psrl_linear_fwd, (xs, w), dict(bias=bias, mul=mul, residual=res, activation="silu", want_z=True)),
            (lib.psrl_linear_fwd, (xs, head), dict()),                                                                 # one row, one column
            (lib.psrl_linear_fwd, (codes[r], wc), dict(x_scale=scales[r], weight_scale=ws, residual=res)),
            (lib.psrl_linear_fwd, (xs.float(), w.float()), dict(mul=mul.float())),
            (lib.psrl_linear_bwd, (xs, w, d[r, 16:]), dict(z=z, activation="gelu", mul=mul, want_bias=True)),
            (lib.psrl_linear_bwd, (xs.float(), w.float(), d[r, 16:].float()), dict(want_bias=True)),
        ]
        for f, args, kw in calls:
            got, want = f(*args, **kw), f(*args, **kw, stream=here)
            whole = f(*(a.contiguous() for a in args[:1]), *(a if a is None else a.contiguous() for a in args[1:]),
                      **{k: v.contiguous() if isinstance(v, torch.Tensor) else v for k, v in kw.items()})
            torch.cuda.synchronize()
            for a, b, c in zip(got, want, whole):
                assert (a is None and b is None and c is None) or (same(a, b) and same(a, c)), (f.__name__, kw)
