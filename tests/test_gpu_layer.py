"""A transformer layer around the tree attention, all of it through the library, as an update step runs it: norm -> Q, K, V in one
product with bias -> norms of q and k by head -> rotary positions with three axes into the pools -> tree attention -> output projection
onto the residual stream -> norm -> gated MLP -> norm -> log-probabilities of the next tokens, and all the gradients back to the layer's
input and its weights; and the forward alone with 8-bit operands, as reference and old-policy passes run it.

The reference computes every sample on its own in fp64 (torch autograd): causal attention at the sample's positions, softmax over the
vocabulary, and sums loss and gradients over the samples, each with an advantage of its own.

Tolerance: every matrix that is kept is rounded to bf16, half a step, 2^-8 of its values.  Forward at most 12 of them lie one behind the
other (norm, projection, q/k norm, rotation, P, attention, stream, norm, factor, gate, stream, norm), backward as many and the
weights' own: 25 x 2^-8 in the 2-norm.  With 8-bit operands a product's two operands are off by 2^-4 each, four products one behind the
other: 8 x 2^-4 of the logits' spread, at most."""
import numpy as np
import pytest
import torch

from oracle import sample_paths
from oracle.layer import oracle_axes
from oracle.rope import oracle_rope_frequencies
from paper_2608_25683_b200.workloads import Workload

from util import build_plan, to_np

pytestmark = pytest.mark.gpu
Hq, Hkv, D, H, F, VOCAB = 4, 2, 128, 512, 1040, 701
SECTIONS, ORDER, BASE, EPS, SCALE = [24, 20, 20], "cyclic", 10000.0, 1e-5, 128 ** -0.5
FOREST = dict(parent=[-1, 0, 0, 2, 2, -1, 5, 5], seg_len=[130, 33, 70, 1, 45, 64, 17, 129], gbs=[64, 16])


def make(T, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    bf = torch.bfloat16
    w = dict(norm1=1 + 0.1 * rnd(H), qkv=rnd((Hq + 2 * Hkv) * D, H) / H ** 0.5, qkv_bias=0.1 * rnd((Hq + 2 * Hkv) * D), q_norm=1 + 0.1 * rnd(D), k_norm=1 + 0.1 * rnd(D),
             out=rnd(H, Hq * D) / (Hq * D) ** 0.5, norm2=1 + 0.1 * rnd(H), up=rnd(F, H) / H ** 0.5, gate=rnd(F, H) / H ** 0.5, down=rnd(H, F) / F ** 0.5, norm3=1 + 0.1 * rnd(H),
             head=0.2 * rnd(VOCAB, H))
    pos = torch.randint(0, 40, (3, T), generator=g, device="cuda", dtype=torch.int32)
    return rnd(T, H).to(bf), {k: v.to(bf) for k, v in w.items()}, pos, torch.randint(0, VOCAB, (T,), generator=g, device="cuda")


def paths_of(V):
    return [[t for c in path for t in range(V["seg_tok_off"][c], V["seg_tok_off"][c] + V["seg_len"][c])] for path in sample_paths(V)]


def reference(V, x, w, pos, ids, advantage):
    """Log-probabilities of the transitions and the gradients of x and the weights, sample by sample in fp64."""
    x = x.double().cpu().requires_grad_(True)
    w = {k: v.double().cpu().requires_grad_(True) for k, v in w.items()}
    freq = torch.as_tensor(oracle_rope_frequencies(D, BASE)[0])
    angle = pos.cpu().double()[torch.as_tensor(oracle_axes(SECTIONS, ORDER))].T * freq
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    norm = lambda v, gain: v * (v.pow(2).mean(-1, keepdim=True) + EPS).rsqrt() * gain
    loss, logprob = 0.0, {}
    for tok, a in zip(paths_of(V), advantage):
        h = x[tok]
        qkv = (norm(h, w["norm1"]) @ w["qkv"].T + w["qkv_bias"]).view(len(tok), -1, D)
        turn = lambda v: torch.cat([v[..., :D // 2] * cos[tok] - v[..., D // 2:] * sin[tok], v[..., D // 2:] * cos[tok] + v[..., :D // 2] * sin[tok]], -1)
        q, k, v = turn(norm(qkv[:, :Hq], w["q_norm"])), turn(norm(qkv[:, Hq:Hq + Hkv], w["k_norm"])), qkv[:, Hq + Hkv:]
        k, v = (t.repeat_interleave(Hq // Hkv, 1) for t in (k, v))
        s = torch.einsum("ihd,jhd->hij", q, k) * SCALE
        s = s.masked_fill(torch.ones(len(tok), len(tok), dtype=torch.bool).triu(1), float("-inf"))
        h = h + torch.einsum("hij,jhd->ihd", s.softmax(-1), v).reshape(len(tok), -1) @ w["out"].T
        y = norm(h, w["norm2"])
        h = h + (torch.nn.functional.silu(y @ w["gate"].T) * (y @ w["up"].T)) @ w["down"].T
        lp = torch.log_softmax(norm(h, w["norm3"])[:-1] @ w["head"].T, -1)[torch.arange(len(tok) - 1), ids[tok[1:]]]
        loss = loss + a * lp.sum()
        logprob.update({(i, j): float(l) for i, j, l in zip(tok, tok[1:], lp.detach())})
    loss.backward()
    return logprob, x.grad, {k: v.grad for k, v in w.items()}


def forward(lib, plan, rope, x, w, pos, linear):
    """All that the backward needs; linear(rows, name, **epilogue) is a product with weight `name` of normed or plain rows."""
    f = {}
    V = plan.oracle
    f["qkv"] = linear(x, "qkv", "norm1", bias=w["qkv_bias"]).view(V["T_q"], -1, D)
    f["q"] = lib.psrl_rms_norm_fwd(f["qkv"][:, :Hq], w["q_norm"], EPS)[0]
    f["k"] = lib.psrl_rms_norm_fwd(f["qkv"][:, Hq:Hq + Hkv], w["k_norm"], EPS)[0]
    f["pools"] = [torch.full((Hkv, V["pool_slots"], D), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    f["q_rot"] = lib.psrl_rope_axes_qkv_fwd(plan, rope, pos, f["q"], f["k"], f["qkv"][:, Hq + Hkv:], *f["pools"])
    f["o"], f["lse"] = lib.psrl_tree_attn_fwd(plan, f["q_rot"], *f["pools"], SCALE)
    f["attn"] = linear(f["o"].view(V["T_q"], -1), "out", None)
    f["y2"], f["h1"], _, _ = lib.psrl_rms_norm_fwd(f["attn"], w["norm2"], EPS, residual=x)
    f["up"] = linear(f["h1"], "up", "norm2")
    f["act"], f["z"] = linear(f["h1"], "gate", "norm2", activation="silu", mul=f["up"], want_z=True)
    f["h2"] = linear(f["act"], "down", None, residual=f["h1"])
    f["y3"] = lib.psrl_rms_norm_fwd(f["h2"], w["norm3"], EPS)[0]
    return f


@pytest.mark.parametrize("seed", [1, 2])
def test_one_layer_there_and_back(lib, seed):
    plan = build_plan(lib, Workload("l", FOREST["parent"], FOREST["seg_len"], FOREST["gbs"], Hq, Hkv, D, "bf16"))
    V = plan.oracle
    x, w, pos, ids = make(V["T"], seed)
    advantage = np.random.default_rng(seed).normal(size=V["n_samples"])
    want_lp, want_x, want_w = reference(V, x, w, pos, ids.cpu(), advantage)
    weights = {}
    for tok, a in zip(paths_of(V), advantage):
        for t in zip(tok, tok[1:]):
            weights[t] = weights.get(t, 0.0) + a
    rope = lib.Rope(D, base=BASE, sections=SECTIONS, order=ORDER)
    normed = {}

    def linear(rows, name, gain, **kw):
        if gain is not None:
            key = (rows.data_ptr(), gain)
            if key not in normed:
                normed[key] = lib.psrl_rms_norm_fwd(rows, w[gain], EPS)[0]
            rows = normed[key]
        y, z = lib.psrl_linear_fwd(rows, w[name], **kw)
        return (y, z) if kw.get("want_z") else y

    f = forward(lib, plan, rope, x, w, pos, linear)
    off, nxt = plan.next_tokens()
    off_d, targets = torch.as_tensor(off, device="cuda"), ids[torch.as_tensor(nxt, device="cuda").long()].to(torch.int32)
    lp, z_lse = lib.psrl_token_logprob_fwd(f["y3"], w["head"], targets, off_d)
    row = np.repeat(np.arange(V["T_q"]), np.diff(off))
    ref_lp = np.array([want_lp[(int(r), int(t))] for r, t in zip(row, nxt)])
    spread = float((f["y3"].double() @ w["head"].double().T).std(1).max())
    assert np.abs(to_np(lp) - ref_lp).max() <= 12 * 2.0 ** -8 * 4 * spread

    grad = torch.as_tensor([weights[(int(r), int(t))] for r, t in zip(row, nxt)], dtype=torch.float32, device="cuda")
    g = {}
    d, g["head"] = lib.psrl_token_logprob_bwd(f["y3"], w["head"], targets, lp, z_lse, grad, off_d)
    d_h2, g["norm3"] = lib.psrl_rms_norm_bwd(f["h2"], w["norm3"], d, EPS)
    d_act, g["down"], _, _ = lib.psrl_linear_bwd(f["act"], w["down"], d_h2)
    y2 = f["y2"]
    d_y2, g["gate"], _, d_up = lib.psrl_linear_bwd(y2, w["gate"], d_act, z=f["z"], activation="silu", mul=f["up"])
    d_y2_up, g["up"], _, _ = lib.psrl_linear_bwd(y2, w["up"], d_up)
    # the two products of y2 each give a gradient of it
    d_y2 = (d_y2.float() + d_y2_up.float()).to(torch.bfloat16)
    d_h1, g["norm2"] = lib.psrl_rms_norm_bwd(f["h1"], w["norm2"], d_y2, EPS, d_summed=d_h2)
    d_o, g["out"], _, _ = lib.psrl_linear_bwd(f["o"].view(V["T_q"], -1), w["out"], d_h1)
    dq, dkp, dvp = lib.psrl_tree_attn_bwd(plan, f["q_rot"], *f["pools"], f["o"], f["lse"], d_o.view_as(f["o"]), SCALE)
    d_qkv = torch.empty_like(f["qkv"])
    lib.psrl_rope_axes_qkv_bwd(plan, rope, pos, dq, dkp, dvp, dq_out=d_qkv[:, :Hq], dk_out=d_qkv[:, Hq:Hq + Hkv], dv_out=d_qkv[:, Hq + Hkv:])
    _, g["q_norm"] = lib.psrl_rms_norm_bwd(f["qkv"][:, :Hq], w["q_norm"], d_qkv[:, :Hq], EPS, d_x=d_qkv[:, :Hq])
    _, g["k_norm"] = lib.psrl_rms_norm_bwd(f["qkv"][:, Hq:Hq + Hkv], w["k_norm"], d_qkv[:, Hq:Hq + Hkv], EPS, d_x=d_qkv[:, Hq:Hq + Hkv])
    y1 = normed[(x.data_ptr(), "norm1")]
    d_y1, g["qkv"], g["qkv_bias"], _ = lib.psrl_linear_bwd(y1, w["qkv"], d_qkv.view(V["T_q"], -1), want_bias=True)
    d_x, g["norm1"] = lib.psrl_rms_norm_bwd(x, w["norm1"], d_y1, EPS, d_summed=d_h1)
    assert lib.psrl_device_status(plan, "bwd") == 0
    assert set(g) == set(want_w)
    for name, got, want in [("x", d_x, want_x)] + [(k, g[k], want_w[k]) for k in g]:
        rel = float((got.double().cpu() - want).norm() / want.norm())
        assert rel <= 25 * 2.0 ** -8, (name, rel)


def test_forward_with_8_bit_operands(lib):
    plan = build_plan(lib, Workload("l", FOREST["parent"], FOREST["seg_len"], FOREST["gbs"], Hq, Hkv, D, "bf16"))
    V = plan.oracle
    x, w, pos, ids = make(V["T"], 3)
    want_lp, _, _ = reference(V, x, w, pos, ids.cpu(), np.ones(V["n_samples"]))
    rope = lib.Rope(D, base=BASE, sections=SECTIONS, order=ORDER)
    codes = {k: lib.psrl_quantize_rows(w[k]) for k in ("qkv", "out", "up", "gate", "down")}      # laid out once

    def linear(rows, name, gain, **kw):
        if gain is not None:
            _, _, q, s = lib.psrl_rms_norm_fwd(rows, w[gain], EPS, want_y=False, want_codes=True)
        else:
            q, s = lib.psrl_quantize_rows(rows)
        y, z = lib.psrl_linear_fwd(q, codes[name][0], x_scale=s, weight_scale=codes[name][1], **kw)
        return (y, z) if kw.get("want_z") else y

    f = forward(lib, plan, rope, x, w, pos, linear)
    off, nxt = plan.next_tokens()
    off_d, targets = torch.as_tensor(off, device="cuda"), ids[torch.as_tensor(nxt, device="cuda").long()].to(torch.int32)
    lp, _ = lib.psrl_token_logprob_fwd(f["y3"], w["head"], targets, off_d)
    row = np.repeat(np.arange(V["T_q"]), np.diff(off))
    ref_lp = np.array([want_lp[(int(r), int(t))] for r, t in zip(row, nxt)])
    spread = float((f["y3"].double() @ w["head"].double().T).std(1).max())
    err = np.abs(to_np(lp) - ref_lp)
    assert err.max() <= 8 * 2.0 ** -4 * 4 * spread and np.sqrt((err ** 2).mean()) <= 8 * 2.0 ** -4 * spread


def test_calls_in_one_step_are_the_calls(lib):
    """The plain case of a call goes to the library in one step, any other through the wrapper (a stream given, a tensor's subclass, an
    output given): the same bits, the same refusals."""
    T = 70
    plan = build_plan(lib, Workload("s", [-1, 0], [50, 20], [16], Hq, Hkv, D, "bf16"))
    x, w, pos, _ = make(T, 4)
    here = torch.cuda.current_stream()
    rope = lib.Rope(D, base=BASE, sections=SECTIONS, order=ORDER)
    same = lambda a, b: (a is None and b is None) or (a.shape == b.shape and a.dtype == b.dtype and torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)))
    class Sub(torch.Tensor):
        pass
    sub = x.as_subclass(Sub)
    d = torch.randn(T, F, device="cuda").to(torch.bfloat16)
    mul, z = d * 0.5, d * 0.25
    wide = torch.randn(T, F + 24, device="cuda").to(torch.bfloat16)
    codes, scales = lib.psrl_quantize_rows(x)
    wc, ws = lib.psrl_quantize_rows(w["up"])
    calls = [
        (lib.psrl_rms_norm_fwd, (x, w["norm1"]), dict(eps=EPS, residual=x, want_codes=True)),
        (lib.psrl_rms_norm_fwd, (wide[:, 8:8 + F], None), dict(want_y=0, want_codes=1)),
        (lib.psrl_rms_norm_fwd, (x.view(T, 4, 128)[:, 1:3], w["q_norm"]), dict(want_codes=True)),
        (lib.psrl_rms_norm_fwd, (x.view(-1, 8), None), dict(want_codes=True)),        # codes 16 bytes apart: not the plain case
        (lib.psrl_rms_norm_bwd, (x, w["norm1"], x * 0.5), dict(eps=EPS, d_summed=x)),
        (lib.psrl_rms_norm_bwd, (x, None, x * 0.5), dict()),
        (lib.psrl_rms_norm_bwd, (x, w["norm1"], x * 0.5), dict(want_x=False)),
        (lib.psrl_linear_fwd, (x, w["up"]), dict(mul=mul, residual=wide[:, 16:16 + F], activation="gelu", want_z=True)),
        (lib.psrl_linear_fwd, (codes, wc), dict(x_scale=scales, weight_scale=ws)),
        (lib.psrl_linear_fwd, (x, w["head"]), dict()),                                 # 701 columns
        (lib.psrl_linear_fwd, (x.float(), w["head"].float()), dict(activation="silu")),
        (lib.psrl_linear_bwd, (x, w["up"], d), dict(z=z, activation="silu", mul=mul, want_bias=True)),
        (lib.psrl_linear_bwd, (x, w["up"], d), dict(want_x=False)),
        (lib.psrl_linear_bwd, (x.float(), w["up"].float(), d.float()), dict(want_bias=True)),
        (lib.psrl_linear_fwd, (x[:0], w["up"]), dict(want_z=True)),
        (lib.psrl_rms_norm_fwd, (x[:0], w["norm1"]), dict(want_codes=True)),
    ]
    for f, args, kw in calls:
        got, want = f(*args, **kw), f(*args, **kw, stream=here)
        torch.cuda.synchronize()
        assert len(got) == len(want) and all(same(a, b) for a, b in zip(got, want)), (f.__name__, kw)
    assert all(same(a, b) for a, b in zip(lib.psrl_linear_fwd(sub, w["up"]), lib.psrl_linear_fwd(x, w["up"])))
    q, k, v = (torch.randn(T, h, D, device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
    pools = lambda: [torch.zeros(Hkv, plan.oracle["pool_slots"], D, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    a, b = pools(), pools()
    assert same(lib.psrl_rope_axes_qkv_fwd(plan, rope, pos, q, k, v, *a), lib.psrl_rope_axes_qkv_fwd(plan, rope, pos, q, k, v, *b, stream=here))
    torch.cuda.synchronize()
    assert same(a[0], b[0]) and same(a[1], b[1])
    for got, want in zip(lib.psrl_rope_axes_qkv_bwd(plan, rope, pos, q, *a), lib.psrl_rope_axes_qkv_bwd(plan, rope, pos, q, *a, stream=here)):
        torch.cuda.synchronize()
        assert same(got, want)
    got, want = lib.psrl_rope_axes_rows(rope, q, pos, inverse=1), lib.psrl_rope_axes_rows(rope, q, pos, inverse=True, stream=here)
    torch.cuda.synchronize()
    assert same(got, want)
    # a plan of another type, one that is not uploaded, one that is closed
    f32 = build_plan(lib, Workload("s", [-1, 0], [50, 20], [16], Hq, Hkv, D, "f32"))
    with pytest.raises(TypeError):
        lib.psrl_rope_axes_qkv_fwd(f32, rope, pos, q, k, v, *a)
    fresh = lib.Plan([-1, 0], [50, 20], [16], Hq, Hkv, D, "bf16")
    with pytest.raises(lib.PsrlError) as e:
        lib.psrl_rope_axes_qkv_fwd(fresh, rope, pos, q, k, v, *a)
    assert e.value.name == "PSRL_ERR_WORKSPACE"
    fresh.upload().close()
    with pytest.raises(lib.PsrlError) as e:
        lib.psrl_rope_axes_qkv_fwd(fresh, rope, pos, q, k, v, *a)
    assert e.value.name == "PSRL_ERR_INVALID_ARG"
    # memory that is out is torch's error
    tall = torch.zeros(1 << 20, 8, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(torch.OutOfMemoryError):
        lib.psrl_linear_fwd(tall, tall)
