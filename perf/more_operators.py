"""The operators of a transformer layer between the tree attention calls, in plain form and through the library.

  rms_fwd, rms_bwd         root-mean-square norm of h = x + residual, h handed on as the new residual stream; per row, or per
                           head of a row (norms of q and k, on slices of a projection); output in the inputs' type, in 8
                           bits (e4m3) with a scale for each row, or both; and the gradients
  linear_fwd, linear_bwd   y = act(x weight^T + bias) * mul + residual and its gradients; bf16, f32, and 8-bit operands with
                           scales for each row of x and of weight
  axes_fwd, axes_bwd       rotary positions with several axes (time, height, width), Q row by row, K on its way into the paged
                           pool, V copied beside it; and the way back
  axes_rows                the same rotation of rows at positions of their own
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------- the cases

def rms(kind, rows, dim, heads=1, dtype="bf16", residual=True, out="y", name=None):
    c = dict(kind=kind, rows=rows, dim=dim, heads=heads, dtype=dtype, residual=residual, out=out)
    return dict(c, name=name) if name else c


def linear(kind, rows, k, n, dtype="bf16", act="none", bias=False, mul=False, residual=False, z=False, name=None):
    c = dict(kind=kind, rows=rows, k=k, n=n, dtype=dtype, act=act, bias=bias, mul=mul, residual=residual, z=z)
    return dict(c, name=name) if name else c


def axes(kind, groups=1, prefix=0, branches=0, lo=1, hi=1, block=64, hq=32, hkv=8, d=128, dtype="bf16", layout="half", rotary=128,
         base=1000000.0, sections="16,24,24", order="blocks", forest=1, name=None):
    c = dict(kind=kind, groups=groups, prefix=prefix, branches=branches, lo=lo, hi=hi, block=block, hq=hq, hkv=hkv, d=d, dtype=dtype,
             layout=layout, rotary=rotary, base=base, sections=sections, order=order, forest=forest)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a step-wise group's residual stream through one norm of a 4096-wide model
        rms("rms_fwd", 8192, 4096, name="rms_fwd_group"),
        # the next tokens of 8 rollouts, the norm's output in 8 bits for the product behind it
        rms("rms_fwd", 8, 4096, out="codes", name="rms_fwd_tokens_8bit"),
        # the same norm's gradients, the residual stream's gradient added on the way
        rms("rms_bwd", 8192, 4096, name="rms_bwd_group"),
        # gradients of the norm of 5 heads of q, odd number of rows, fp32
        rms("rms_bwd", 1027, 64, heads=5, dtype="f32", residual=False, name="rms_bwd_heads_f32"),
        # Q, K and V of the group in one product, with bias
        linear("linear_fwd", 8192, 4096, 6144, bias=True, name="linear_fwd_qkv"),
        # the gate of a gated MLP for the next tokens of 8 rollouts: bound by the weights' bytes
        linear("linear_fwd", 8, 4096, 14336, act="silu", mul=True, name="linear_fwd_tokens_gate"),
        # forward-only phases: 8-bit operands, the residual stream added
        linear("linear_fwd", 8192, 14336, 4096, dtype="e4m3", residual=True, name="linear_fwd_8bit_down"),
        # gradients of the gate over a micro-batch
        linear("linear_bwd", 4096, 4096, 14336, act="silu", mul=True, name="linear_bwd_gate"),
        # an odd micro-batch of a small model with biases
        linear("linear_bwd", 777, 1000, 3584, act="gelu_tanh", bias=True, name="linear_bwd_odd"),
        # step-wise group with screenshots: 4096-token prefix, 8 branches
        axes("axes_fwd", prefix=4096, branches=8, lo=256, hi=1024, name="axes_fwd_group"),
        # long agentic group, gradients on their way back
        axes("axes_bwd", prefix=16384, branches=32, lo=512, hi=4096, block=256, hq=64, hkv=8, sections="24,20,20", order="cyclic", name="axes_bwd_long"),
        # one new token for each of 8 sequences
        dict(name="axes_rows_tokens", kind="axes_rows", rows=8, heads=40, d=128, dtype="bf16", layout="half", rotary=128, base=1000000.0,
             sections="16,24,24", order="blocks", far=32768, inverse=False),
    ]


def spread(rng, lo, hi):
    """A whole number of lo..hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def sections_of(rng, pairs):
    """Pairs of three axes (one of them cyclic over the pairs, the other in blocks), as text."""
    if rng.random() < 0.5:
        h = rng.randint(1, pairs // 3)
        w = rng.randint(1, pairs // 3)
        return "%d,%d,%d" % (pairs - h - w, h, w), "cyclic"
    h, w = rng.randint(0, pairs // 2), rng.randint(1, pairs // 2)
    return "%d,%d,%d" % (pairs - h - w, h, w), "blocks"


def draw(rng):
    kind = rng.choice(["rms_fwd", "rms_bwd", "linear_fwd", "linear_fwd", "linear_bwd", "axes_fwd", "axes_bwd", "axes_rows"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("rms_fwd", "rms_bwd"):
        out = rng.choice(["y", "y", "codes", "both"]) if kind == "rms_fwd" else "y"
        if rng.random() < 0.3:
            return rms(kind, spread(rng, 1, 8192), rng.choice([64, 80, 128, 256]), spread(rng, 1, 64), dtype, False, out)
        return rms(kind, spread(rng, 1, 8192), 8 * spread(rng, 32, 1024), 1, dtype, rng.random() < 0.7, out)
    if kind == "linear_fwd":
        dtype = rng.choice(["bf16", "bf16", "e4m3", "f32"])
        f32 = dtype == "f32"
        mul, residual, n = rng.random() < 0.4, rng.random() < 0.4, spread(rng, 256, 2048 if f32 else 8192)
        # beside other matrices of whole 16-byte vectors; alone as it comes
        return linear(kind, spread(rng, 1, 1024 if f32 else 8192), 16 * spread(rng, 16, 128 if f32 else 512), n // 8 * 8 if mul or residual else n, dtype,
                      rng.choice(["none", "none", "relu", "silu", "gelu", "gelu_tanh"]), rng.random() < 0.5, mul, residual, rng.random() < 0.3)
    if kind == "linear_bwd":
        f32 = dtype == "f32"
        return linear(kind, spread(rng, 1, 1024 if f32 else 4096), 8 * spread(rng, 32, 256 if f32 else 768), 8 * spread(rng, 32, 256 if f32 else 1024), dtype,
                      rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]), rng.random() < 0.5, rng.random() < 0.4)
    layout, base = rng.choice(["half", "interleaved"]), rng.choice([10000.0, 500000.0, 1000000.0])
    if kind == "axes_rows":
        d = rng.choice([64, 128])
        rotary = rng.choice([d, d // 2])
        sections, order = sections_of(rng, rotary // 2)
        return dict(kind=kind, rows=spread(rng, 1, 5000), heads=rng.choice([1, 5, 8, 40, 72]), d=d, dtype=dtype, layout=layout, rotary=rotary,
                    base=base, sections=sections, order=order, far=spread(rng, 2, 1000000), inverse=rng.random() < 0.5)
    d = 128 if dtype == "bf16" else rng.choice([64, 128])
    hkv = rng.choice([1, 2, 4, 8])
    rotary = rng.choice([d, d, d // 2])
    sections, order = sections_of(rng, rotary // 2)
    return axes(kind, rng.choice([1, 1, 2, 5]), spread(rng, 1, 8192), spread(rng, 1, 24), 1, spread(rng, 2, 1024), rng.choice([16, 64, 256]),
                hkv * rng.choice([1, 3, 4, 7]), hkv, d, dtype, layout, rotary, base, sections, order, rng.randrange(1 << 20))


# --------------------------------------------------------------------------------------------------- the inputs

def forest_of(c):
    """Star forests in canonical order: per group one prefix and its branches. (parent, lengths)"""
    r = random.Random(c["forest"])
    parent, length = [], []
    for _ in range(c["groups"]):
        root = len(parent)
        parent.append(-1)
        length.append(c["prefix"])
        for _ in range(c["branches"]):
            parent.append(root)
            length.append(r.randint(c["lo"], c["hi"]))
    return parent, length


def slots_of(c):
    """Per row its slot, and the number of slots: blocks of whole pages, one segment after the other."""
    at, slot = 0, []
    for n in forest_of(c)[1]:
        slot.append(np.arange(at, at + n))
        at += -(-n // c["block"]) * c["block"]
    return np.concatenate(slot), at


def positions_of(c):
    """[3, rows]: text, where the axes go together, with images in it, whose tokens lie on a grid; text goes on behind the
    largest coordinate. A branch goes on where its prefix ends."""
    r = random.Random(c["forest"] + 1)
    parent, length = forest_of(c)
    out, end = [], []
    for p, n in zip(parent, length):
        at, left, parts = (0 if p < 0 else end[p]), n, []
        while left:
            text = min(left, spread(r, 1, 400))
            parts.append(np.tile(np.arange(at, at + text), (3, 1)))
            at, left = at + text, left - text
            t, h, w = r.choice([1, 1, 4]), r.randint(2, 24), r.randint(2, 24)
            if left >= t * h * w:
                i = np.arange(t * h * w)
                parts.append(at + np.stack([i // (h * w), i // w % h, i % w]))
                at, left = at + max(t, h, w), left - t * h * w
        end.append(at)
        out.append(np.concatenate(parts, axis=1))
    return np.concatenate(out, axis=1).astype(np.int32)


def prepare(case, seed):
    c, kind = case, case["kind"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    s = {"case": c}
    if kind in ("rms_fwd", "rms_bwd"):
        t, n, h, d = TYPES[c["dtype"]], c["rows"], c["heads"], c["dim"]
        # the stream of a deep layer: rows of different size, a few channels that stand out
        loud = 1.0 + 20.0 * (torch.rand(d, generator=g, device="cuda") < 0.002)
        stream = lambda: rnd(n, h, d) * loud * (0.5 + 2.0 * torch.rand(n, 1, 1, generator=g, device="cuda"))  # noqa: E731
        if h > 1:   # q of a projection whose rows hold k and v as well
            s["x"] = torch.cat([stream(), rnd(n, 2, d)], dim=1).to(t)[:, :h]
        else:
            s["x"] = stream()[:, 0].to(t)
        s["weight"] = (1.0 + 0.2 * rnd(d)).to(t)
        like = lambda: rnd(*s["x"].shape).to(t)  # noqa: E731
        if kind == "rms_fwd":
            s["residual"] = like() if c["residual"] else None
        else:
            s["d_y"], s["d_summed"] = like(), like() if c["residual"] else None
    elif kind in ("linear_fwd", "linear_bwd"):
        m, k, n = c["rows"], c["k"], c["n"]
        t = TYPES.get(c["dtype"], torch.bfloat16)
        x, w = rnd(m, k), rnd(n, k) * (1.0 + torch.rand(n, 1, generator=g, device="cuda")) / math.sqrt(k)
        if c["dtype"] == "e4m3":
            s["x"], s["x_scale"] = plain_codes(x)
            s["weight"], s["weight_scale"] = plain_codes(w)
        else:
            s["x"], s["weight"] = x.to(t), w.to(t)
        s["bias"] = (0.3 * rnd(n)).to(t) if c["bias"] else None
        s["mul"] = rnd(m, n).to(t) if c["mul"] else None
        if kind == "linear_fwd":
            s["residual"] = rnd(m, n).to(t) if c["residual"] else None
        else:
            s["d_y"] = rnd(m, n).to(t)
            z = s["x"].float() @ s["weight"].float().T
            s["z"] = (z if s["bias"] is None else z + s["bias"].float()).to(t) if c["act"] != "none" or c["mul"] else None
    elif kind == "axes_rows":
        s["x"] = rnd(c["rows"], c["heads"], c["d"]).to(TYPES[c["dtype"]])
        s["positions"] = torch.randint(0, c["far"], (3, c["rows"]), generator=g, device="cuda", dtype=torch.int32)
        if own:
            s["rope"] = rope_handle(c)
    else:
        t, d = TYPES[c["dtype"]], c["d"]
        slot, slots = slots_of(c)
        rows = len(slot)
        s["slot"], s["positions"] = torch.from_numpy(slot).cuda(), torch.from_numpy(positions_of(c)).cuda()
        s["q"] = rnd(rows, c["hq"], d).to(t)
        s["k"], s["v"] = rnd(rows, c["hkv"], d).to(t), rnd(rows, c["hkv"], d).to(t)
        s["k_pool"], s["v_pool"] = rnd(c["hkv"], slots, d).to(t), rnd(c["hkv"], slots, d).to(t)
        s["q_out"] = torch.empty_like(s["q"])
        if own:
            from paper_2608_25683_b200 import binding
            parent, length = forest_of(c)
            s["plan"] = binding.Plan(parent, length, [c["block"]] * c["groups"], c["hq"], c["hkv"], d, c["dtype"]).upload()
            s["rope"] = rope_handle(c)
    return s


def rope_handle(c):
    from paper_2608_25683_b200 import binding
    return binding.Rope(c["d"], rotary_dim=c["rotary"], base=c["base"], layout=c["layout"],
                        sections=[int(x) for x in c["sections"].split(",")], order=c["order"])


# ------------------------------------------------------------------------------------------------- one pass

def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        from paper_2608_25683_b200 import binding as b
        act = None if c.get("act") == "none" else c.get("act")
        if kind == "rms_fwd":
            y, summed, codes, scales = b.psrl_rms_norm_fwd(s["x"], s["weight"], EPS, residual=s["residual"], want_y=c["out"] != "codes",
                                                           want_codes=c["out"] != "y")
            return {"y": y, "summed": summed, "codes": codes, "scales": scales}
        if kind == "rms_bwd":
            return b.psrl_rms_norm_bwd(s["x"], s["weight"], s["d_y"], EPS, d_summed=s["d_summed"])
        if kind == "linear_fwd":
            return b.psrl_linear_fwd(s["x"], s["weight"], bias=s["bias"], activation=act, mul=s["mul"], residual=s["residual"],
                                     x_scale=s.get("x_scale"), weight_scale=s.get("weight_scale"), want_z=c["z"])
        if kind == "linear_bwd":
            return b.psrl_linear_bwd(s["x"], s["weight"], s["d_y"], z=s["z"], activation=act, mul=s["mul"], want_bias=c["bias"])
        if kind == "axes_fwd":
            q = b.psrl_rope_axes_qkv_fwd(s["plan"], s["rope"], s["positions"], s["q"], s["k"], s["v"], s["k_pool"], s["v_pool"], q_out=s["q_out"])
            return q, s["k_pool"], s["v_pool"]
        if kind == "axes_bwd":
            return b.psrl_rope_axes_qkv_bwd(s["plan"], s["rope"], s["positions"], s["q"], s["k_pool"], s["v_pool"], dq_out=s["q_out"],
                                            dk_out=s["k"], dv_out=s["v"])
        return b.psrl_rope_axes_rows(s["rope"], s["x"], s["positions"], inverse=c["inverse"])
    if kind == "rms_fwd":
        return plain_rms(s)
    if kind == "rms_bwd":
        return plain_rms_bwd(s)
    if kind == "linear_fwd":
        return plain_linear(s)
    if kind == "linear_bwd":
        return plain_linear_bwd(s)
    if kind == "axes_fwd":
        s["k_pool"][:, s["slot"]] = plain_rotate(s["k"], s["positions"], c, False).transpose(0, 1)
        s["v_pool"][:, s["slot"]] = s["v"].transpose(0, 1)
        return plain_rotate(s["q"], s["positions"], c, False), s["k_pool"], s["v_pool"]
    if kind == "axes_bwd":
        dk = plain_rotate(s["k_pool"][:, s["slot"]].transpose(0, 1), s["positions"], c, True)
        return plain_rotate(s["q"], s["positions"], c, True), dk, s["v_pool"][:, s["slot"]].transpose(0, 1).contiguous()
    return plain_rotate(s["x"], s["positions"], c, c["inverse"])


# ------------------------------------------------------------------------------------------------- plain forms

def plain_codes(y):
    """Rows in 8 bits: the values' codes and a scale for each row."""
    scale = (y.abs().amax(-1) / 448.0).clamp(min=2.0 ** -126)
    return (y / scale[..., None]).clamp(-448.0, 448.0).to(E4M3), scale


def plain_rms(s):
    h, summed = s["x"], None
    if s["residual"] is not None:
        h = summed = (h.float() + s["residual"].float()).to(h.dtype)
    f = h.float()
    y = f * ((f * f).mean(-1, keepdim=True) + EPS).rsqrt() * s["weight"].float()
    out = s["case"]["out"]
    codes, scales = plain_codes(y) if out != "y" else (None, None)
    return {"y": y.to(h.dtype) if out != "codes" else None, "summed": summed, "codes": codes, "scales": scales}


def plain_rms_bwd(s):
    h, w, dy = s["x"].float(), s["weight"].float(), s["d_y"].float()
    r = ((h * h).mean(-1, keepdim=True) + EPS).rsqrt()
    unit, g = h * r, dy * w
    dx = (g - unit * (g * unit).mean(-1, keepdim=True)) * r
    if s["d_summed"] is not None:
        dx = dx + s["d_summed"].float()
    return dx.to(s["x"].dtype), (dy * unit).flatten(0, -2).sum(0).to(s["x"].dtype)


def plain_act(z, act):
    """The activation's value and its slope."""
    if act == "relu":
        return z * (z > 0), (z > 0).float()
    if act == "silu":
        e = 1.0 / (1.0 + (-z).exp())
        return z * e, e * (1.0 + z * (1.0 - e))
    if act == "gelu":
        cdf = 0.5 * (1.0 + (z * math.sqrt(0.5)).erf())
        return z * cdf, cdf + z * (-0.5 * z * z).exp() / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = (c * (z + 0.044715 * z * z * z)).tanh()
        return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    return z, torch.ones_like(z)


def plain_linear(s):
    t = s["x"].dtype if s["x"].dtype != E4M3 else torch.bfloat16
    z = s["x"].float() @ s["weight"].float().T
    if "x_scale" in s:
        z = z * s["x_scale"][:, None] * s["weight_scale"]
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = plain_act(z, s["case"]["act"])[0] if s["case"]["act"] != "none" else z
    if s["mul"] is not None:
        y = y * s["mul"].float()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(t), z.to(t) if s["case"]["z"] else None


def plain_linear_bwd(s):
    t, x, w, dz = s["x"].dtype, s["x"].float(), s["weight"].float(), s["d_y"].float()
    d_mul = None
    if s["z"] is not None:
        a, slope = plain_act(s["z"].float(), s["case"]["act"])
        if s["mul"] is not None:
            d_mul = (dz * a).to(t)
            dz = dz * s["mul"].float()
        dz = dz * slope
    d_bias = dz.sum(0).to(t) if s["case"]["bias"] else None
    return (dz @ w).to(t), (dz.T @ x).to(t), d_bias, d_mul


def axis_of(c):
    """The axis that each pair of elements goes by."""
    n = [int(x) for x in c["sections"].split(",")]
    if c["order"] == "blocks":
        return [a for a in range(len(n)) for _ in range(n[a])]
    return [i % 3 if i < 3 * n[i % 3] else 0 for i in range(sum(n))]


def plain_rotate(x, pos, c, inverse):
    r = c["rotary"]
    freq = c["base"] ** (-2.0 * torch.arange(r // 2, dtype=torch.float64, device="cuda") / r)
    angle = pos.double()[axis_of(c)].T * freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    sin = -sin if inverse else sin
    f = x.float()
    if c["layout"] == "half":
        a, b = f[..., : r // 2], f[..., r // 2 : r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = f[..., 0:r:2], f[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([turned.to(x.dtype), x[..., r:]], dim=-1)


# ------------------------------------------------------------------------------------------- the work of one pass

def work(case):
    c, kind = case, case["kind"]
    b = {"bf16": 2, "f32": 4, "e4m3": 1}[c["dtype"]]
    if kind in ("rms_fwd", "rms_bwd"):
        n, d = c["rows"] * c["heads"], c["dim"]
        if kind == "rms_bwd":
            return {"bytes": n * d * b * (4 if c["residual"] else 3) + 2 * d * b, "flops": 12 * n * d}
        out = {"y": b, "codes": 1, "both": b + 1}[c["out"]]
        return {"bytes": n * d * (b * (3 if c["residual"] else 1) + out) + d * b + (4 * n if c["out"] != "y" else 0), "flops": 6 * n * d}
    if kind in ("linear_fwd", "linear_bwd"):
        m, k, n = c["rows"], c["k"], c["n"]
        o = max(b, 2)
        if kind == "linear_fwd":
            return {"bytes": b * k * (m + n) + o * m * n * (1 + c["mul"] + c["residual"] + c["z"]) + o * n * c["bias"] + (4 * (m + n) if b == 1 else 0),
                    "flops": 2 * m * n * k}
        kept = c["act"] != "none" or c["mul"]
        return {"bytes": 2 * b * k * (m + n) + b * m * n * (1 + kept + 2 * c["mul"]) + b * n * c["bias"], "flops": 4 * m * n * k}
    if kind == "axes_rows":
        return {"bytes": 2 * c["rows"] * c["heads"] * c["d"] * b + 12 * c["rows"], "flops": 3 * c["rows"] * c["heads"] * c["rotary"]}
    rows = sum(forest_of(c)[1])
    return {"bytes": 2 * rows * (c["hq"] + 2 * c["hkv"]) * c["d"] * b + 16 * rows, "flops": 3 * rows * (c["hq"] + c["hkv"]) * c["rotary"]}


# ------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "rms_fwd":
        h = s["x"] if s["residual"] is None else (s["x"].double() + s["residual"].double()).to(s["x"].dtype)
        y = h.double() / torch.sqrt(torch.linalg.vector_norm(h.double(), dim=-1, keepdim=True) ** 2 / case["dim"] + EPS) * s["weight"].double()
        scale = torch.clamp(torch.linalg.vector_norm(y, ord=math.inf, dim=-1) / 448, min=2.0 ** -126)
        codes = (y / scale[..., None]).float().to(E4M3).double()
        out = case["out"]
        return {"y": y if out != "codes" else None, "summed": None if s["residual"] is None else h.double(),
                "codes": codes if out != "y" else None, "scales": scale if out != "y" else None}
    if kind == "rms_bwd":
        h, w, dy = (s[n].double() for n in ("x", "weight", "d_y"))
        ms = torch.einsum("...d,...d->...", h, h) / case["dim"] + EPS
        along = torch.einsum("...d,...d,d->...", h, dy, w) / case["dim"]
        dx = dy * w / ms[..., None] ** 0.5 - h * (along / ms ** 1.5)[..., None]
        if s["d_summed"] is not None:
            dx += s["d_summed"].double()
        return dx, torch.einsum("nd,nd,n->d", dy.flatten(0, -2), h.flatten(0, -2), ms.flatten() ** -0.5)
    if kind.startswith("linear"):
        x, w = s["x"].double(), s["weight"].double()
        act = case["act"]

        def curve(z):
            if act == "relu":
                return torch.clamp(z, min=0), torch.where(z > 0, 1.0, 0.0)
            if act == "silu":
                e = torch.special.expit(z)
                return z * e, e + z * e * (1 - e)
            if act == "gelu":
                e = torch.special.ndtr(z)
                return z * e, e + z * torch.exp(-z * z / 2) * 0.3989422804014327
            if act == "gelu_tanh":
                u = 1.5957691216057308 * (z + 0.044715 * z ** 3)   # 1 + tanh(u / 2) = 2 expit(u)
                e = torch.special.expit(u)
                return z * e, e + z * e * (1 - e) * 1.5957691216057308 * (1 + 0.134145 * z * z)
            return z, torch.ones_like(z)

        if kind == "linear_fwd":
            if "x_scale" in s:
                x, w = x * s["x_scale"].double()[:, None], w * s["weight_scale"].double()[:, None]
            z = torch.nn.functional.linear(x, w, None if s["bias"] is None else s["bias"].double())
            y = curve(z)[0]
            y = y if s["mul"] is None else y * s["mul"].double()
            y = y if s["residual"] is None else y + s["residual"].double()
            return y, z if case["z"] else None
        dy, d_mul = s["d_y"].double(), None
        if s["z"] is not None:
            a, slope = curve(s["z"].double())
            if s["mul"] is not None:
                d_mul, dy = dy * a, dy * s["mul"].double()
            dy = dy * slope
        return torch.einsum("mn,nk->mk", dy, w), torch.einsum("mn,mk->nk", dy, x), torch.einsum("mn->n", dy) if case["bias"] else None, d_mul
    r, sign = case["rotary"], -1.0 if kind == "axes_bwd" or case.get("inverse") else 1.0
    first, step = (r // 2, 1) if case["layout"] == "half" else (1, 2)
    counts = [int(x) for x in case["sections"].split(",")]
    if case["order"] == "blocks":
        axis = np.repeat(np.arange(3), counts)
    else:   # axis 0 everywhere but at every third pair from 1 on and from 2 on
        axis = np.zeros(r // 2, dtype=np.int64)
        for a in (1, 2):
            axis[a:3 * counts[a]:3] = a

    def turn(x):
        y, p = x.double(), s["positions"].double()
        at = torch.arange(r // 2, device="cuda") * step
        theta = torch.stack([p[int(a)] * case["base"] ** (-2.0 * i / r) for i, a in enumerate(axis)], 1) * sign
        z = torch.complex(y[..., at], y[..., at + first]) * torch.polar(torch.ones_like(theta), theta)[:, None]
        y[..., at], y[..., at + first] = z.real, z.imag
        return y

    if kind == "axes_rows":
        return turn(s["x"])
    if kind == "axes_bwd":
        return turn(s["q"]), turn(s["k_pool"].transpose(0, 1)[s["slot"]]), s["v_pool"].transpose(0, 1)[s["slot"]].double()
    k, v = s["k_pool"].double(), s["v_pool"].double()
    k.transpose(0, 1)[s["slot"]] = turn(s["k"])
    v.transpose(0, 1)[s["slot"]] = s["v"].double()
    return turn(s["q"]), k, v
