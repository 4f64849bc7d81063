"""The operators around the tree attention of a training step, in plain form and through the library.

  rope_fwd, rope_bwd   rotary positions of the tree's query rows: Q rotated row by row, K rotated on its way into the
                       paged pool, V copied beside it; and the way back, the inverse rotation of dQ and of the
                       gradient pool's dK
  rope_rows            the same rotation of a few rows at positions of their own (one token per sequence)
  kv_copy              blocks of the K/V pools copied to other pools (offload of evicted blocks, restoring them)
  kv_move              blocks of the K/V pools moved down in place (compaction of the arena)
  logprob_fwd          log-probabilities of target tokens under softmax(scale * hidden weight^T) over a large
                       vocabulary; a row may have no target, one, or several (the children of a branching point)
  logprob_bwd          gradients of hidden and weight
"""
import math
import random

import numpy as np
import torch

own = False


# ---------------------------------------------------------------------------------------------------- the cases

def rope_case(kind, name=None, groups=1, prefix=0, branches=0, lo=1, hi=1, cached=False, block=64, hq=32, hkv=8, d=128,
              dtype="bf16", layout="half", rotary=128, base=10000.0, scaling="none", factor=1.0, original=0, forest=1):
    c = dict(kind=kind, groups=groups, prefix=prefix, branches=branches, lo=lo, hi=hi, cached=cached, block=block,
             hq=hq, hkv=hkv, d=d, dtype=dtype, layout=layout, rotary=rotary, base=base, scaling=scaling, factor=factor,
             original=original, forest=forest)
    return dict(c, name=name) if name else c


def listed():
    return [
        # step-wise group: one 4096-token prefix and 8 branches of 256..1024 tokens, the projections' rows into the pools
        rope_case("rope_fwd", "rope_fwd_group", prefix=4096, branches=8, lo=256, hi=1024),
        # long agentic group: 32768-token prefix, 64 branches of 1024..4096, gradients on their way back
        rope_case("rope_bwd", "rope_bwd_long", prefix=32768, branches=64, lo=1024, hi=4096, block=256, hq=64, hkv=8,
                  base=1000000.0, scaling="yarn", factor=4.0, original=32768),
        # fp32, half of a 64-wide head rotated, neighbouring elements paired; several groups, 16-slot blocks
        rope_case("rope_fwd", "rope_fwd_f32_part", groups=5, prefix=777, branches=7, lo=33, hi=301, block=16, hq=8, hkv=8,
                  d=64, dtype="f32", layout="interleaved", rotary=32, scaling="linear", factor=2.0, original=2048),
        # rollout: one new token for each of 8 sequences, far positions
        dict(name="rope_rows_decode", kind="rope_rows", rows=8, heads=40, d=128, dtype="bf16", layout="half", rotary=128,
             base=500000.0, scaling="banded", factor=8.0, original=8192, far=131072, inverse=False),
        # a micro-batch evicts some hundred blocks of a mixed arena to a spill buffer
        dict(name="kv_copy_evict", kind="kv_copy", extents=300, lo=16, hi=2048, hkv=8, d=128, dtype="bf16", forest=3),
        # three short branches are restored
        dict(name="kv_copy_small", kind="kv_copy", extents=3, lo=16, hi=48, hkv=8, d=128, dtype="bf16", forest=4),
        # an arena of some 200,000 slots is compacted after a tenth of its blocks was freed
        dict(name="kv_move_arena", kind="kv_move", extents=150, lo=64, hi=4096, hole=0.1, hkv=8, d=128, dtype="bf16", forest=5),
        # a small arena, overlapping moves by one block
        dict(name="kv_move_small", kind="kv_move", extents=12, lo=16, hi=160, hole=0.2, hkv=2, d=64, dtype="f32", forest=6),
        # the policy's log-probabilities of one step-wise group (reference model, old policy: forward only)
        dict(name="logprob_fwd_group", kind="logprob_fwd", rows=8192, hidden=4096, vocab=131072, scale=1.0, masked=0.3, fan=8),
        # one row: the next token of a rollout
        dict(name="logprob_fwd_token", kind="logprob_fwd", rows=1, hidden=4096, vocab=131072, scale=0.7, masked=0.0, fan=1),
        # the update of a share of that group
        dict(name="logprob_bwd_group", kind="logprob_bwd", rows=4096, hidden=4096, vocab=131072, scale=1.0, masked=0.3, fan=8),
        # a short odd micro-batch over an odd vocabulary
        dict(name="logprob_bwd_odd", kind="logprob_bwd", rows=777, hidden=3584, vocab=50257, scale=1.0, masked=0.5, fan=4),
    ]


def spread(rng, lo, hi):
    """A whole number of lo..hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope_fwd", "rope_bwd", "rope_rows", "kv_copy", "kv_move", "logprob_fwd", "logprob_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    scaling = rng.choice(["none", "none", "linear", "ntk", "yarn", "banded"])
    rope = dict(base=rng.choice([10000.0, 500000.0, 1000000.0]), scaling=scaling,
                factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]),
                original=0 if scaling == "none" else rng.choice([2048, 8192, 32768]), layout=rng.choice(["half", "interleaved"]))
    if kind in ("rope_fwd", "rope_bwd"):
        d = 128 if dtype == "bf16" else rng.choice([64, 128])
        hkv = rng.choice([1, 2, 4, 8])
        return rope_case(kind, groups=rng.choice([1, 1, 2, 5]), prefix=spread(rng, 1, 8192), branches=spread(rng, 1, 24),
                         lo=1, hi=spread(rng, 2, 1024), cached=rng.random() < 0.3, block=rng.choice([16, 64, 256]),
                         hq=hkv * rng.choice([1, 3, 4, 7]), hkv=hkv, d=d, dtype=dtype,
                         rotary=rng.choice([d, d, d // 2, d // 4]), forest=rng.randrange(1 << 20), **rope)
    if kind == "rope_rows":
        d = rng.choice([64, 128])
        return dict(kind=kind, rows=spread(rng, 1, 5000), heads=rng.choice([1, 5, 8, 40, 72]), d=d, dtype=dtype,
                    rotary=rng.choice([d, d // 2]), far=spread(rng, 2, 1000000), inverse=rng.random() < 0.5, **rope)
    if kind in ("kv_copy", "kv_move"):
        c = dict(kind=kind, extents=spread(rng, 1, 250), lo=rng.choice([16, 64]), hi=spread(rng, 64, 2048),
                 hkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128]), dtype=dtype, forest=rng.randrange(1 << 20))
        return dict(c, hole=rng.choice([0.05, 0.2, 0.5])) if kind == "kv_move" else c
    backward = kind == "logprob_bwd"
    return dict(kind=kind, rows=spread(rng, 1, 1500 if backward else 3000), hidden=rng.choice([512, 1024, 2048, 2568, 3584, 4096]),
                vocab=spread(rng, 1000, 131072), scale=rng.choice([1.0, 1.0, 0.7, 0.125]), masked=rng.choice([0.0, 0.3, 0.6]),
                fan=rng.choice([1, 4, 16]))


TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


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


def rope_rows_of(c):
    """Per query row its position in the sequence and its slot, and the number of slots: blocks of whole pages, one segment
    after the other. The rows of a cached prefix are not computed here: its keys are in the pool already."""
    parent, length = forest_of(c)
    at, pos, slot = 0, [], []
    for p, n in zip(parent, length):
        if p >= 0 or not c["cached"]:
            first = 0 if p < 0 else length[p]
            pos.append(np.arange(first, first + n))
            slot.append(np.arange(at, at + n))
        at += -(-n // c["block"]) * c["block"]
    return np.concatenate(pos), np.concatenate(slot), at


def extents_of(c):
    """[n, 3] (source slot, destination slot, slots) and the number of slots of the source and of the destination."""
    r = random.Random(c["forest"])
    sizes = [-(-spread(r, c["lo"], c["hi"]) // 16) * 16 for _ in range(c["extents"])]
    ext, at = [], 0
    if c["kind"] == "kv_move":
        to = at = 16  # the first block stays
        for n in sizes:
            at += 16 * max(0, int(round(n * 2 * r.random() * c["hole"] / 16))) + (16 if to == at else 0)
            ext.append((at, to, n))
            at, to = at + n, to + n
        return np.array(ext, dtype=np.int32), at, at
    for n in sizes:
        at += 16 * r.randint(0, 4)
        ext.append([at, 0, n])
        at += n
    r.shuffle(ext)
    to = 0
    for e in ext:
        e[1] = to
        to += e[2]
    return np.array(ext, dtype=np.int32), at, to


def prepare(case, seed):
    c, kind = case, case["kind"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    s = {"case": c}
    if kind in ("rope_fwd", "rope_bwd"):
        t, d = TYPES[c["dtype"]], c["d"]
        pos, slot, slots = rope_rows_of(c)
        s["pos"], s["slot"] = (torch.from_numpy(x).cuda() for x in (pos, slot))
        s["q"] = rnd(len(pos), c["hq"], d).to(t)
        s["k_pool"], s["v_pool"] = rnd(c["hkv"], slots, d).to(t), rnd(c["hkv"], slots, d).to(t)
        s["q_out"] = torch.empty_like(s["q"])
        s["k"], s["v"] = rnd(len(pos), c["hkv"], d).to(t), rnd(len(pos), c["hkv"], d).to(t)
        if own:
            from paper_2608_25683_b200 import binding
            parent, length = forest_of(c)
            flags = [(0 if p < 0 and c["cached"] else 1) | (2 if p >= 0 else 0) for p in parent]
            s["plan"] = binding.Plan(parent, length, [c["block"]] * c["groups"], c["hq"], c["hkv"], d, c["dtype"], flags).upload()
            s["rope"] = rope_handle(binding, c)
    elif kind == "rope_rows":
        s["x"] = rnd(c["rows"], c["heads"], c["d"]).to(TYPES[c["dtype"]])
        s["positions"] = torch.randint(0, c["far"], (c["rows"],), generator=g, device="cuda", dtype=torch.int32)
        s["y"] = torch.empty_like(s["x"])
        if own:
            from paper_2608_25683_b200 import binding
            s["rope"] = rope_handle(binding, c)
    elif kind in ("kv_copy", "kv_move"):
        s["extents"], n_src, n_dst = extents_of(c)
        s["src"], s["dst"] = (torch.from_numpy(np.concatenate([np.arange(e[i], e[i] + e[2]) for e in s["extents"]])).cuda() for i in (0, 1))
        t = TYPES[c["dtype"]]
        s["k_src"], s["v_src"] = (rnd(c["hkv"], n_src, c["d"]).to(t) for _ in range(2))
        if kind == "kv_copy":
            s["k_dst"], s["v_dst"] = (torch.zeros(c["hkv"], n_dst, c["d"], dtype=t, device="cuda") for _ in range(2))
    else:
        n, h, v = c["rows"], c["hidden"], c["vocab"]
        s["weight"] = (rnd(v, h) * 0.02).to(torch.bfloat16)
        likely = torch.randint(0, v, (n,), generator=g, device="cuda")
        some = torch.rand(n, 1, generator=g, device="cuda") * 10.0 * 4096 / h
        s["hidden"] = (rnd(n, h) + some * s["weight"][likely].float()).to(torch.bfloat16)
        # rows without a target (prompts, ends of samples), rows with one, and branching points with `fan` of them
        kinds = np.random.RandomState(n).rand(n)
        count = np.where(kinds < c["masked"], 0, np.where(kinds > 0.999, c["fan"], 1))
        count[0] = c["fan"]
        count = torch.from_numpy(count).cuda()
        s["target_off"] = torch.nn.functional.pad(count.cumsum(0), (1, 0)).to(torch.int32)
        row = torch.repeat_interleave(torch.arange(n, device="cuda"), count)
        target = torch.where(torch.rand(len(row), generator=g, device="cuda") < 0.7, likely[row],
                             torch.randint(0, v, (len(row),), generator=g, device="cuda"))
        s["targets"] = torch.where(torch.rand(len(row), generator=g, device="cuda") < 0.02, -1, target).to(torch.int32)
        if kind == "logprob_bwd":
            s["logprob"], s["lse"] = plain_logprob(s)
            s["d_logprob"] = rnd(len(row)) * (torch.rand(len(row), generator=g, device="cuda") < 0.9)
    return s


def rope_handle(binding, c):
    return binding.Rope(c["d"], rotary_dim=c["rotary"], base=c["base"], layout=c["layout"], scaling=c["scaling"],
                        factor=c["factor"], original_positions=c["original"])


# ------------------------------------------------------------------------------------------------- one pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        from paper_2608_25683_b200 import binding as b
        if kind == "rope_fwd":
            q = b.psrl_rope_qkv_fwd(s["plan"], s["rope"], s["q"], s["k"], s["v"], s["k_pool"], s["v_pool"], q_out=s["q_out"])
            return q, s["k_pool"], s["v_pool"]
        if kind == "rope_bwd":
            return b.psrl_rope_qkv_bwd(s["plan"], s["rope"], s["q"], s["k_pool"], s["v_pool"], dq_out=s["q_out"], dk_out=s["k"],
                                       dv_out=s["v"])
        if kind == "rope_rows":
            return b.psrl_rope_rows(s["rope"], s["x"], s["positions"], y=s["y"], inverse=s["case"]["inverse"])
        if kind == "kv_copy":
            b.psrl_kv_copy(s["extents"], s["k_src"], s["v_src"], s["k_dst"], s["v_dst"])
            return s["k_dst"], s["v_dst"]
        if kind == "kv_move":
            b.psrl_kv_move(s["extents"], s["k_src"], s["v_src"])
            return s["k_src"], s["v_src"]
        if kind == "logprob_fwd":
            return b.psrl_token_logprob_fwd(s["hidden"], s["weight"], s["targets"], s["target_off"], scale=s["case"]["scale"])
        return b.psrl_token_logprob_bwd(s["hidden"], s["weight"], s["targets"], s["logprob"], s["lse"], s["d_logprob"],
                                        s["target_off"], scale=s["case"]["scale"])
    if kind == "rope_fwd":
        s["k_pool"][:, s["slot"]] = plain_rotate(s["k"], s["pos"], s["case"], False).transpose(0, 1)
        s["v_pool"][:, s["slot"]] = s["v"].transpose(0, 1)
        return plain_rotate(s["q"], s["pos"], s["case"], False), s["k_pool"], s["v_pool"]
    if kind == "rope_bwd":
        dk = plain_rotate(s["k_pool"][:, s["slot"]].transpose(0, 1), s["pos"], s["case"], True)
        return plain_rotate(s["q"], s["pos"], s["case"], True), dk, s["v_pool"][:, s["slot"]].transpose(0, 1).contiguous()
    if kind == "rope_rows":
        return plain_rotate(s["x"], s["positions"], s["case"], s["case"]["inverse"])
    if kind == "kv_copy":
        s["k_dst"][:, s["dst"]] = s["k_src"][:, s["src"]]
        s["v_dst"][:, s["dst"]] = s["v_src"][:, s["src"]]
        return s["k_dst"], s["v_dst"]
    if kind == "kv_move":
        s["k_src"][:, s["dst"]] = s["k_src"][:, s["src"]]
        s["v_src"][:, s["dst"]] = s["v_src"][:, s["src"]]
        return s["k_src"], s["v_src"]
    return plain_logprob(s) if kind == "logprob_fwd" else plain_logprob_bwd(s)


# ------------------------------------------------------------------------------------------------- plain forms

def frequencies(c):
    """Radians per position of each pair of elements, and the factor on cos and sin, in 64 bits."""
    r, base, f = c["rotary"], c["base"], c["factor"]
    i = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    if c["scaling"] == "ntk":
        base = base * f ** (r / (r - 2.0))
    freq = base ** (-2.0 * i / r)
    if c["scaling"] == "linear":
        return freq / f, 1.0
    if c["scaling"] == "yarn":
        # pairs that turn more than 32 times over the original length stay, those below one turn are stretched
        edge = lambda turns: r * math.log(c["original"] / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(edge(32.0)), 0), min(math.ceil(edge(1.0)), r - 1)
        keep = 1.0 - ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return freq * keep + freq / f * (1.0 - keep), 0.1 * math.log(f) + 1.0
    if c["scaling"] == "banded":
        # by wavelength: below original / 4 as they are, above original stretched, between them a mix
        turns = c["original"] * freq / (2 * math.pi)
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        return freq * keep + freq / f * (1.0 - keep), 1.0
    return freq, 1.0


def plain_rotate(x, pos, c, inverse):
    freq, scale = frequencies(c)
    angle = pos.double()[:, None] * freq[None, :]
    cos, sin = (angle.cos() * scale).float()[:, None], (angle.sin() * scale).float()[:, None]
    sin = -sin if inverse else sin
    r, f = c["rotary"], x.float()
    if c["layout"] == "half":
        a, b = f[..., : r // 2], f[..., r // 2 : r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = f[..., 0:r:2], f[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([turned.to(x.dtype), x[..., r:]], dim=-1)


def pairs(s):
    """Row and target of every (row, target) pair, and which of them count."""
    off = s["target_off"].long()
    row = torch.repeat_interleave(torch.arange(len(off) - 1, device="cuda"), off[1:] - off[:-1], output_size=len(s["targets"]))
    t = s["targets"].long()
    return row, t.clamp(min=0), t >= 0


def plain_logprob(s):
    z = s["hidden"].float() @ s["weight"].float().T * s["case"]["scale"]
    top = z.amax(1, keepdim=True)
    lse = top[:, 0] + (z - top).exp().sum(1).log()
    row, t, on = pairs(s)
    return torch.where(on, z[row, t] - lse[row], 0.0), lse


def plain_logprob_bwd(s):
    h, w = s["hidden"].float(), s["weight"].float()
    row, t, on = pairs(s)
    grad = torch.where(on, s["d_logprob"], 0.0)
    total = torch.zeros(len(h), device="cuda").index_add_(0, row, grad)
    dz = (h @ w.T * s["case"]["scale"] - s["lse"][:, None]).exp() * -total[:, None]
    dz.view(-1).index_add_(0, row * w.shape[0] + t, grad)
    dz *= s["case"]["scale"]
    return (dz @ w).to(torch.bfloat16), (dz.T @ h).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------- the work of one pass

def work(case):
    c, kind = case, case["kind"]
    if kind in ("rope_fwd", "rope_bwd"):
        rows, b = len(rope_rows_of(c)[0]), 2 if c["dtype"] == "bf16" else 4
        return {"bytes": 2 * rows * (c["hq"] + 2 * c["hkv"]) * c["d"] * b + 8 * rows, "flops": 3 * rows * (c["hq"] + c["hkv"]) * c["rotary"]}
    if kind == "rope_rows":
        b = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": 2 * c["rows"] * c["heads"] * c["d"] * b + 4 * c["rows"], "flops": 3 * c["rows"] * c["heads"] * c["rotary"]}
    if kind in ("kv_copy", "kv_move"):
        slots = int(extents_of(c)[0][:, 2].sum())
        return {"bytes": 4 * slots * c["hkv"] * c["d"] * (2 if c["dtype"] == "bf16" else 4), "flops": 0}
    n, h, v = c["rows"], c["hidden"], c["vocab"]
    if kind == "logprob_fwd":
        return {"bytes": 2 * h * (n + v) + 16 * n, "flops": 2 * n * h * v}
    return {"bytes": 4 * h * (n + v) + 20 * n, "flops": 6 * n * h * v}


# ------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind in ("kv_copy", "kv_move"):
        to = ("k_dst", "v_dst") if kind == "kv_copy" else ("k_src", "v_src")
        old = (s["k_src"].clone(), s["v_src"].clone())
        for e in s["extents"].tolist():
            for i in (0, 1):
                s[to[i]][:, e[1]:e[1] + e[2]] = old[i][:, e[0]:e[0] + e[2]]
        return s[to[0]].double(), s[to[1]].double()
    if kind.startswith("rope"):
        freq, scale = frequencies(case)
        r, sign = case["rotary"], -1.0 if kind == "rope_bwd" or case.get("inverse") else 1.0
        first, step = (r // 2, 1) if case["layout"] == "half" else (1, 2)

        def turn(x, pos):
            y = x.double()
            unit = torch.polar(torch.full((len(pos), r // 2), scale, dtype=torch.float64, device="cuda"), sign * torch.outer(pos.double(), freq))
            at = torch.arange(r // 2, device="cuda") * step
            z = torch.complex(y[..., at], y[..., at + first]) * unit[:, None]
            y[..., at], y[..., at + first] = z.real, z.imag
            return y

        if kind == "rope_rows":
            return turn(s["x"], s["positions"])
        if kind == "rope_bwd":
            return (turn(s["q"], s["pos"]), turn(s["k_pool"].transpose(0, 1)[s["slot"]], s["pos"]),
                    s["v_pool"].transpose(0, 1)[s["slot"]].double())
        k, v = s["k_pool"].double(), s["v_pool"].double()
        k.transpose(0, 1)[s["slot"]] = turn(s["k"], s["pos"])
        v.transpose(0, 1)[s["slot"]] = s["v"].double()
        return turn(s["q"], s["pos"]), k, v
    # rows in parts: the logits of all rows in 64 bits are large
    w, off, targets = s["weight"].double(), s["target_off"].tolist(), s["targets"].long()
    logprob, lse, dh = [], [], []
    dw = torch.zeros_like(w) if kind == "logprob_bwd" else None
    for a in range(0, len(s["hidden"]), 2048):
        h = s["hidden"][a:a + 2048].double()
        z = case["scale"] * (h @ w.T)
        l = torch.logsumexp(z, 1)
        b = min(a + 2048, len(s["hidden"]))
        mine = slice(off[a], off[b])
        t = targets[mine]
        row = torch.repeat_interleave(torch.arange(b - a), torch.tensor([off[i + 1] - off[i] for i in range(a, b)])).cuda()
        keep = t >= 0
        if dw is None:
            logprob.append((z[row, t.clamp(min=0)] - l[row]) * keep)
            lse.append(l)
            continue
        grad = s["d_logprob"][mine].double() * keep
        total = torch.zeros(b - a, dtype=torch.float64, device="cuda").index_add_(0, row, grad)
        dz = -total[:, None] * torch.softmax(z, 1)
        dz.index_put_((row, t.clamp(min=0)), grad, accumulate=True)
        dz *= case["scale"]
        dh.append(dz @ w)
        dw += dz.T @ h
    return (torch.cat(logprob), torch.cat(lse)) if dw is None else (torch.cat(dh), dw)
