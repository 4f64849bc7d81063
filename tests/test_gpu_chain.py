"""The operators together, as an update step uses them: projections' rows -> rotary positions and pools -> tree attention
-> log-probabilities of the next tokens -> their gradients -> attention backward -> inverse rotation; in one call each, and
over micro-batches with blocks evicted, restored and compacted in between.

The reference computes every sample on its own in fp64 (torch autograd): rotary positions, causal attention, softmax over the
vocabulary, and sums loss and gradients over the samples, each with an advantage of its own.

Tolerance: between a bf16 input and a gradient lie at most ten roundings to bf16 (rotated q and k, P, o; dz, d_hidden, P and dS
in the backward, the attention's gradient, the rotated gradient), each off by at most half a step, 2^-8 of the values: 10 x 2^-8
in the 2-norm; on the log-probabilities the first four, times the spread of the logits around their mean."""
import numpy as np
import pytest
import torch

from oracle import oracle_plan, sample_paths
from oracle.rope import oracle_rope_frequencies
from paper_2608_25683_b200.workloads import Workload

from util import build_plan, to_np

pytestmark = pytest.mark.gpu
Hq, Hkv, D, VOCAB = 4, 2, 128, 701
ROPE = dict(base=10000.0, scaling="yarn", factor=4.0, original_positions=64)
SCALE = 1.0 / np.sqrt(D)


def reference(V, q, k, v, weight, ids, advantage):
    """Per tree token (canonical order): loss of every transition, gradients of q, k, v [T, H, D] and of weight."""
    q, k, v, weight = (t.double().cpu().requires_grad_(True) for t in (q, k, v, weight))
    freq, scale = oracle_rope_frequencies(D, **ROPE)
    loss, logprob = 0.0, {}
    for path, a in zip(sample_paths(V), advantage):
        tok = [t for c in path for t in range(V["seg_tok_off"][c], V["seg_tok_off"][c] + V["seg_len"][c])]
        angle = torch.outer(torch.arange(len(tok), dtype=torch.float64), torch.as_tensor(freq))[:, None]
        cos, sin = angle.cos() * scale, angle.sin() * scale
        turn = lambda x: torch.cat([x[..., :D // 2] * cos - x[..., D // 2:] * sin, x[..., D // 2:] * cos + x[..., :D // 2] * sin], -1)
        qs, ks, vs = turn(q[tok]), turn(k[tok]), v[tok]
        ks, vs = (x.repeat_interleave(Hq // Hkv, 1) for x in (ks, vs))
        s = torch.einsum("ihd,jhd->hij", qs, ks) * SCALE
        s = s.masked_fill(torch.ones(len(tok), len(tok), dtype=torch.bool).triu(1), float("-inf"))
        o = torch.einsum("hij,jhd->ihd", s.softmax(-1), vs).reshape(len(tok), Hq * D)
        lp = torch.log_softmax(o[:-1] @ weight.T, -1)[torch.arange(len(tok) - 1), ids[tok[1:]]]
        loss = loss + a * lp.sum()
        logprob.update({(x, y): float(l) for x, y, l in zip(tok, tok[1:], lp.detach())})
    loss.backward()
    return logprob, q.grad, k.grad, v.grad, weight.grad


def transitions(V, advantage):
    """{(token, next token): summed advantage of the samples that make the step}"""
    w = {}
    for path, a in zip(sample_paths(V), advantage):
        tok = [t for c in path for t in range(V["seg_tok_off"][c], V["seg_tok_off"][c] + V["seg_len"][c])]
        for x in zip(tok, tok[1:]):
            w[x] = w.get(x, 0.0) + a
    return w


def draw(T, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = rnd(T, Hq + 2 * Hkv, D).to(torch.bfloat16)
    weight = (rnd(VOCAB, Hq * D) * 0.2).to(torch.bfloat16)
    ids = torch.randint(0, VOCAB, (T,), generator=g, device="cuda")
    return x, weight, ids


def close(got, want, name):
    rel = float((got.double().cpu() - want).norm() / want.norm())
    assert rel <= 10 * 2.0 ** -8, (name, rel)


FOREST = dict(parent=[-1, 0, 0, 2, 2, -1, 5, 5], seg_len=[130, 33, 70, 1, 45, 64, 17, 129], gbs=[64, 16])


def test_one_update_step(lib):
    w = Workload("u", FOREST["parent"], FOREST["seg_len"], FOREST["gbs"], Hq, Hkv, D, "bf16")
    plan = build_plan(lib, w)
    V = plan.oracle
    x, weight, ids = draw(V["T"], 1)
    advantage = np.random.default_rng(0).normal(size=V["n_samples"])
    want_lp, *want = reference(V, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], weight, ids.cpu(), advantage)
    weights = transitions(V, advantage)

    rope = lib.Rope(D, **ROPE)
    pools = [torch.full((Hkv, V["pool_slots"], D), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    q = lib.psrl_rope_qkv_fwd(plan, rope, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], *pools)
    o, lse = lib.psrl_tree_attn_fwd(plan, q, *pools, SCALE)
    off, nxt = plan.next_tokens()
    off_d, targets = torch.as_tensor(off, device="cuda"), ids[torch.as_tensor(nxt, device="cuda").long()].to(torch.int32)
    hidden = o.view(V["T_q"], Hq * D)
    lp, z_lse = lib.psrl_token_logprob_fwd(hidden, weight, targets, off_d)
    row = np.repeat(np.arange(V["T_q"]), np.diff(off))       # every segment has queries: row r is token r
    grad = torch.as_tensor([weights[(int(r), int(t))] for r, t in zip(row, nxt)], dtype=torch.float32, device="cuda")
    ref_lp = np.array([want_lp[(int(r), int(t))] for r, t in zip(row, nxt)])
    spread = float((hidden.double() @ weight.double().T).std(1).max())
    assert np.abs(to_np(lp) - ref_lp).max() <= 4 * 2.0 ** -8 * 4 * spread    # four roundings; a logit is within 4 deviations
    dh, dw = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, z_lse, grad, off_d)
    dq, dkp, dvp = lib.psrl_tree_attn_bwd(plan, q, *pools, o, lse, dh.view_as(o), SCALE)
    out = torch.empty_like(x)
    lib.psrl_rope_qkv_bwd(plan, rope, dq, dkp, dvp, dq_out=out[:, :Hq], dk_out=out[:, Hq:Hq + Hkv], dv_out=out[:, Hq + Hkv:])
    assert lib.psrl_device_status(plan, "bwd") == 0
    for got, ref, name in zip((out[:, :Hq], out[:, Hq:Hq + Hkv], out[:, Hq + Hkv:], dw), want, ("dq", "dk", "dv", "dw")):
        close(got, ref, name)


def test_micro_batches_with_blocks_on_the_move(lib):
    """The same forest over four micro-batches in an arena too small for all of it: prefixes are read in place with their keys
    rotated, evicted blocks go to a spill pool and come back, the arena is compacted after every micro-batch (gradient sums in
    the same layout move along), and the prefixes' K gradients are rotated back once, at the end."""
    parent, seg_len, gbs = FOREST["parent"], FOREST["seg_len"], FOREST["gbs"]
    mb, M, cap = [0, 2, 0, 3, 2, 1, 3, 1], 4, 496
    V = oracle_plan(parent, seg_len, gbs)
    x, weight, ids = draw(V["T"], 2)
    advantage = np.random.default_rng(1).normal(size=V["n_samples"])
    _, *want = reference(V, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], weight, ids.cpu(), advantage)
    weights = transitions(V, advantage)
    after = {}
    for (a, b), g in weights.items():
        after.setdefault(a, []).append((b, g))
    tokens = [np.arange(V["seg_tok_off"][c], V["seg_tok_off"][c] + V["seg_len"][c]) for c in V["canon_of_input"]]
    block = [64] * 5 + [16] * 3
    extent = [-(-n // b) * b for n, b in zip(seg_len, block)]

    rope, cache = lib.Rope(D, **ROPE), lib.Cache(parent, seg_len, gbs, mb, M, capacity_slots=cap)
    pool = lambda t=torch.bfloat16, fill=float("nan"), n=cap: torch.full((Hkv, n, D), fill, device="cuda", dtype=t)
    K, P = pool(), pool()
    acc = pool(torch.float32, 0.0), pool(torch.float32, 0.0)
    spill, spilled, seen = (pool(n=2048), pool(n=2048)), {}, dict(evict=0, reload=0, move=0)
    spill_acc = pool(torch.float32, 0.0, 2048), pool(torch.float32, 0.0, 2048)
    got_q = torch.zeros(V["T"], Hq, D, device="cuda", dtype=torch.float64)
    got_k, got_v = (torch.zeros(V["T"], Hkv, D, device="cuda", dtype=torch.float32) for _ in range(2))
    got_w = torch.zeros(VOCAB, Hq * D, device="cuda", dtype=torch.float64)
    base = {}

    def collect(s):
        """The finished gradient sums of a segment, token-major; its slots start again at zero."""
        t = torch.as_tensor(tokens[s], device="cuda")
        for pool_, to in zip(acc, (got_k, got_v)):
            to[t] = pool_[:, base[s]:base[s] + seg_len[s]].transpose(0, 1)
            pool_[:, base[s]:base[s] + extent[s]] = 0

    for m in range(M):
        step = cache.begin(m)
        if step["evict"]:
            e = [[old, s * 256, extent[s]] for s, old in step["evict"]]
            lib.psrl_kv_copy(e, K, P, *spill)
            lib.psrl_kv_copy(e, *acc, *spill_acc)
            for s, old in step["evict"]:
                K[:, old:old + extent[s]] = float("nan")
                for a in acc:
                    a[:, old:old + extent[s]] = 0
                spilled[s] = True
        base = dict(zip(step["seg_id"], step["seg_slot_base"]))
        if step["reload"]:
            e = [[s * 256, base[s], extent[s]] for s in step["reload"]]
            lib.psrl_kv_copy(e, *spill, K, P)
            lib.psrl_kv_copy(e, *spill_acc, *acc)
        seen["evict"] += len(step["evict"])
        seen["reload"] += len(step["reload"])
        plan = lib.Plan(step["parent"], step["seg_len"], step["group_block_size"], Hq, Hkv, D, "bf16", seg_flags=step["seg_flags"],
                        seg_slot_base=step["seg_slot_base"]).upload()
        PV = plan.view
        rows = np.concatenate([tokens[step["seg_id"][PV["input_of_canon"][c]]] for c in range(PV["n_seg"]) if PV["seg_q_off"][c] >= 0])
        xm = x[torch.as_tensor(rows, device="cuda")]
        q = lib.psrl_rope_qkv_fwd(plan, rope, xm[:, :Hq], xm[:, Hq:Hq + Hkv], xm[:, Hq + Hkv:], K, P)
        o, lse = lib.psrl_tree_attn_fwd(plan, q, K, P, SCALE)
        # the rows' next tokens: the plan's own, and those that later micro-batches bring
        pairs = [after.get(int(t), []) for t in rows]
        off = torch.as_tensor(np.concatenate([[0], np.cumsum([len(p) for p in pairs])]).astype(np.int32), device="cuda")
        flat = [y for p in pairs for y in p]
        listed = {(int(rows[r]), int(b)) for r in range(len(rows)) for b, _ in pairs[r]}
        toff, tnext = plan.next_tokens()
        tok_of = np.concatenate([tokens[step["seg_id"][PV["input_of_canon"][c]]] for c in range(PV["n_seg"])])
        assert {(int(rows[r]), int(tok_of[t])) for r in range(len(rows)) for t in tnext[toff[r]:toff[r + 1]]} <= listed
        targets = ids[torch.as_tensor([b for b, _ in flat], device="cuda")].to(torch.int32)
        grad = torch.as_tensor([g for _, g in flat], dtype=torch.float32, device="cuda")
        hidden = o.view(len(rows), Hq * D)
        lp, z_lse = lib.psrl_token_logprob_fwd(hidden, weight, targets, off)
        dh, dw = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, z_lse, grad, off)
        got_w += dw.double()
        dq, dkp, dvp = lib.psrl_tree_attn_bwd(plan, q, K, P, o, lse, dh.view_as(o), SCALE, dk_pool=torch.zeros_like(K), dv_pool=torch.zeros_like(P))
        assert lib.psrl_device_status(plan, "bwd") == 0
        dq = lib.psrl_rope_rows(rope, dq, torch.as_tensor(np.concatenate([np.arange(n) + a for n, a, r in zip(
            PV["seg_len"], PV["seg_anc_tokens"], PV["seg_q_off"]) if r >= 0]).astype(np.int32), device="cuda"), inverse=True)
        got_q[torch.as_tensor(rows, device="cuda")] = dq.double()
        acc[0].add_(dkp)
        acc[1].add_(dvp)
        for s in cache.end(m)["freed"]:
            collect(s)
            base.pop(s)
        moves, top = cache.compact()
        seen["move"] += len(moves)
        lib.psrl_kv_move(moves, K, P)
        lib.psrl_kv_move(moves, *acc)
        # what the moves left behind counts as free: its sums start at zero
        for a in acc:
            a[:, top:] = 0
    assert min(seen.values()) >= 1, seen
    pos = np.zeros(V["T"], dtype=np.int32)
    for c in range(V["n_seg"]):
        t = V["seg_tok_off"][c]
        pos[t:t + V["seg_len"][c]] = V["seg_anc_tokens"][c] + np.arange(V["seg_len"][c])
    got_k = lib.psrl_rope_rows(rope, got_k, torch.as_tensor(pos, device="cuda"), inverse=True)
    for got, ref, name in zip((got_q, got_k, got_v, got_w), want, ("dq", "dk", "dv", "dw")):
        close(got, ref, name)
