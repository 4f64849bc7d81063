"""Token log-probabilities and their gradients in fp64, row by row from the definition, and the next tokens of a tree from
its samples.  Test infrastructure; shares nothing with the library.

Pins: finite differences and a row of equal logits (tests/test_logprob.py)."""
import numpy as np

from .attention import sample_paths


def oracle_logprob(hidden, weight, targets, off=None, scale=1.0, d_logprob=None):
    """hidden [N, H], weight [V, H] (fp64).  Returns a dict with logprob, lse and, given d_logprob, d_hidden, d_weight,
    and sums of absolute values that error bounds are made of."""
    N, V = len(hidden), len(weight)
    off = np.arange(N + 1) if off is None else np.asarray(off)
    out = dict(logprob=np.zeros(len(targets)), lse=np.zeros(N))
    if d_logprob is not None:
        out.update(d_hidden=np.zeros_like(hidden), d_weight=np.zeros_like(weight), dh_abs=np.zeros_like(hidden),
                   dw_abs=np.zeros_like(weight))
    for r in range(N):
        z = scale * (weight @ hidden[r])
        top = z.max()
        p = np.exp(z - top)
        out["lse"][r] = top + np.log(p.sum())
        p /= p.sum()
        dz = np.zeros(V)
        for t in range(off[r], off[r + 1]):
            y = targets[t]
            if not 0 <= y < V:
                continue
            out["logprob"][t] = z[y] - out["lse"][r]
            if d_logprob is not None:
                dz -= d_logprob[t] * p
                dz[y] += d_logprob[t]
        if d_logprob is not None:
            dz *= scale
            out["d_hidden"][r] = dz @ weight
            out["dh_abs"][r] = np.abs(dz) @ np.abs(weight)
            out["d_weight"] += np.outer(dz, hidden[r])
            out["dw_abs"] += np.outer(np.abs(dz), np.abs(hidden[r]))
    return out


def oracle_next_tokens(V):
    """{query row: sorted tokens it predicts} of an oracle plan: walks every sample token by token."""
    row_of = {}
    for c in range(V["n_seg"]):
        if V["seg_q_off"][c] >= 0:
            for i in range(V["seg_len"][c]):
                row_of[V["seg_tok_off"][c] + i] = V["seg_q_off"][c] + i
    nxt = {r: set() for r in row_of.values()}
    for path in sample_paths(V):
        toks = [t for c in path for t in range(V["seg_tok_off"][c], V["seg_tok_off"][c] + V["seg_len"][c])]
        for a, b in zip(toks, toks[1:]):
            if a in row_of:
                nxt[row_of[a]].add(b)
    return {int(r): sorted(int(t) for t in s) for r, s in nxt.items()}
