"""Token log-probabilities and gradients on the GPU against the fp64 oracle on the same bf16 inputs.

Error bounds, with A = max over v of |scale| sum_i |h_i w_vi| of the row:
  logits    products of bf16 are exact in fp32; a 16-deep step adds them to the fp32 sum with at most 2^-22 of the sizes
            involved, so a logit is off by (H/16 + 8) 2^-22 A; the target's own dot product adds H/32 + 8 terms in fp32
  lse       the logits' error, and 2^-20 for exponentials and their sum, and the rounding of a number of lse's size
  dz        exp of that error, half a bf16 step (2^-8), 2^-18 for the exponential and the products; at a target
            dz = scale (g_t - G p) with p = exp(lp): an error e of lp moves it by |scale G| p e, whatever is left of dz
            itself where p is near 1, so scale |G| e (e as for logprob) times the other operand is added there
  products  sums in fp32 as above over K terms, then half a bf16 step of the result
  f32       the same with K terms added one by one in fp32 (K 2^-24) and half steps of 2^-24
Sums of absolute values come from the oracle."""
import numpy as np
import pytest
import torch

from oracle.logprob import oracle_logprob
from paper_2608_25683_b200.workloads import Workload

from util import build_plan, to_np

pytestmark = pytest.mark.gpu


def make(n, h, v, seed, m=None, spread=1.0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    hidden = rnd(n, h).to(dtype)
    weight = (rnd(v, h) * (spread / np.sqrt(h))).to(dtype)
    m = n if m is None else m
    targets = torch.randint(0, v, (m,), generator=g, device="cuda").to(torch.int32)
    return hidden, weight, targets, rnd(m)


def sum_error(k, dtype):
    return (k / 16 + 8) * 2.0 ** -22 if dtype == torch.bfloat16 else (k + 8) * 2.0 ** -24


def bounds(hidden, weight, scale, want, dtype=torch.bfloat16):
    a = np.abs(scale) * (np.abs(hidden) @ np.abs(weight).T).max(1)
    z = sum_error(hidden.shape[1], dtype) * a
    return z, z + 2.0 ** -20 + 2.0 ** -22 * np.abs(want["lse"])


def check(lib, hidden, weight, targets, g, off=None, scale=1.0, **kw):
    hn, wn, tn = to_np(hidden), to_np(weight), targets.cpu().numpy()
    on = None if off is None else off.cpu().numpy()
    want = oracle_logprob(hn, wn, tn, on, scale, to_np(g))
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets, off, scale=scale, **kw)
    half = 2.0 ** -8 if hidden.dtype == torch.bfloat16 else 2.0 ** -24
    zerr, lerr = bounds(hn, wn, scale, want, hidden.dtype)
    assert (np.abs(to_np(lse) - want["lse"]) <= lerr).all()
    row = np.arange(len(hn)) if on is None else np.repeat(np.arange(len(hn)), np.diff(on))
    size = np.abs(want["logprob"]) + 2 * np.abs(want["lse"][row])
    lperr = lerr[row] + zerr[row] + 2.0 ** -22 * size
    assert (np.abs(to_np(lp) - want["logprob"]) <= lperr).all()
    on_target = (tn >= 0) & (tn < len(wn))
    total = np.zeros(len(hn))
    np.add.at(total, row[on_target], to_np(g)[on_target])
    moved = np.zeros((len(hn), len(wn)))           # what lp's error does to dz at the targets
    np.maximum.at(moved, (row[on_target], tn[on_target]), (np.abs(scale * total[row]) * lperr)[on_target])
    dh, dw = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g, off, scale=scale, **kw)
    assert dh.dtype == dw.dtype == hidden.dtype
    pe = (lerr + zerr).max() * 2 + half + 2.0 ** -18
    for got, d, absd, k, far in ((dh, want["d_hidden"], want["dh_abs"], len(wn), moved @ np.abs(wn)),
                                 (dw, want["d_weight"], want["dw_abs"], len(hn), moved.T @ np.abs(hn))):
        tol = far + (pe + sum_error(k, hidden.dtype) + 2.0 ** -18) * absd + half * np.abs(d) * (1 + 2.0 ** -7) + 1e-37
        err = np.abs(to_np(got) - d) - tol
        assert err.max() <= 0, (float(err.max()), float(np.abs(d).max()))
    return lp, lse, dh, dw


@pytest.mark.parametrize("n,h,v", [(1, 8, 1), (1, 64, 7), (3, 72, 255), (128, 64, 256), (129, 136, 257), (256, 128, 512),
                                   (257, 200, 1000), (300, 512, 777), (33, 1024, 5000), (600, 64, 2049), (1, 4096, 3001)])
@pytest.mark.parametrize("scale", [1.0, -0.4])
def test_one_target_per_row(lib, n, h, v, scale):
    hidden, weight, targets, g = make(n, h, v, n + h + v)
    check(lib, hidden, weight, targets, g, scale=scale)


@pytest.mark.parametrize("n,h,v", [(1, 8, 1), (3, 72, 255), (64, 64, 64), (65, 136, 130), (130, 40, 1000), (33, 256, 5000), (700, 16, 3001)])
@pytest.mark.parametrize("scale", [1.0, -0.4])
def test_fp32(lib, n, h, v, scale):
    hidden, weight, targets, g = make(n, h, v, n + h + v, dtype=torch.float32)
    check(lib, hidden, weight, targets, g, scale=scale)


def test_fp32_ragged_and_strided(lib):
    """Rows with none, one and several targets, slices of wider matrices, several pieces of the vocabulary."""
    rng = np.random.default_rng(2)
    n, h, v = 9000, 16, 9001
    count = rng.choice([0, 1, 1, 2], n)
    off = torch.as_tensor(np.concatenate([[0], np.cumsum(count)]).astype(np.int32), device="cuda")
    hidden, weight, targets, g = make(n, h, v, 22, m=int(count.sum()), dtype=torch.float32)
    targets[::50] = -1
    wide = torch.full((n, h + 12), float("nan"), device="cuda")
    wide[:, 4:4 + h] = hidden
    lp, lse = lib.psrl_token_logprob_fwd(wide[:, 4:4 + h], weight, targets, off)
    out = torch.full_like(wide, 5.0)
    dh, dw = lib.psrl_token_logprob_bwd(wide[:, 4:4 + h], weight, targets, lp, lse, g, off, d_hidden=out[:, 4:4 + h])
    assert (out[:, :4] == 5).all() and (out[:, 4 + h:] == 5).all()
    hd, wd = hidden.double(), weight.double()
    z = hd @ wd.T
    ref = torch.logsumexp(z, 1)
    assert ((lse.double() - ref).abs() <= 2.0 ** -19 + 2.0 ** -21 * ref.abs()).all()
    row = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.as_tensor(count, device="cuda"))
    keep = targets >= 0
    want = (z[row, targets.long().clamp(min=0)] - ref[row]) * keep
    assert ((lp.double() - want).abs() <= 2.0 ** -18 + 2.0 ** -21 * want.abs()).all()
    total = torch.zeros(n, device="cuda", dtype=torch.float64).index_add_(0, row, g.double() * keep)
    dz = -total[:, None] * torch.exp(z - ref[:, None])
    dz.index_put_((row, targets.long().clamp(min=0)), g.double() * keep, accumulate=True)
    # at the targets: |G| times the error of lp (below 2^-18 + 2^-21 x 25 < 2^-16) times the other operand
    big, t = (total[row].abs() * keep)[:, None] * 2.0 ** -16, targets.long().clamp(min=0)
    far_h, far_w = (torch.zeros_like(x).index_add_(0, i, big * y[j].abs()) for x, i, y, j in ((hd, row, wd, t), (wd, t, hd, row)))
    for got, d, absd, k, far in ((dh, dz @ wd, dz.abs() @ wd.abs(), v, far_h), (dw, dz.T @ hd, dz.abs().T @ hd.abs(), n, far_w)):
        assert ((got.double() - d).abs() <= (sum_error(k, torch.float32) + 2.0 ** -16) * absd + far).all()


def test_confident_rows(lib):
    """Probabilities from near 0 to 1 - 1e-6: the gradient at the target keeps its relative precision."""
    hidden, weight, targets, g = make(200, 256, 900, 5)
    boost = torch.linspace(0, 22, 200, device="cuda")[:, None]
    w = weight[targets.long()].float()
    hidden = (hidden.float() + boost * w / (w * w).sum(1, keepdim=True)).to(torch.bfloat16)
    lp, lse, dh, dw = check(lib, hidden, weight, targets, g)
    assert lp.max() > -1e-3 and (lp <= 0).all()


def test_large_logits(lib):
    """Logits of several hundred: nothing overflows."""
    hidden, weight, targets, g = make(70, 128, 400, 6, spread=60.0)
    check(lib, hidden, weight, targets, g)


@pytest.mark.parametrize("seed", [0, 1])
def test_ragged_targets(lib, seed):
    """Rows without targets, with several, the same token twice, ignored ones; one row with very many."""
    rng = np.random.default_rng(seed)
    n, h, v = 333, 136, 700
    count = rng.choice([0, 0, 1, 1, 1, 2, 5], n)
    count[[0, 17, n - 1]] = [0, 150, 40]
    off = torch.as_tensor(np.concatenate([[0], np.cumsum(count)]).astype(np.int32), device="cuda")
    hidden, weight, targets, g = make(n, h, v, seed, m=int(count.sum()))
    row = np.repeat(np.arange(n), count)
    t = targets.cpu().numpy()
    t[rng.random(len(t)) < 0.1] = -100
    t[rng.random(len(t)) < 0.05] = v
    t[rng.random(len(t)) < 0.02] = 2 ** 31 - 1
    again = np.flatnonzero(np.diff(row) == 0)[::3]
    t[again + 1] = t[again]
    g[::7] = 0
    targets = torch.as_tensor(t, device="cuda")
    lp, lse, dh, dw = check(lib, hidden, weight, targets, g, off, scale=0.7)
    ignored = torch.as_tensor((t < 0) | (t >= v), device="cuda")
    assert (lp[ignored] == 0).all()
    empty = torch.as_tensor([not ((row == r) & (t >= 0) & (t < v)).any() for r in range(n)], device="cuda")
    assert empty.any() and (dh[empty] == 0).all()


def test_a_row_with_very_many_targets(lib):
    """300,000 targets in one row, most tokens many times over: the cost grows with their number, not with its square."""
    n, h, v, k = 40, 64, 5000, 300000
    hidden, weight, targets, g = make(n, h, v, 21, m=k + n)
    off = torch.arange(n + 1, device="cuda", dtype=torch.int32)
    off[8:] += k
    targets[3000:4000] = -7
    check(lib, hidden, weight, targets, g / 500, off)


def test_no_targets_and_no_rows(lib):
    hidden, weight, targets, g = make(40, 64, 300, 3)
    none = torch.zeros(41, dtype=torch.int32, device="cuda")
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets[:0], none)
    assert lp.shape == (0,) and torch.isfinite(lse).all()
    dh, dw = lib.psrl_token_logprob_bwd(hidden, weight, targets[:0], lp, lse, g[:0], none)
    assert (dh == 0).all() and (dw == 0).all()
    ignored = torch.full_like(targets, -1)
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, ignored)
    assert (lp == 0).all()
    dh, dw = lib.psrl_token_logprob_bwd(hidden, weight, ignored, lp, lse, g)
    assert (dh == 0).all() and (dw == 0).all()
    lp, lse = lib.psrl_token_logprob_fwd(hidden[:0], weight, targets[:0])
    dh, dw = lib.psrl_token_logprob_bwd(hidden[:0], weight, targets[:0], lp, lse, g[:0], d_weight=torch.full_like(weight, 3.0))
    assert lse.shape == (0,) and dh.shape == (0, 64) and (dw == 0).all()


def test_padding_rows_may_hold_anything(lib):
    """A row whose targets are all ignored (padding) may hold NaN or infinities: it reaches no other row and no gradient."""
    hidden, weight, targets, g = make(300, 128, 1000, 8)
    targets[100:140] = -1
    clean = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    want = lib.psrl_token_logprob_bwd(hidden, weight, targets, *clean, g)
    dirty = hidden.clone()
    dirty[100:120], dirty[120:140] = float("nan"), float("inf")
    lp, lse = lib.psrl_token_logprob_fwd(dirty, weight, targets)
    keep = torch.ones(300, dtype=torch.bool, device="cuda")
    keep[100:140] = False
    assert torch.equal(lp, clean[0]) and torch.equal(lse[keep], clean[1][keep])
    dh, dw = lib.psrl_token_logprob_bwd(dirty, weight, targets, lp, lse, g)
    assert torch.equal(dh, want[0]) and torch.equal(dw, want[1]) and (dh[100:140] == 0).all()


def test_strides_and_single_gradients(lib):
    """Rows of a wider matrix in and out; either gradient alone; bitwise the same every time."""
    n, h, v = 270, 192, 1111
    hidden, weight, targets, g = make(n, h, v, 9)
    wide = torch.full((n, h + 40), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide[:, 8:8 + h] = hidden
    wide_w = torch.full((v, h + 8), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide_w[:, :h] = weight
    lp, lse, dh, dw = check(lib, hidden, weight, targets, g)
    x, w = wide[:, 8:8 + h], wide_w[:, :h]
    assert all(torch.equal(a, b) for a, b in zip(lib.psrl_token_logprob_fwd(x, w, targets), (lp, lse)))
    out, out_w = torch.full_like(wide, 5.0), torch.full_like(wide_w, 5.0)
    got = lib.psrl_token_logprob_bwd(x, w, targets, lp, lse, g, d_hidden=out[:, 8:8 + h], d_weight=out_w[:, :h])
    assert torch.equal(got[0], dh) and torch.equal(got[1], dw)
    assert (out[:, :8] == 5).all() and (out[:, 8 + h:] == 5).all() and (out_w[:, h:] == 5).all()
    only = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g, want_weight=False)
    assert torch.equal(only[0], dh) and only[1] is None
    only = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g, want_hidden=False)
    assert only[0] is None and torch.equal(only[1], dw)


def test_several_pieces_of_the_vocabulary(lib):
    """More vocabulary than one piece of the workspace: the sums over the pieces, an odd last piece, several row groups."""
    n, h, v = 9000, 64, 20011
    hidden, weight, targets, g = make(n, h, v, 10)
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    z = hidden.double() @ weight.double().T
    ref = torch.logsumexp(z, 1)
    a = (hidden.double().abs() @ weight.double().abs().T).amax(1)
    tol = (h / 16 + 8) * 2.0 ** -22 * a + 2.0 ** -20 + 2.0 ** -22 * ref.abs()
    assert ((lse.double() - ref).abs() <= tol).all()
    at = torch.arange(n, device="cuda")
    dz = -g.double()[:, None] * torch.exp(z - ref[:, None])
    dz[at, targets.long()] += g.double()
    dh, dw = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g)
    pe = 2 * float(tol.max()) + 2.0 ** -8 + 2.0 ** -18
    for got, d, absd, k in ((dh, dz @ weight.double(), dz.abs() @ weight.double().abs(), v),
                            (dw, dz.T @ hidden.double(), dz.abs().T @ hidden.double().abs(), n)):
        bound = (pe + (k / 16 + 24) * 2.0 ** -22) * absd + 2.0 ** -8 * d.abs() * (1 + 2.0 ** -7)
        assert ((got.double() - d).abs() <= bound).all()


def test_gradient_against_differences(lib):
    """Steps of 2^-4 on inputs that are multiples of 2^-4: the moved inputs are bf16 numbers too.  The oracle's own
    difference says how much of the gap is the loss's curvature."""
    g0 = torch.Generator(device="cuda").manual_seed(11)
    n, h, v = 60, 64, 300
    grid = lambda *s: (torch.randint(-16, 17, s, generator=g0, device="cuda") / 16)
    hidden, weight = grid(n, h).to(torch.bfloat16), (grid(v, h) / 4).to(torch.bfloat16)
    targets = torch.randint(0, v, (n,), generator=g0, device="cuda").to(torch.int32)
    g = torch.randn(n, generator=g0, device="cuda")
    step = (torch.randint(0, 2, (n, h), generator=g0, device="cuda") * 2 - 1) / 16
    lp, lse, dh, dw = check(lib, hidden, weight, targets, g)
    sides = [(hidden.float() + s * step).to(torch.bfloat16) for s in (1, -1)]
    got = [float((lib.psrl_token_logprob_fwd(x, weight, targets)[0].double() * g.double()).sum()) for x in sides]
    ref = [float((oracle_logprob(to_np(x), to_np(weight), targets.cpu().numpy())["logprob"] * to_np(g)).sum()) for x in sides]
    slope = float((dh.double() * step.double()).sum()) * 2
    want = oracle_logprob(to_np(hidden), to_np(weight), targets.cpu().numpy(), None, 1.0, to_np(g))
    exact = float((want["d_hidden"] * to_np(step)).sum()) * 2
    noise = 2 * float(g.abs().sum()) * 2.0 ** -16 + 2.0 ** -6 * float((want["dh_abs"] * np.abs(to_np(step))).sum())
    assert abs((got[0] - got[1]) - slope) <= abs((ref[0] - ref[1]) - exact) + noise


def test_streams_and_graphs(lib):
    hidden, weight, targets, g = make(300, 256, 3000, 12)
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    dh, dw = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = lib.psrl_token_logprob_fwd(hidden, weight, targets, stream=side)
    b = lib.psrl_token_logprob_bwd(hidden, weight, targets, *a, g, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(a + b, (lp, lse, dh, dw)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = lib.psrl_token_logprob_fwd(hidden, weight, targets)
        b = lib.psrl_token_logprob_bwd(hidden, weight, targets, *a, g)
    hidden.neg_(); g.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    dh, dw = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g)
    assert all(torch.equal(x, y) for x, y in zip(a + b, (lp, lse, dh, dw)))


def test_calls_that_overlap(lib):
    """Two streams, each with inputs and temporaries of its own, many calls in flight at once."""
    sets = [make(n, 192, 3000, 30 + n) for n in (3, 300)]
    want = []
    for hidden, weight, targets, g in sets:
        lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets)
        want.append((lp, lse) + lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g))
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, (hidden, weight, targets, g) in enumerate(sets):
            a = lib.psrl_token_logprob_fwd(hidden, weight, targets, stream=streams[i])
            got[i].append(a + lib.psrl_token_logprob_bwd(hidden, weight, targets, *a, g, stream=streams[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        for x in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(x, want[i]))


def test_device_status_and_wrapper_refusals(lib):
    import ctypes

    hidden, weight, targets, g = make(20, 64, 100, 13)
    need = lib.psrl_token_logprob_workspace_bytes(20, 64, 100, 20, True)
    buf = torch.full((need + 256,), 7, dtype=torch.uint8, device="cuda")
    ws = (buf.data_ptr() + 255) // 256 * 256, need
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets, workspace=ws)
    lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g, workspace=ws)
    assert lib.lib().psrl_device_status(ctypes.c_void_p(ws[0]), None) == 0
    for x, w in ((hidden.float(), weight), (hidden.half(), weight.half())):
        with pytest.raises(TypeError):
            lib.psrl_token_logprob_fwd(x, w, targets)
    for bad in (dict(targets=targets.long()), dict(weight=weight[:, :56]), dict(target_off=targets), dict(lse=lse[:3])):
        with pytest.raises(ValueError):
            lib.psrl_token_logprob_fwd(**{**dict(hidden=hidden, weight=weight, targets=targets), **bad})
    with pytest.raises(ValueError):
        lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g, d_weight=weight[:50])
    with pytest.raises(RuntimeError):
        lib.psrl_token_logprob_fwd(hidden.cpu(), weight.cpu(), targets.cpu())
    with pytest.raises(lib.PsrlError) as e:
        lib.psrl_token_logprob_fwd(hidden, weight, targets[:10])
    assert e.value.name == "PSRL_ERR_SHAPE"


@pytest.mark.parametrize("h", [4096, 4168])
def test_pairs_that_keep_pace(lib, h):
    """Enough rows, depth and vocabulary that the pairs of CTAs wait for one another: four forwards in flight on two streams,
    more CTAs than the device holds at once, then a captured one replayed; all alike, and right for some of the rows."""
    n, v = 1030, 16384 - 37
    hidden, weight, targets, _ = make(n, h, v, 50)
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    rows = torch.tensor([0, 1, 255, 256, 1023, 1024, n - 1], device="cuda")
    hn, wn = to_np(hidden[rows]), to_np(weight)
    want = oracle_logprob(hn, wn, targets[rows].cpu().numpy())
    zerr, lerr = bounds(hn, wn, 1.0, want)
    assert (np.abs(to_np(lse[rows]) - want["lse"]) <= lerr).all()
    size = np.abs(want["logprob"]) + 2 * np.abs(want["lse"])
    assert (np.abs(to_np(lp[rows]) - want["logprob"]) <= lerr + zerr + 2.0 ** -22 * size).all()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [lib.psrl_token_logprob_fwd(hidden, weight, targets, stream=s) for _ in range(2) for s in streams]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got.append(lib.psrl_token_logprob_fwd(hidden, weight, targets))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for x in got:
        assert torch.equal(x[0], lp) and torch.equal(x[1], lse)


@pytest.mark.parametrize("n,dtype", [(1, torch.bfloat16), (5, torch.bfloat16), (128, torch.bfloat16), (200, torch.bfloat16), (3, torch.float32)])
def test_few_rows_over_several_pieces(lib, n, dtype):
    """A vocabulary of more than one piece for few rows, whose dz is kept in two parts, with several targets a row."""
    h, v, m = 16, 600011 if n <= 128 else 700001, 3 * n
    if dtype == torch.float32:
        v = 1100003
    hidden, weight, targets, g = make(n, h, v, 70 + n, m=m, dtype=dtype)
    off = torch.arange(0, m + 1, 3, device="cuda", dtype=torch.int32)
    targets[1] = targets[0]
    targets[2] = v - 1
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets, off)
    dh, dw = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g, off)
    hd, wd, gd, t = hidden.double(), weight.double(), g.double(), targets.long()
    row = torch.arange(n, device="cuda").repeat_interleave(3)
    z = hd @ wd.T
    ref = torch.logsumexp(z, 1)
    a = (hd.abs() @ wd.abs().T).amax(1)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    zerr = sum_error(h, dtype) * a
    lerr = zerr + 2.0 ** -20 + 2.0 ** -22 * ref.abs()
    assert ((lse.double() - ref).abs() <= lerr).all()
    want = z[row, t] - ref[row]
    lperr = lerr[row] + zerr[row] + 2.0 ** -22 * (want.abs() + 2 * ref[row].abs())
    assert ((lp.double() - want).abs() <= lperr).all()
    total = torch.zeros(n, device="cuda", dtype=torch.float64).index_add_(0, row, gd)
    dz = -total[:, None] * torch.exp(z - ref[:, None])
    dz.index_put_((row, t), gd, accumulate=True)
    moved = (total[row].abs() * lperr)[:, None]
    far_h = torch.zeros_like(hd).index_add_(0, row, moved * wd[t].abs())
    far_w = torch.zeros_like(wd).index_add_(0, t, moved * hd[row].abs())
    pe = float((lerr + zerr).max()) * 2 + half + 2.0 ** -18
    for got, d, absd, k, far in ((dh, dz @ wd, dz.abs() @ wd.abs(), v, far_h), (dw, dz.T @ hd, dz.abs().T @ hd.abs(), n, far_w)):
        tol = far + (pe + sum_error(k, dtype) + 2.0 ** -18) * absd + half * d.abs() * (1 + 2.0 ** -7) + 1e-37
        assert ((got.double() - d).abs() <= tol).all()
