"""Block copies and in-place moves on the GPU: byte-exact against plain slicing on the CPU, untouched slots included."""
import numpy as np
import pytest
import torch

from paper_2608_25683_b200.workloads import Workload

from test_gpu_microbatch import gbs_of, run_forest, setup_gbs  # noqa: F401

pytestmark = pytest.mark.gpu
TYPES = [("bf16", 128), ("f32", 64), ("f32", 128), ("bf16", 64)]


def bits(t):
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def pools(seed, heads, cap, d, dtype, n=2):
    """Random bits: NaN and infinities among them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, raw = (torch.bfloat16, torch.int16) if dtype == "bf16" else (torch.float32, torch.int32)
    lo, hi = (-2 ** 15, 2 ** 15) if dtype == "bf16" else (-2 ** 31, 2 ** 31)
    return [torch.randint(lo, hi, (heads, cap, d), device="cuda", generator=g).to(raw).view(t) for _ in range(n)]


def plain(extents, src, dst):
    out, src = bits(dst).cpu().clone(), bits(src).cpu()
    for s, d, n in np.asarray(extents).tolist():
        out[:, d:d + n] = src[:, s:s + n]
    return out


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,longest,heads", [(1, 1, 1), (3, 40, 2), (64, 70, 3), (65, 16, 8), (1000, 9, 1), (2300, 5, 2), (20, 3000, 2)])
def test_copy(lib, dtype, d, n, longest, heads):
    rng = np.random.default_rng(n + longest)
    size = rng.integers(0 if n > 1 else 1, longest + 1, n)
    gap = rng.integers(0, 3, (2, n))
    at = [np.cumsum(size + gap[i]) - size for i in (0, 1)]
    e = np.stack([rng.permutation(np.stack([at[0], size], 1)), np.zeros((n, 2), dtype=np.int64)], 1)[:, 0]
    size = e[:, 1]
    to = np.cumsum(size + gap[1]) - size
    e = np.stack([e[:, 0], to, size], 1).astype(np.int32)[rng.permutation(n)]
    cap, cap2 = int((e[:, 0] + e[:, 2]).max()) + 3, int((e[:, 1] + e[:, 2]).max()) + 5
    (ks, vs), (kd, vd) = pools(1, heads, cap, d, dtype), pools(2, heads, cap2, d, dtype)
    want = plain(e, ks, kd), plain(e, vs, vd)
    lib.psrl_kv_copy(e, ks, vs, kd, vd)
    assert torch.equal(bits(kd).cpu(), want[0]) and torch.equal(bits(vd).cpu(), want[1])
    # and inside one pool, to slots that nothing reads
    k, v = pools(3, heads, 2 * cap, d, dtype)
    inside = np.concatenate([e[:, :1], cap + e[:, :1], e[:, 2:]], 1)
    want = plain(inside, k, k), plain(inside, v, v)
    lib.psrl_kv_copy(inside.tolist(), k, v, k, v)
    assert torch.equal(bits(k).cpu(), want[0]) and torch.equal(bits(v).cpu(), want[1])


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,longest,heads,hole", [
    (1, 1, 1, 1), (1, 5000, 2, 1),          # one block far longer than its hole: every slot overlaps
    (12, 160, 2, 40), (40, 300, 8, 16), (1000, 7, 1, 2), (2500, 6, 2, 3),
    (60, 4000, 8, 100),                     # many chunks of the whole grid
    (7, 64, 3, 5000),                       # nothing overlaps
])
def test_move(lib, dtype, d, n, longest, heads, hole):
    rng = np.random.default_rng(n + longest)
    size = rng.integers(1, longest + 1, n) if n > 1 else np.array([longest])
    gap = rng.integers(0, hole + 1, n)
    gap[0] = hole
    src = np.cumsum(size + gap) - size
    dst, end = [], 0
    for i in range(n):
        # the first blocks of a long list stay where they are, every third leaves a slot of its hole free
        to = int(src[i]) if n > 10 and i < n // 5 else min(end + (i % 3 == 1), int(src[i]))
        dst.append(to)
        end = to + int(size[i])
    e = np.stack([src, dst, size], 1).astype(np.int32)
    k, v = pools(4, heads, int(src[-1] + size[-1]) + 7, d, dtype)
    want = plain(e, k, k), plain(e, v, v)
    lib.psrl_kv_move(e, k, v)
    assert torch.equal(bits(k).cpu(), want[0]) and torch.equal(bits(v).cpu(), want[1])


def test_offsets_past_32_bits(lib):
    """Pools of more than 4 GiB each: the last head's slots lie beyond 32-bit byte and element offsets."""
    heads, cap, d = 9, 1 << 21, 128          # 9 x 2^21 x 128 = 2.4 G elements, 4.8 GB per pool
    k, v = (torch.zeros(heads, cap, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    k[:, cap - 64:cap - 32], v[:, cap - 64:cap - 32] = 1.0, 2.0
    lib.psrl_kv_move([[cap - 64, cap - 80, 32]], k, v)
    lib.psrl_kv_copy([[cap - 80, 5, 32]], k, v, k, v)
    for t, x in ((k, 1.0), (v, 2.0)):
        assert (t[:, cap - 80:cap - 32] == x).all() and (t[:, 5:37] == x).all() and (t[:, cap - 32:] == 0).all()
        assert (t[:, 37:cap - 80] == 0).all() and (t[:, :5] == 0).all()
    # the same by the kernel for large moves, the whole of the last slots
    for t in (k, v):
        t[:, cap - 40000:] = torch.arange(40000, device="cuda")[:, None] % 251
    lib.psrl_kv_move([[cap - 40000, cap - 40100, 40000]], k, v)
    for t in (k, v):
        assert (t[:, cap - 40100:cap - 100] == (torch.arange(40000, device="cuda") % 251).to(torch.bfloat16)[:, None]).all()


def test_streams_graphs_and_empty_lists(lib):
    k, v = pools(5, 2, 4000, 128, "bf16")
    e = np.array([[100, 90, 800], [1000, 890, 2500]], dtype=np.int32)
    want = plain(e, k, k), plain(e, v, v)
    first = k.clone(), v.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lib.psrl_kv_move(e, k, v, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(bits(k).cpu(), want[0]) and torch.equal(bits(v).cpu(), want[1])
    # two graphs with workspaces of their own, replayed back to back
    graphs = []
    spill = [torch.zeros(2, 64, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    ws = [torch.empty(512, dtype=torch.uint8, device="cuda") for _ in range(2)]
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lib.psrl_kv_copy([[0, 3, 40], [90, 43, 10]], k, v, *spill)
            lib.psrl_kv_move(e, k, v, workspace=((ws[i].data_ptr() + 255) // 256 * 256, 256))
        graphs.append(graph)
    for i in range(2):
        k.copy_(first[0]); v.copy_(first[1])
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(k).cpu(), want[0]) and torch.equal(bits(v).cpu(), want[1])
        assert torch.equal(bits(spill[0][:, 43:53]), bits(first[0][:, 90:100]))
    # nothing to do
    lib.psrl_kv_move([], k, v)
    lib.psrl_kv_move([[5, 5, 100]], k, v)
    lib.psrl_kv_copy(np.zeros((0, 3), dtype=np.int32), k, v, *spill)
    assert torch.equal(bits(k).cpu(), want[0])


def test_moves_that_overlap_in_time(lib):
    """Large and small moves on two streams at once, each with a workspace of its own."""
    e = [np.array([[700, 650, 30000], [30800, 30650, 9000]], dtype=np.int32), np.array([[90, 60, 500]], dtype=np.int32)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    start = [pools(40 + i, 8, 40000 if i == 0 else 600, 128, "bf16") for i in (0, 1)]
    want = []
    for i in (0, 1):
        k, v = (t.clone() for t in start[i])
        lib.psrl_kv_move(e[i], k, v)
        want.append((bits(k).clone(), bits(v).clone()))
        assert torch.equal(bits(k).cpu(), plain(e[i], start[i][0], start[i][0]))
    copies = [[tuple(t.clone() for t in start[i]) for _ in range(6)] for i in (0, 1)]
    torch.cuda.synchronize()
    for j in range(6):
        for i in (0, 1):
            lib.psrl_kv_move(e[i], *copies[i][j], stream=streams[i])
    torch.cuda.synchronize()
    for i in (0, 1):
        for k, v in copies[i]:
            assert torch.equal(bits(k), want[i][0]) and torch.equal(bits(v), want[i][1])


def test_wrapper_refusals(lib):
    k, v = pools(6, 2, 32, 128, "bf16")
    k2, v2 = pools(7, 2, 32, 128, "bf16")
    with pytest.raises(TypeError):
        lib.psrl_kv_move([], k.half(), v.half())
    with pytest.raises(ValueError):
        lib.psrl_kv_move([], k, v[:, :16])
    with pytest.raises(ValueError):
        lib.psrl_kv_copy([], k, v, k2[:1], v2[:1])
    with pytest.raises(RuntimeError):
        lib.psrl_kv_move([], k.cpu(), v.cpu())
    with pytest.raises(lib.PsrlError) as e:
        lib.psrl_kv_copy([[0, 0, 33]], k, v, k2, v2)
    assert e.value.name == "PSRL_ERR_SHAPE"


def test_cached_blocks_survive_compaction(lib):
    """The cache manager's own moves on real pools, over the micro-batches of a forest: every block's K and V are found
    where the next micro-batch's plan reads them."""
    parent = [-1, 0, 0, -1, 3, 3, 0, -1, 7, 3]
    seg_len = [300, 70, 129, 200, 45, 33, 150, 97, 20, 64]
    gbs, mb, M = [64, 32, 16], [0, 0, 1, 0, 1, 2, 3, 1, 2, 3], 4
    setup_gbs(parent, gbs)
    cache = lib.Cache(parent, seg_len, gbs, mb, M)
    rows = [torch.randn(2, n, 128, device="cuda").to(torch.bfloat16) for n in seg_len]
    K, V = (torch.full((2, 2048, 128), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    moved = 0
    for m in range(M):
        step = cache.begin(m)
        for s, b in zip(step["seg_id"], step["seg_slot_base"]):
            if s in step["new"]:
                K[:, b:b + seg_len[s]], V[:, b:b + seg_len[s]] = rows[s], -rows[s]
            assert torch.equal(K[:, b:b + seg_len[s]], rows[s]) and torch.equal(V[:, b:b + seg_len[s]], -rows[s])
        cache.end(m)
        moves, top = cache.compact()
        moved += len(moves)
        lib.psrl_kv_move(moves, K, V)
    assert moved >= 1


@pytest.mark.parametrize("kind", ["half freed", "far then near", "one slot"])
def test_large_moves_beside_other_work(lib, kind):
    """Several hundred MB moved on one stream while matrix products keep another busy, so that the move's blocks neither start
    nor run alike: half of the arena freed; each head's first blocks far down and its last ones hardly at all; one block of
    nearly the whole arena by one slot.  Byte-exact every time, and the status word is clear."""
    rng = np.random.default_rng(3)
    if kind == "half freed":
        size, gap = 16 * rng.integers(1, 80, 150), 16 * rng.integers(0, 80, 150)
    elif kind == "far then near":
        size, gap = 16 * rng.integers(1, 120, 100), np.where(np.arange(100) % 2, 16, 0)
        gap[0] = 30000
    else:
        size, gap = np.array([90001]), np.array([1])
    src = np.cumsum(size + gap) - size
    e = np.stack([src, np.cumsum(size) - size, size], 1).astype(np.int32)
    heads, cap, d = 8, int(src[-1] + size[-1]) + 5, 128
    k0, v0 = pools(60, heads, cap, d, "bf16")
    want = []
    for t in (k0, v0):
        w = bits(t).clone()
        for s, to, n in e.tolist():
            w[:, to:to + n] = bits(t)[:, s:s + n]
        want.append(w)
    a = torch.randn(2048, 2048, device="cuda").to(torch.bfloat16)
    move, other = torch.cuda.Stream(), torch.cuda.Stream()
    buf = torch.empty(512, dtype=torch.uint8, device="cuda")
    ws = (buf.data_ptr() + 255) // 256 * 256, 256
    for _ in range(8):
        k, v = k0.clone(), v0.clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            for _ in range(30):
                a @ a
        lib.psrl_kv_move(e, k, v, stream=move, workspace=ws)
        torch.cuda.synchronize()
        assert lib.lib().psrl_device_status(ws[0], None) == 0
        assert torch.equal(bits(k), want[0]) and torch.equal(bits(v), want[1])
