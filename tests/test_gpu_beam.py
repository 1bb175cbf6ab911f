"""pc_beam_select / pc_beam_reorder against sorts of every candidate in 64 bits: all element types, one to 64 beams and survivors,
ties, masked and dead beams, finished beams, rows longer and shorter than any tile, in ascending, descending and constant order.

The choice is exact where z carries the score (no normaliser): the order is that of exact sums.  With a normaliser beams are compared by
running + z - lse, whose lse the library holds to some 1e-7 (a sum of exp with 2^-24 each, added in 64 bits at the end): the tests draw
inputs whose candidates of different beams lie further apart than 1e-5, checked on the reference."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2406_00766_amd import binding as pcb
from tests.replay import replayed

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def reference(z, running, n, done=None, done_token=0, normalise=False):
    z = z.double().numpy().copy()
    running = running.double().numpy()
    G, W = running.shape
    V = z.shape[1]
    scores, parents, tokens, gap = np.zeros((G, n)), np.zeros((G, n), int), np.zeros((G, n), int), np.inf
    with np.errstate(all="ignore"):
        for g in range(G):
            rows = []
            for b in range(W):
                v, run = z[g * W + b], running[g, b]
                run = run if run < np.inf else -np.inf
                if done is not None and done[g, b]:
                    v = np.full(V, -np.inf)
                    v[done_token] = 0.0
                elif normalise:
                    m = v.max()
                    lse = m + np.log(np.sum(np.exp(v - m)))
                    v = v - lse if np.isfinite(lse) else np.full(V, -np.inf)
                v = np.where(np.isnan(v), -np.inf, v)
                if run == -np.inf:
                    v = np.full(V, -np.inf)
                best = np.lexsort((np.arange(V), -v))[:n]
                s = run + v[best]
                rows += [(s[i], b, i, best[i]) for i in range(len(best))]
            rows.sort(key=lambda r: (-r[0], r[1], r[2]))
            for a, b in zip(rows[:n], rows[1:n + 1]):
                if a[1] != b[1] and np.isfinite(a[0]) and np.isfinite(b[0]) and a[0] != b[0]:
                    gap = min(gap, a[0] - b[0])
            for i, r in enumerate(rows[:n]):
                scores[g, i], parents[g, i], tokens[g, i] = r[0], r[1], r[3]
    return scores, parents, tokens, gap


def select(z, running, n, done=None, done_token=0, normalise=False, pad=0):
    G = running.shape[0]
    held = torch.full((z.shape[0], z.shape[1] + pad), 1e4, dtype=z.dtype, device="cuda")
    held[:, :z.shape[1]] = z.cuda()
    a = pcb.beam(held[:, :z.shape[1]], running.cuda(), n, done=None if done is None else torch.from_numpy(done).cuda(), done_token=done_token, normalise=normalise)
    ws = torch.full((pcb.pc_beam_workspace_bytes(a),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((G, n), 9.0, device="cuda"), torch.full((G, n), -9, dtype=torch.int32, device="cuda"), torch.full((G, n), -9, dtype=torch.int32, device="cuda")
    pcb.pc_beam_select(a, ws, *out)
    return [t.cpu().numpy() for t in out]


def check(z, running, n, **kw):
    got = select(z, running, n, **kw)
    kw.pop("pad", None)
    scores, parents, tokens, gap = reference(z, running, n, **kw)
    assert not kw.get("normalise") or gap > 1e-5, gap
    assert np.array_equal(got[1], parents) and np.array_equal(got[2], tokens)
    fin = np.isfinite(scores)
    assert np.array_equal(got[0][~fin], scores[~fin])
    assert np.all(np.abs(got[0][fin] - scores[fin]) <= 2.0 ** -23 * np.abs(scores[fin]) + 2e-6)
    return got


def draw(G, W, V, dtype, seed, spread=3.0):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy(rng.normal(size=(G * W, V)) * spread).to(TYPES[dtype])
    return z, torch.from_numpy((-10 * rng.random((G, W))).astype(np.float32)), rng


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("G,W,V,n,pad", [(1, 1, 1, 1, 0), (2, 1, 7, 5, 1), (3, 2, 5, 10, 0), (1, 4, 50257, 8, 3), (5, 3, 1000, 6, 1), (2, 64, 70, 64, 2), (70, 8, 333, 16, 0),
                                         (1, 1, 100003, 64, 1), (2, 33, 4097, 40, 0), (300, 4, 64, 4, 5), (1, 64, 3, 64, 0), (1, 64, 1, 64, 0)])
@pytest.mark.parametrize("normalise", [False, True])
def test_selection_matches_a_full_sort(dtype, G, W, V, n, pad, normalise):
    print(f"case beam {dtype} G={G} W={W} V={V} n={n} normalise={normalise}", flush=True)
    for seed in range(50):                                  # the first seed whose close calls are none (see above)
        z, running, _ = draw(G, W, V, dtype, seed)
        if not normalise or reference(z, running, n, normalise=True)[3] > 1e-5:
            break
    check(z, running, n, normalise=normalise, pad=pad)


@pytest.mark.parametrize("order", ["ascending", "descending", "constant", "steps", "two_values", "peaks_last", "mostly_excluded", "all_lowest"])
@pytest.mark.parametrize("dtype,V", [("f32", 30011), ("bf16", 9001), ("f16", 5000), ("f32", 300)])
@pytest.mark.parametrize("n", [1, 7, 64])
def test_orders_of_a_row_and_ties(order, dtype, V, n):
    i = np.arange(V, dtype=np.float64)
    row = {"ascending": i / V, "descending": -i / V, "constant": 0 * i + 0.5, "steps": np.floor(i / 100), "two_values": (i % 2) * 1.0, "peaks_last": np.where(i > V - 40, i, 0.0),
           "mostly_excluded": np.where(i % 997 == 5, i / V, -np.inf), "all_lowest": np.full(V, float(torch.finfo(TYPES[dtype]).min))}[order]
    z = torch.from_numpy(np.stack([row, row, row[::-1].copy()])).to(TYPES[dtype])
    running = torch.tensor([[-1.0, -1.0, -1.0]])
    check(z, running, n)
    check(z[:1], running[:, :1], min(n, V), pad=1)


@pytest.mark.parametrize("order", ["ascending", "descending", "constant", "steps", "random", "peaks_last", "mostly_excluded", "all_excluded", "late_excluded"])
@pytest.mark.parametrize("dtype,V", [("f32", 20011), ("bf16", 33001), ("f16", 17003)])
@pytest.mark.parametrize("n", [5, 64])
def test_rows_that_one_workgroup_walks_through(order, dtype, V, n):
    """So many rows that each is one segment of several chunks; the same four rows in every group, at every alignment."""
    i = np.arange(V, dtype=np.float64)
    row = {"ascending": i / V, "descending": -i / V, "constant": 0 * i + 0.5, "steps": np.floor(i / 3000), "random": np.random.default_rng(3).normal(size=V) * 3,
           "peaks_last": np.where(i > V - 40, i, 0.0), "mostly_excluded": np.where(i % 4999 == 17, i / V, -np.inf), "all_excluded": np.full(V, -np.inf),
           "late_excluded": np.where(i < V - 3, -np.inf, i / V)}[order]
    four = torch.from_numpy(np.stack([row, row[::-1].copy(), np.roll(row, V // 2), row])).to(TYPES[dtype])
    G = 300                                                 # 1200 rows
    running = torch.tensor([[-0.5, -0.25, -1.0, -0.5]])
    got = select(four.repeat(G, 1), running.repeat(G, 1), n, pad=1)
    scores, parents, tokens, _ = reference(four, running, n)
    for g in (got[1] != parents, got[2] != tokens, got[0] != scores.astype(np.float32)):
        assert not g.any()


@pytest.mark.parametrize("live", [0, 1, 2, 40])
@pytest.mark.parametrize("V", [64, 9000])
def test_many_beams_of_which_few_live(live, V):
    """64 beams and survivors: 4096 entries to join, most or all of them at -inf."""
    z, running, rng = draw(2, 64, V, "f32", 61)
    running[:, live:] = -float("inf")
    done = np.zeros((2, 64), np.uint8)
    done[1, ::2] = 1
    for n in (1, 64):
        check(z, running, n)
        check(z, running, n, done=done, done_token=V - 1)
        check(torch.zeros_like(z), torch.zeros_like(running), n)    # every candidate ties


def test_signed_zeros_tie_and_numbers_that_are_none_come_last():
    inf, nan = float("inf"), float("nan")
    z = torch.tensor([[-0.0, 0.0, -0.0, nan, -inf, 1.0, nan, -1.0], [inf, inf, 0.0, -inf, nan, -inf, 2.0, inf]])
    check(z, torch.tensor([[0.0, 0.5]]), 16)
    check(z[:1], torch.tensor([[0.0]]), 8)


def test_dead_masked_and_finished_beams():
    inf, nan = float("inf"), float("nan")
    z, running, rng = draw(6, 5, 400, "f32", 21)
    running[0, 1:] = -inf                                   # a search begins with one beam
    running[1, 2] = nan
    running[1, 3] = inf
    running[2, :] = -inf                                    # nothing lives
    z[3 * 5 + 1] = -inf                                     # a beam without candidates
    z[3 * 5 + 2] = nan
    z[3 * 5 + 3, 7] = nan
    z[3 * 5 + 4, 9] = inf
    running[4, :] = -3.4e38                                 # scores that swallow z: the order within a beam stays that of z
    done = (rng.random((6, 5)) < 0.3).astype(np.uint8)
    done[0, 0] = 0
    done[5, :] = 2                                          # all have ended: five survivors, then -inf
    for normalise in (False, True):
        for n in (1, 5, 9, 64):
            check(z, running, n, normalise=normalise)
            check(z, running, n, normalise=normalise, done=done, done_token=3)
            check(z, running, n, normalise=normalise, done=done, done_token=0)


def test_scores_far_below_zero_keep_their_order_across_beams():
    z, running, _ = draw(2, 6, 50, "f32", 22)
    running = running - 2.0 ** 20                           # exact in 64 bits, ties in 32
    check(z, running, 30)


def test_offsets_beyond_32_bits():
    V, ld = 130, 1 << 30
    big = torch.zeros(3 * ld + V, dtype=torch.float16, device="cuda")
    scores = big.as_strided((4, V), (ld, 1))
    z, running, _ = draw(2, 2, V, "f16", 23)
    scores.copy_(z)
    a = pcb.beam(scores, running.cuda(), 5)
    ws = torch.empty(pcb.pc_beam_workspace_bytes(a), dtype=torch.uint8, device="cuda")
    out = torch.empty((2, 5), device="cuda"), torch.empty((2, 5), dtype=torch.int32, device="cuda"), torch.empty((2, 5), dtype=torch.int32, device="cuda")
    pcb.pc_beam_select(a, ws, *out)
    want = reference(z, running, 5)
    assert np.array_equal(out[1].cpu().numpy(), want[1]) and np.array_equal(out[2].cpu().numpy(), want[2])


@pytest.mark.parametrize("G,W,n", [(1, 1, 1), (3, 4, 8), (100, 5, 5), (2, 64, 64)])
def test_states_follow_their_beams(G, W, n):
    """Rows of every alignment, odd lengths, strided; the bytes between rows of dst stay."""
    rng = np.random.default_rng(31)
    parents = torch.from_numpy(rng.integers(0, W, (G, n)).astype(np.int32)).cuda()
    row = (torch.arange(G, device="cuda")[:, None] * W + parents.long()).reshape(-1)
    states, want = [], []
    for shape, dtype, pad, off in [((32,), torch.int32, 0, 0), ((33,), torch.uint8, 3, 1), ((1,), torch.uint8, 0, 0), ((257,), torch.float16, 1, 1), ((3, 5, 7), torch.float32, 0, 0),
                                   ((4096,), torch.float32, 4, 0), ((1025,), torch.int64, 1, 0), ((6000,), torch.bfloat16, 8, 8)]:
        m = int(np.prod(shape))
        src = torch.from_numpy(rng.integers(0, 100, (G * W, m + pad + off))).to(dtype).cuda()
        dst = torch.full((G * n, m + pad + off), 77, dtype=dtype, device="cuda")
        expect = dst.clone()
        expect[:, off:off + m] = src[row, off:off + m]
        if len(shape) == 1:
            states.append((src[:, off:off + m], dst[:, off:off + m]))
        else:
            states.append((src.view(G * W, *shape), dst.view(G * n, *shape)))
        want.append((dst, expect))
    pcb.pc_beam_reorder(states, parents, W)
    for got, expect in want:
        assert torch.equal(got, expect)


def test_parents_out_of_range_leave_their_rows():
    src, dst = torch.arange(12, device="cuda").view(4, 3), torch.full((6, 3), 9, device="cuda")
    parents = torch.tensor([[1, -1, 0], [2, 1, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")
    pcb.pc_beam_reorder([(src, dst)], parents, 2)
    assert dst.tolist() == [[3, 4, 5], [9, 9, 9], [0, 1, 2], [9, 9, 9], [9, 9, 9], [9, 9, 9]][:4] + [[9, 10, 11], [9, 9, 9]]


def test_no_groups():
    out = torch.empty((0, 3), device="cuda"), torch.empty((0, 3), dtype=torch.int32, device="cuda"), torch.empty((0, 3), dtype=torch.int32, device="cuda")
    a = pcb.beam(torch.empty((0, 9), device="cuda"), torch.empty((0, 2), device="cuda"), 3)
    pcb.pc_beam_select(a, torch.empty(pcb.pc_beam_workspace_bytes(a), dtype=torch.uint8, device="cuda"), *out)
    pcb.pc_beam_reorder([(torch.empty((0, 4), device="cuda"), torch.empty((0, 4), device="cuda"))], out[1], 2)


@pytest.mark.parametrize("G,W,V,n", [(1, 4, 50257, 8), (40, 8, 300, 16)])
def test_captured_and_replayed(G, W, V, n):
    z, running, _ = draw(G, W, V, "f32", 41)
    z, running = z.cuda(), running.cuda()
    a = pcb.beam(z, running, n, normalise=True)
    ws = torch.empty(pcb.pc_beam_workspace_bytes(a), dtype=torch.uint8, device="cuda")
    scores, parents, tokens = torch.empty((G, n), device="cuda"), torch.empty((G, n), dtype=torch.int32, device="cuda"), torch.empty((G, n), dtype=torch.int32, device="cuda")
    src = torch.randint(0, 99, (G * W, 50), device="cuda")
    dst = torch.empty((G * n, 50), dtype=torch.int64, device="cuda")

    def step():
        pcb.pc_beam_select(a, ws, scores, parents, tokens)
        pcb.pc_beam_reorder([(src, dst)], parents, W)
        return scores, parents, tokens, dst

    replayed(step, lambda: (z.copy_(torch.roll(z, 1, 1) * 1.01), src.add_(1)))


def test_two_searches_at_once_with_a_workspace_each():
    cases = []
    for seed in (51, 52):
        z, running, _ = draw(8, 4, 20011, "bf16", seed)
        a = pcb.beam(z.cuda(), running.cuda(), 8)
        out = torch.empty((8, 8), device="cuda"), torch.empty((8, 8), dtype=torch.int32, device="cuda"), torch.empty((8, 8), dtype=torch.int32, device="cuda")
        cases.append((a, torch.empty(pcb.pc_beam_workspace_bytes(a), dtype=torch.uint8, device="cuda"), out, reference(z, running, 8)))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (a, ws, out, _) in zip(streams, cases):
            pcb.pc_beam_select(a, ws, *out, stream=s)
    torch.cuda.synchronize()
    for _, _, out, want in cases:
        assert np.array_equal(out[1].cpu().numpy(), want[1]) and np.array_equal(out[2].cpu().numpy(), want[2])
