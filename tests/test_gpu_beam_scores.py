"""How near pc_beam_select's scores come to running + z - log sum exp(z): with a running score that nearly cancels z - log sum exp(z) the sum,
which is taken in 64 bits, shows the normaliser's own error and hardly any rounding.

Tolerance, relative to the sum of exponentials, in units of u = 2^-24.  An exponential is taken in fp32 from a difference d to a reference that lies at
most 8 below the maximum so far: its argument d log2(e) is off by 1.5 u |d| (one rounding, and the constant's), the instruction adds 2 u.  Up to 32 of them
are added in fp32 (31 u), everything after that in 64 bits but for the factors from one reference to the next, where the maximum has risen by more than 8,
and at last to the row's: 1.5 u of each distance and 2 u again.  For an entry the distances add up to at most |z - max| + 16, and it meets at most that / 8
factors: 1.75 |z - max| + 24 + 4 + 4 + 31 in all.  No term grows with the row's length."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2406_00766_amd import binding as pcb

pytestmark = pytest.mark.gpu


def bound(row):
    a = row - row.max()
    e = np.exp(a)
    return 2.0 ** -24 * (1.75 * np.sum(np.where(e > 0, np.abs(a) * e, 0)) / np.sum(e) + 63)


def check(row, dtype, rows):
    """`rows` groups of one beam with the same row each (so many that a row is one workgroup's, or few, of which several share one)."""
    V = len(row)
    held = torch.from_numpy(row).to(dtype)
    z64 = held.double().numpy()
    best = int(np.argmax(z64))
    lse = z64.max() + np.log(np.sum(np.exp(z64 - z64.max())))
    running = np.float32(lse - z64[best])
    scores = torch.empty((rows, V), dtype=dtype, device="cuda")
    scores[:] = held.cuda()
    a = pcb.beam(scores, torch.full((rows, 1), float(running), device="cuda"), 1, normalise=True)
    out = torch.empty((rows, 1), device="cuda"), torch.empty((rows, 1), dtype=torch.int32, device="cuda"), torch.empty((rows, 1), dtype=torch.int32, device="cuda")
    pcb.pc_beam_select(a, torch.empty(pcb.pc_beam_workspace_bytes(a), dtype=torch.uint8, device="cuda"), *out)
    want = np.float64(running) + (z64[best] - lse)
    got = out[0].double().cpu().numpy()
    worst = np.max(np.abs(got - want)) / (bound(z64) + 2.0 ** -24 * abs(want))
    assert worst <= 1.0, worst
    assert bool((out[2] == best).all()) and bool((out[1] == 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,V", [(1, 50257), (3, 1000), (700, 50257), (2, 1000003)])
def test_normalisers_of_random_rows(dtype, rows, V):
    print(f"case normaliser {dtype} rows={rows} V={V}", flush=True)
    check(np.random.default_rng(V).normal(size=V) * 3, dtype, rows)


@pytest.mark.parametrize("V", [50257, 4200000])
def test_errors_of_equal_terms_do_not_add_up_along_a_row(V):
    """Every addition of equal terms rounds the same way; a lane of the longer row adds 512 times 32 of them."""
    print(f"case equal terms V={V}", flush=True)
    row = np.full(V, -float(np.float16(0.96)))
    row[:8200] = 0.0                                       # every lane's maximum
    check(row, torch.float16, 513)


@pytest.mark.parametrize("step", [1e-4, 5e-4, 0.05])
def test_errors_of_rising_maxima_do_not_add_up_along_a_row(step):
    """Rows in ascending order by steps of a chunk: every chunk has a new maximum."""
    V = 2000000
    print(f"case rising step={step}", flush=True)
    check(np.floor(np.arange(V) / 4096) * step, torch.float32, 513)
    far = np.arange(V) / V * 300.0                         # references are left behind many times over
    check(far, torch.float32, 2)


@pytest.mark.parametrize("G,W", [(1, 1), (300, 4), (2000, 7)])
def test_running_scores_replaced_in_place(G, W):
    V = 333
    rng = np.random.default_rng(5)
    z = torch.from_numpy(rng.normal(size=(G * W, V)).astype(np.float32)).cuda()
    running = torch.from_numpy(rng.normal(size=(G, W)).astype(np.float32)).cuda()
    a = pcb.beam(z, running, W, normalise=True)
    ws = torch.empty(pcb.pc_beam_workspace_bytes(a), dtype=torch.uint8, device="cuda")
    want = torch.empty((G, W), device="cuda"), torch.empty((G, W), dtype=torch.int32, device="cuda"), torch.empty((G, W), dtype=torch.int32, device="cuda")
    got = running, torch.empty_like(want[1]), torch.empty_like(want[2])
    pcb.pc_beam_select(a, ws, *want)
    pcb.pc_beam_select(a, ws, *got)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
