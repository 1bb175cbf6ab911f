"""pc_distill_forward / pc_distill_backward against the formulas in 64 bits: all element types, odd vocabularies and strides, lists
that are short, empty, doubled or out of range, masked and extreme logits, few and many rows; the gradient against
differences of the loss.

Tolerances, in units of u = 2^-24.  exp((z - m) / T) has an argument a that is rounded by 2 u |a| and an error of 2 u itself; |a| e^a < 0.37, so a sum of V
terms is off by at most (2 V' + n) u relative to itself, with V' = (sum of |a| e^a) / (sum of e^a) + 1 taken from the row and n = the
additions in a row (V / 64 on one lane, 64 more across lanes and segments).  A log-probability adds 4 u |logp|, a log q the same
with its own list.  A gradient is rounded once to its type (half a step, or half the smallest subnormal)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2406_00766_amd import binding as pcb
from tests.replay import replayed

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def exact(z, ids, t, T, lse=None, normalised=False):
    """64-bit loss, gradient (before scaling), stats, and the bounds of what fp32 may lose of the loss and of the gradient."""
    z, t = z.double().numpy(), t.double().numpy()
    rows, V = z.shape
    loss, grad, stats = np.zeros(rows), np.zeros((rows, V)), np.zeros((rows, 2))
    loss_tol, grad_tol = np.zeros(rows), np.zeros((rows, V))
    with np.errstate(all="ignore"):
        for r in range(rows):
            on = (ids[r] >= 0) & (ids[r] < V) & ~np.isneginf(t[r])
            at, tt = ids[r][on], t[r][on]
            if normalised:
                logp, spread = z[r].copy(), 0.0
            else:
                m = np.nan if np.isnan(z[r]).any() else z[r].max()
                a = (z[r] - m) / T if np.isfinite(m) else np.where(np.isneginf(z[r]), -np.inf, np.nan) if m != -np.inf else np.full(V, -np.inf)
                s = np.exp(a).sum()
                stats[r] = m, np.log(s)
                spread = 2 * (np.sum(np.where(np.isneginf(a), 0, np.abs(a) * np.exp(a))) / s + 1) + V / 64 + 64 if s > 0 else 0.0
                logp = a - np.log(s) if s > 0 or np.isnan(s) else a
            if not on.any():
                continue
            if lse is None:
                b = (tt - tt.max()) / T
                logq = b - np.log(np.exp(b).sum())
            else:
                logq = tt / T - float(lse[r])
            q = np.exp(logq)
            use = ~(q == 0)
            loss[r] = np.sum(q[use] * (logq[use] - logp[at[use]]))
            err_q = np.where(use, 2 * np.abs(np.where(np.isfinite(logq), logq, 0)) + 4 * (np.abs(tt) / T + 1) + 16, 0.0)
            lp = np.where(np.isfinite(logp), logp, 0.0)
            loss_tol[r] = U * np.sum(q[use] * (err_q[use] * (1 + np.abs(logq[use] - lp[at[use]])) + 8 * np.abs(lp[at[use]]) + spread + len(at)))
            p = np.zeros(V) if normalised else np.where(np.isneginf(logp), 0.0, np.exp(logp))
            g = p * q.sum()
            np.subtract.at(g, at, q)
            grad[r] = g / T
            e = p * q.sum() * (spread + 8 * np.abs(lp) + err_q.max() + len(at) + 8)
            np.add.at(e, at, q * (err_q + 8) + len(at) * q)
            grad_tol[r] = U * e / T
    return np.where(loss > 3.4028235e38, np.inf, loss), grad, stats, loss_tol, grad_tol      # what fp32 does not hold is inf


def step_of(dtype):
    f = torch.finfo(dtype)
    return f.eps / 2, float(f.smallest_normal) * f.eps


def run(z, ids, t, T=1.0, lse=None, normalised=False, scale=1.0, dloss=None, pad=0, in_place=False):
    rows, V = z.shape
    held = torch.full((rows, V + pad), 3.0, dtype=z.dtype, device="cuda")
    held[:, :V] = z.cuda()
    d = pcb.distill(held[:, :V], torch.from_numpy(ids).cuda(), t.cuda(), temperature=T, teacher_lse=None if lse is None else lse.cuda(), normalised=normalised)
    ws = torch.full((max(16, pcb.pc_distill_workspace_bytes(d)),), 255, dtype=torch.uint8, device="cuda")
    loss, stats = torch.full((rows,), 9.0, device="cuda"), torch.full((rows, 2), 9.0, device="cuda")
    pcb.pc_distill_forward(d, ws, loss, stats)
    out = held if in_place else torch.full((rows, V + pad), 5.0, dtype=z.dtype, device="cuda")
    pcb.pc_distill_backward(d, stats, None if dloss is None else dloss.cuda(), scale, out[:, :V])
    assert bool((out[:, V:] == (3.0 if in_place else 5.0)).all()), "columns behind a row are not touched"
    return loss.cpu().double().numpy(), out[:, :V].cpu().double().numpy(), stats.cpu().double().numpy()


def check(z, ids, t, T=1.0, lse=None, normalised=False, scale=1.0, dloss=None, **kw):
    got_loss, got_grad, got_stats = run(z, ids, t, T, lse, normalised, scale, dloss, **kw)
    loss, grad, stats, loss_tol, grad_tol = exact(z, ids, t, T, lse, normalised)
    # A loss within its own tolerance of FLT_MAX may round to inf: sum q_j * FLT_MAX with fp32 q that add up to 1 + n 2^-24 is above
    # FLT_MAX (1 + 2^-25), which rounds to inf.  So for the row of lowest values at T = 1, whose exact loss is FLT_MAX itself.
    edge = np.isfinite(loss) & np.isposinf(got_loss) & (loss + loss_tol > 3.4028235e38)
    got_loss = np.where(edge, loss, got_loss)
    fin = np.isfinite(loss)
    assert np.array_equal(got_loss[~fin], loss[~fin], equal_nan=True)
    assert np.all(np.abs(got_loss[fin] - loss[fin]) <= loss_tol[fin] + 1e-37), np.max(np.abs(got_loss[fin] - loss[fin]) / (loss_tol[fin] + 1e-37))
    if not normalised:
        assert np.array_equal(got_stats[:, 0], stats[:, 0], equal_nan=True)
    factor = scale * (np.ones(len(loss)) if dloss is None else dloss.double().numpy())[:, None]
    half, tiny = step_of(z.dtype)
    with np.errstate(all="ignore"):
        want = np.where(factor == 0, 0.0, grad * factor)
        tol = grad_tol * np.abs(factor) * (1 + half) + half * np.abs(want) + tiny
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got_grad), np.isnan(want))
    assert np.all(np.abs(got_grad[fin] - want[fin]) <= tol[fin]), np.max(np.abs(got_grad[fin] - want[fin]) / tol[fin])
    return got_loss, got_grad


def inputs(rows, V, top, student, teacher, seed, spread=2.0):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy(rng.normal(size=(rows, V)) * spread).to(TYPES[student])
    ids = np.stack([rng.permutation(V)[:top] if top <= V else rng.integers(0, V, top) for _ in range(rows)]).astype(np.int32)
    t = torch.from_numpy(rng.normal(size=(rows, top)) * 2 + 8).to(TYPES[teacher])
    return z, ids, t, rng


@pytest.mark.parametrize("student,teacher", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f16"), ("f16", "f32"), ("f16", "f16"), ("f32", "f16"),
                                             ("bf16", "f32"), ("f16", "bf16")])
@pytest.mark.parametrize("rows,V,top,pad,T", [(1, 1, 1, 0, 1.0), (2, 3, 2, 1, 0.5), (5, 63, 7, 2, 2.0), (3, 1025, 64, 0, 1.0), (2, 50257, 33, 3, 4.0), (300, 517, 5, 8, 1.0)])
def test_loss_and_gradient_match_64_bits(student, teacher, rows, V, top, pad, T):
    print(f"case distill {student} {teacher} rows={rows} V={V} top={top} T={T}", flush=True)
    z, ids, t, rng = inputs(rows, V, top, student, teacher, rows + V)
    check(z, ids, t, T, scale=0.75, dloss=torch.from_numpy(rng.random(rows).astype(np.float32)), pad=pad)


@pytest.mark.parametrize("rows,V", [(1, 200003), (7, 30011), (40, 9001), (1100, 260), (3000, 40)])
def test_few_long_and_many_short_rows(rows, V):
    print(f"case distill rows={rows} V={V}", flush=True)
    z, ids, t, _ = inputs(rows, V, 20, "f32", "f32", V)
    check(z, ids, t, 1.0, pad=1)


@pytest.mark.parametrize("student", list(TYPES))
def test_lists_that_are_short_empty_doubled_or_out_of_range(student):
    rows, V, top = 9, 700, 40
    z, ids, t, rng = inputs(rows, V, top, student, "f32", 3)
    ids[0, :] = -1                                         # no entry
    ids[1, 1:] = -1                                        # one entry
    ids[2, 5:9] = [V, V + 1, 2 ** 31 - 1, -2 ** 31]        # outside
    ids[3, :] = ids[3, 0]                                  # one category forty times
    ids[4, 20:] = ids[4, :20]
    t[5, :] = -float("inf")                                # no entry either
    t[6, 3] = -float("inf")
    t[7, :] = torch.finfo(torch.float32).min
    t[7, 2] = 0.0
    loss, grad = check(z, ids, t, 0.5)
    assert loss[0] == 0 and np.all(grad[0] == 0) and loss[5] == 0 and np.all(grad[5] == 0)
    lse = torch.logsumexp(t.double(), 1).float() + 0.25
    lse[5] = 0.0
    lse[7] = 1.0
    check(z, ids, t, 1.0, lse=lse)


@pytest.mark.parametrize("student", list(TYPES))
@pytest.mark.parametrize("T", [0.25, 1.0, 8.0])
def test_masked_and_extreme_student_logits(student, T):
    low, inf = torch.finfo(TYPES[student]).min, float("inf")
    rows, V, top = 9, 1500, 6
    z, ids, t, rng = inputs(rows, V, top, student, "f32", 4)
    z[0, rng.random(V) < 0.5] = -inf
    z[0, ids[0]] = 0.0
    z[1, :] = low                                          # uniform
    z[2, :] = low
    z[2, 11] = 1.0
    z[3, :] = -inf                                         # nothing left: p = 0 everywhere, loss +inf
    z[4, ids[4, 1]] = -inf                                 # listed and excluded
    z[5, 3] = inf
    z[6, 1400] = float("nan")
    z[7, :] = -inf
    z[7, 900] = 2.0
    ids[7, :] = [900, -1, -1, -1, -1, -1]                  # one category left, and it is listed: loss 0
    z[8, :] = float("nan")
    ids[8, :] = -1                                         # no entry: 0 whatever the row holds
    loss, grad = check(z, ids, t, T)
    assert np.isposinf(loss[[3, 4]]).all() and np.isnan(loss[[5, 6]]).all() and loss[7] == 0 and loss[8] == 0 and np.all(grad[8] == 0)


@pytest.mark.parametrize("student", list(TYPES))
@pytest.mark.parametrize("rows,V,pad,in_place", [(9, 5, 0, False), (9, 70, 1, True), (11, 4001, 3, False), (11, 8501, 3, True), (530, 8501, 1, False), (530, 8501, 7, True), (515, 8504, 0, False)])
def test_ends_of_rows(student, rows, V, pad, in_place):
    """The elements in no whole 16-byte pack, in rows that start at every offset; one, four and sixteen waves a row."""
    print(f"case ends {student} rows={rows} V={V} pad={pad}", flush=True)
    inf = float("inf")
    z, ids, t, rng = inputs(rows, V, 4, student, "f32", V + pad)
    ids[:, 0], ids[:, 1] = 0, V - 1
    z[0, 0] = 30.0
    z[1, V - 1] = 30.0
    z[2, 0] = float("nan")
    z[3, V - 1] = float("nan")
    z[4, V - 1] = inf
    z[5, 0] = z[5, V - 1] = -inf
    z[6, :] = -inf
    z[6, V - 1] = -4.0                                     # the one category left
    ids[6, :] = [V - 1, -1, -1, -1]
    z[7, :] = -inf
    z[7, 0] = 5.0
    ids[7, :] = [0, -1, -1, V]
    z[8, :] = -inf
    loss, _ = check(z, ids, t, 2.0, pad=pad, in_place=in_place, dloss=torch.from_numpy(rng.random(rows).astype(np.float32) + 0.5))
    assert np.isnan(loss[[2, 3, 4]]).all() and np.isposinf(loss[[5, 8]]).all() and loss[6] == 0 and loss[7] == 0


def test_rows_of_nan_alone_and_teachers_that_are_no_numbers():
    z, ids, t, _ = inputs(4, 90, 5, "f32", "f32", 6)
    z[0, :] = float("nan")
    t[1, 2] = float("nan")
    t[2, 2] = float("inf")
    loss, grad, _ = run(z, ids, t)
    assert np.isnan(loss[:3]).all() and np.isnan(grad[:3]).all() and np.isfinite(loss[3]) and np.isfinite(grad[3]).all()


def test_rows_whose_gradient_is_not_wanted():
    z, ids, t, _ = inputs(6, 333, 9, "bf16", "bf16", 7)
    z[2, 5] = float("nan")
    dloss = torch.tensor([1.0, 0.0, 0.0, 2.0, -1.0, 1.0])
    _, grad, _ = run(z, ids, t, dloss=dloss)
    assert np.all(grad[[1, 2]] == 0) and np.isfinite(grad).all() and np.any(grad[0] != 0)


@pytest.mark.parametrize("student,rows,V", [("f32", 5, 700), ("bf16", 3, 40001), ("f16", 600, 300)])
def test_normalised_rows_take_no_softmax(student, rows, V):
    z, ids, t, rng = inputs(rows, V, 12, student, "f32", 8)
    z = torch.log_softmax(z.float(), 1).to(TYPES[student])
    z[0, rng.random(V) < 0.2] = -float("inf")
    z[0, ids[0]] = -3.0
    z[1, (ids[1].max() + 1) % V] = float("nan") if (ids[1].max() + 1) % V not in ids[1] else z[1, 0]
    ids[1, 3] = ids[1, 4]
    loss, grad = check(z, ids, t, 1.0, normalised=True, pad=1)
    assert np.isfinite(loss).all()
    listed = np.zeros((rows, V), bool)
    np.put_along_axis(listed, ids.astype(np.int64), True, 1)
    assert np.all(grad[~listed] == 0) and np.all(np.abs(-grad.sum(1) - 1) <= 12 * 2.0 ** -8)


@pytest.mark.parametrize("student,rows,V", [("f32", 3, 50001), ("bf16", 700, 333), ("f16", 4, 2048)])
def test_gradient_in_place(student, rows, V):
    z, ids, t, _ = inputs(rows, V, 30, student, "bf16", 9)
    check(z, ids, t, 2.0, in_place=True, pad=5)


def test_longest_list():
    z, ids, t, _ = inputs(3, 5000, 1024, "f32", "f32", 10)
    ids[1, 512:] = ids[1, :512]
    check(z, ids, t, 1.0)


def test_offsets_beyond_32_bits():
    """Rows that start behind 2^32 bytes and 2^31 elements."""
    V, ld = 70, 1 << 30
    big = torch.zeros(2 * ld + V, dtype=torch.bfloat16, device="cuda")
    student = big.as_strided((3, V), (ld, 1))
    z, ids, t, _ = inputs(3, V, 4, "bf16", "f32", 11)
    student.copy_(z)
    d = pcb.distill(student, torch.from_numpy(ids).cuda(), t.cuda())
    ws = torch.empty(max(16, pcb.pc_distill_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
    loss, stats = torch.empty(3, device="cuda"), torch.empty((3, 2), device="cuda")
    pcb.pc_distill_forward(d, ws, loss, stats)
    pcb.pc_distill_backward(d, stats, None, 1.0, student)
    want, grad, _, tol, grad_tol = exact(z, ids, t, 1.0)
    assert np.all(np.abs(loss.cpu().double().numpy() - want) <= tol)
    half, tiny = step_of(torch.bfloat16)
    assert np.all(np.abs(student.cpu().double().numpy() - grad) <= grad_tol * (1 + half) + half * np.abs(grad) + tiny)


def test_gradient_against_differences():
    z, ids, t, _ = inputs(2, 40, 6, "f32", "f32", 12)
    ids[1, 3] = ids[1, 2]
    _, grad, _ = run(z, ids, t, T=2.0)
    eps = 1e-4
    for r, c in [(0, int(ids[0, 0])), (0, 7), (1, int(ids[1, 2])), (1, 39)]:
        up, down = z.double().clone(), z.double().clone()
        up[r, c] += eps
        down[r, c] -= eps
        diff = (exact(up, ids, t, 2.0)[0][r] - exact(down, ids, t, 2.0)[0][r]) / (2 * eps)
        assert abs(diff - grad[r, c]) <= 1e-6


def test_no_rows():
    z, ids, t, _ = inputs(1, 8, 2, "f32", "f32", 13)
    run(z[:0], ids[:0], t[:0], dloss=torch.empty(0))


@pytest.mark.parametrize("rows,V", [(2, 40001), (400, 300)])
def test_captured_and_replayed(rows, V):
    z, ids, t, _ = inputs(rows, V, 16, "f32", "f32", 14)
    z, t = z.cuda(), t.cuda()
    d = pcb.distill(z, torch.from_numpy(ids).cuda(), t)
    ws = torch.empty(max(16, pcb.pc_distill_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
    loss, stats, grad = torch.empty(rows, device="cuda"), torch.empty((rows, 2), device="cuda"), torch.empty_like(z)

    def step():
        pcb.pc_distill_forward(d, ws, loss, stats)
        pcb.pc_distill_backward(d, stats, None, 0.5, grad)
        return loss, stats, grad

    replayed(step, lambda: (z.copy_(torch.roll(z, 1, 1)), t.mul_(0.9)))


def test_same_results_on_every_run():
    z, ids, t, _ = inputs(3, 50257, 64, "f32", "f32", 15)
    first = run(z, ids, t)
    for _ in range(3):
        again = run(z, ids, t)
        assert all(np.array_equal(a, b) for a, b in zip(first, again))
