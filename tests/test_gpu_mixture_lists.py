"""The input blocks that pc_get_mixture names: all of the variable's, by table, then by offset; and predictions through every backward pass that leaves
node flows (chains that one launch walks, dataflow launches, classes of product blocks), against the oracle's forward pass."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import pc_oracle as orc
from paper_2406_00766_amd import binding as pcb
from paper_2406_00766_amd import workloads as W

pytestmark = pytest.mark.gpu


def ints(address, n):
    """n int32 on the device, copied as the one row of a state."""
    out, parent = torch.empty(n, dtype=torch.int32, device="cuda"), torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    state = pcb.pc_state(address, out.data_ptr(), 4 * n, 4 * n, 4 * n)
    assert pcb.lib().pc_beam_reorder(C.byref(state), 1, parent.data_ptr(), 1, 1, 1, torch.cuda.current_stream().cuda_stream) == pcb.PC_OK
    return out.cpu().numpy()


def ready(w, mask):
    c = pcb.Circuit(w)
    c.set_batch(w.x, mask)
    c.forward()
    c.backward(theta_flow=False, table_flow=False)
    return c


@pytest.mark.parametrize("reverse", [False, True])
def test_blocks_of_a_variable_by_table_then_offset(reverse):
    w = W.rat_spn(16, 2, 2, 32, 16, 5, 4, n_cats=11)
    rng = np.random.default_rng(3)
    inputs = np.flatnonzero(np.asarray(w.type) == W.INPUT)
    w.in_table = np.array(w.in_table, copy=True)
    w.in_table[inputs] = rng.integers(0, len(w.tables), len(inputs))          # tables shared and in no order
    if reverse:
        w.in_table[inputs] = np.sort(w.in_table[inputs])[::-1]
    c = ready(w, np.ones(w.x.shape, np.uint8))
    for v in range(w.n_vars):
        m = pcb.pc_get_mixture(c.handle, v, c.B, c._ws, c._ws.numel()).struct
        mine = [u for u in inputs if w.in_var[u] == v]
        mine.sort(key=lambda u: (w.in_table[u], u))
        assert m.n_blocks == len(mine) and m.n_tables == len(w.tables) and m.n_cats == w.n_cats and m.K == w.K
        assert np.array_equal(ints(m.rows, m.n_blocks), [(u + 1) * w.K for u in mine])
        assert np.array_equal(ints(m.table, m.n_blocks), [w.in_table[u] for u in mine])
    c.close()


@pytest.mark.parametrize("make_w", [lambda: W.hmm(6, 64, 9, 64, 7, 1), lambda: W.hmm(6, 32, 9, 32, 300, 2), lambda: W.hmm(3, 128, 9, 128, 5, 3), lambda: W.hmm(16, 64, 9, 64, 600, 4),
                                    lambda: W.hmm(4, 256, 9, 64, 40, 5), lambda: W.rat_spn(24, 2, 2, 64, 32, 50, 6, n_cats=9), lambda: W.hmm(4, 24, 9, 8, 3, 7)])
def test_conditionals_after_every_kind_of_backward_pass(make_w):
    w = make_w()
    rng = np.random.default_rng(8)
    for v in (0, w.n_vars // 2, w.n_vars - 1):
        mask = (rng.random(w.x.shape) < 0.3).astype(np.uint8)
        mask[:, v] = 1
        c = ready(w, mask)
        print(f"case conditional {w.name} v={v}", flush=True)
        got = np.exp(c.predict(v).double().cpu().numpy())
        rest = orc.forward(w, w.theta, w.tables, w.x, mask)[1]
        seen = mask.copy()
        seen[:, v] = 0
        for cat in (0, w.n_cats - 1):
            x = w.x.copy()
            x[:, v] = cat
            want = np.exp(orc.forward(w.with_batch(x), w.theta, w.tables, x, seen)[1] - rest)
            assert np.all(np.abs(got[:, cat] - want) <= 1e-3 * want + 1e-7), cat
        assert np.all(np.abs(got.sum(1) - 1) <= 1e-3)
        c.close()
