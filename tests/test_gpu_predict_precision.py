"""pc_predict holds the bound of tests/test_plane_precision.py on every path: states of all block lengths, one sample to several widths of a
wave, few categories and many, states in parts, a batch in two launches; and a sample's log-probabilities do not depend on the batch it is in beyond it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2406_00766_amd import binding as pcb
from tests.test_plane_precision import inputs, log_p, tolerance

pytestmark = pytest.mark.gpu


def predict(w, t, B):
    nb, V, K = t.shape
    out = torch.empty((B, V), device="cuda")
    pcb.pc_predict(pcb.mixture(torch.from_numpy(w).cuda(), K, V, nb), torch.from_numpy(t).cuda(), B, out)
    return out.cpu().numpy().astype(np.float64)


def check(got, want, fp32=False):
    none = np.isneginf(want)
    assert np.array_equal(np.isneginf(got), none)
    worst = np.max(np.abs(got - want)[~none] / tolerance(want[~none], fp32))
    assert worst <= 1.0, worst


@pytest.mark.parametrize("K,nb,V,B,fp32", [
    (3, 40, 90, 70, True), (1, 7, 5000, 2, True),                              # blocks of fewer than four states
    (128, 2, 9001, 1, True), (33, 3, 40000, 1, True),                          # one sample of many categories
    (32, 3, 300, 20, False), (128, 2, 4095, 33, False), (20, 5, 1000, 1, False), (64, 2, 256, 257, False), (128, 2, 1000, 1200, False), (48, 3, 4000, 520, False),
    (128, 16, 300, 260, False), (128, 8, 40, 1, False),                        # states in parts
    (128, 2, 4096, 16, False), (64, 3, 50257, 20, False), (33, 4, 33000, 5, False), (128, 16, 33000, 21, False),
    (32, 4, 33000, 40, False), (20, 3, 32800, 100, False), (128, 4, 33000, 90, False), (96, 9, 30001, 31, False),
    (32, 4, 33000, 200, False), (20, 5, 33000, 300, False), (128, 3, 50257, 256, False), (36, 3, 33000, 257, False), (32, 2, 40001, 640, False), (100, 8, 5000, 260, False)])
def test_few_states_carry_a_sample(K, nb, V, B, fp32):
    print(f"case precision K={K} blocks={nb} V={V} B={B}", flush=True)
    w, t = inputs(K, nb, V, B, K + V + B)
    check(predict(w, t, B), log_p(w, t), fp32)


def test_log_probabilities_do_not_depend_on_the_batch():
    """Two answers for a sample lie within both bounds of each other, whichever kernels give them: one sample, a few, a batch in two launches."""
    w, t = inputs(128, 3, 33000, 257, 4)
    want = log_p(w, t)
    whole = predict(w, t, 257)
    for first, n in ((0, 1), (256, 1), (0, 2), (200, 40), (100, 130)):
        got = predict(np.ascontiguousarray(w[:, first:first + n]), t, n)
        check(got, want[first:first + n])
        assert np.max(np.abs(got - whole[first:first + n]) / tolerance(want[first:first + n], False)) <= 2.0
