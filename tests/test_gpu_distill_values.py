"""Distillation of `normalised` rows that hold no log-probabilities where they are listed: the loss says so, the gradient, which is -q and reads
nothing of the row, does not depend on it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2406_00766_amd import binding as pcb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V,top", [(40, 5), (9001, 5), (700, 70)])
def test_normalised_rows_with_listed_infinities(dtype, V, top):
    rng = np.random.default_rng(1)
    ids = np.stack([rng.permutation(V)[:top] for _ in range(6)]).astype(np.int32)
    z = torch.log_softmax(torch.from_numpy(rng.normal(size=(6, V))), 1).to(dtype)
    free = [int(np.setdiff1d(np.arange(V), ids[r])[0]) for r in range(6)]
    z[0, ids[0, 2]] = float("inf")
    z[1, ids[1, 0]] = float("nan")
    z[2, ids[2, 1]] = -float("inf")
    z[3, free[3]] = float("inf")                           # not listed
    z[4, free[4]] = float("nan")
    t = torch.from_numpy(rng.normal(size=(6, top)).astype(np.float32))
    d = pcb.distill(z.cuda(), torch.from_numpy(ids).cuda(), t.cuda(), normalised=True)
    loss, stats, grad = torch.empty(6, device="cuda"), torch.empty((6, 2), device="cuda"), torch.empty((6, V), dtype=dtype, device="cuda")
    pcb.pc_distill_forward(d, None, loss, stats)
    pcb.pc_distill_backward(d, stats, None, 1.0, grad)
    loss = loss.cpu().numpy()
    assert np.isnan(loss[[0, 1]]).all() and np.isposinf(loss[2]) and np.isfinite(loss[3:]).all(), loss
    want = np.zeros((6, V))
    np.put_along_axis(want, ids.astype(np.int64), -torch.softmax(t.double(), 1).numpy(), 1)
    # a few roundings of exponentials of arguments below 8 (16 units of 2^-24 each, and the list's sum), then the type's own half step
    err = np.abs(grad.double().cpu().numpy() - want)
    assert np.all(err <= np.abs(want) * (torch.finfo(dtype).eps / 2 + (32 + top) * 2.0 ** -24) + 2.0 ** -25)
