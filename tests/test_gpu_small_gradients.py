"""pc_predict_backward where gradients and table entries are tiny together: a softmax leaves a gradient of about p for a category of probability
p, and its flow T sum W g / p is then of the order of T, which fp32 holds to 2^-24 as long as T is a normal number.

Tolerance.  Operands are kept to 2^-23 each, a term is off by at most 2^-22 of itself and (n + 32) * 2^-24 covers that and n additions; no
floor besides the last step of the smallest numbers (2^-149, four of them), for all flows here are normal numbers."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2406_00766_amd import binding as pcb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K,nb,V,B,share", [(K, nb, V, B, share) for K, nb, V in [(4, 1, 5), (32, 2, 66)]
                                            for B, share in [(3, 1.0), (70, 1.0), (70, 0.3), (200, 1.0), (200, 0.3), (640, 0.9)]] + [(128, 32, 12100, 640, 0.9)])
def test_flows_of_gradients_as_small_as_their_probabilities(K, nb, V, B, share):
    """Samples that mostly count, and few that do; tiles of 64 x 64 and, where there are thousands of them, of 128 x 128."""
    print(f"case small gradients K={K} blocks={nb} V={V} B={B} share={share}", flush=True)
    rng = np.random.default_rng(B + V)
    H = K * nb
    w = ((rng.random((H, B)) + 0.5) / np.sqrt(H)).astype(np.float32)
    t = rng.random((nb, V, K)) + 0.5
    some = np.array([1, 4] if V < 10 else [1, 2, V - 1])   # p is about sqrt(H) times these, a flow B / sqrt(H) times
    t[:, some, :] *= np.array([1e-36, 3e-37, 1e-30][:len(some)])[None, :, None]
    t = t.astype(np.float32)
    w64, t64 = w.astype(np.float64), t.astype(np.float64)
    p = np.stack([t64[:, c, :].reshape(-1) @ w64 for c in some], 1)            # [B, some]
    logp = np.full((B, V), -3.0, np.float32)
    logp[:, some] = np.log(p)
    assert logp.min() > -87.0                              # nothing is below FLT_MIN
    g = np.zeros((B, V), np.float32)
    g[:, some] = np.exp(logp[:, some].astype(np.float64))
    g[rng.random(B) >= share] = 0.0
    r = g[:, some].astype(np.float64) / np.exp(logp[:, some].astype(np.float64))
    flow = torch.full(t.shape, 9.0, device="cuda")
    pcb.pc_predict_backward(pcb.mixture(torch.from_numpy(w).cuda(), K, V, nb), torch.from_numpy(t).cuda(), B, torch.from_numpy(logp).cuda(),
                            torch.from_numpy(g).cuda(), 1.0, flow, accumulate=False)
    got = flow[:, torch.from_numpy(some).cuda(), :].cpu().numpy().astype(np.float64)
    sums = (w64 @ r).reshape(nb, K, len(some)).transpose(0, 2, 1)
    want = t64[:, some, :] * sums
    assert want.min() > 2.0 ** -126
    tol = (B + 32) * 2.0 ** -24 * want + 4 * 2.0 ** -149
    worst = np.max(np.abs(got - want) / tol)
    assert worst <= 1.0, worst
