"""What predictions may lose, on samples of which a few states carry all the weight, so that errors of products do not average out over states.

Operands are three bf16 planes x0 + x1 + x2, each the rounding of what the ones before leave (at most 2^-8 of it): the remainder is 2^-24 of x.  Of the
nine products of planes the six down to 2^-16 are taken; those left out are x1 y2, x2 y1 (2^-24 each) and smaller.  With either operand's remainder a
product is off by at most 4 * 2^-24 = 2^-22 of itself.  A sum of TERMS states is 6 TERMS additions in fp32, 2^-24 of it each.  The logarithm adds 3 * 2^-24
of itself: the device's logf differs from the logarithm in 64 bits by at most 2.72 * 2^-24 of it, taken over every float from FLT_MIN to 1 (a first version of this
bound allowed it 2^-23, which the four cases with fp32 products missed by up to 1.4).  The fp32 kernels (blocks of fewer than four states; one sample of many categories) round each product and addition once.

Here on the CPU: the same arithmetic with two planes and three products misses that bound by far, with three planes it holds it, so that the bound tells
the two apart."""
import numpy as np
import pytest

TERMS = 3


def inputs(K, n_blocks, V, B, seed):
    """Weights [H, B] with TERMS states a sample, one of them at 0.9 and more; tables [n_blocks, V, K], half of each node's mass on one category."""
    rng = np.random.default_rng(seed)
    H = K * n_blocks
    w = np.zeros((H, B), np.float32)
    for b in range(B):
        some = rng.permutation(H)[:TERMS]
        share = rng.random(len(some)) * 0.05
        share[0] = 1 - share[1:].sum()
        w[some, b] = share
    t = rng.exponential(size=(n_blocks, V, K)) ** 2
    t /= t.sum(1, keepdims=True)
    t *= 0.5
    np.put_along_axis(t, rng.integers(0, V, (n_blocks, 1, K)), 0.5 + 0.45 * rng.random((n_blocks, 1, K)), 1)
    return w, t.astype(np.float32)


def log_p(w, t):
    """[B, V] in 64 bits."""
    nb, V, K = t.shape
    p = sum(w[j * K:(j + 1) * K].T.astype(np.float64) @ t[j].T.astype(np.float64) for j in range(nb))
    with np.errstate(divide="ignore"):
        return np.log(p)


def tolerance(want, fp32):
    return (2.0 ** -24 * (1 + TERMS) if fp32 else 2.0 ** -22 + 6 * TERMS * 2.0 ** -24) + 3 * 2.0 ** -24 * np.abs(want)


def bf16(x):
    """To nearest, ties to even."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)


def split(x, planes):
    out = []
    for _ in range(planes):
        out.append(bf16(x))
        x = (x - out[-1]).astype(np.float32)
    return [p.astype(np.float64) for p in out]


@pytest.mark.parametrize("K,nb,V,B", [(32, 1, 300, 20), (128, 4, 5000, 6)])
def test_bound_tells_two_planes_from_three(K, nb, V, B):
    w, t = inputs(K, nb, V, B, 1)
    want, worst = log_p(w, t), {}
    for planes in (2, 3):
        p = 0.0
        for j in range(nb):
            a, b = split(w[j * K:(j + 1) * K] * np.float32(2.0 ** 24), planes), split(t[j] * np.float32(2.0 ** 24), planes)
            p = p + sum(a[i].T @ b[k].T for i in range(planes) for k in range(planes - i))
        worst[planes] = np.max(np.abs(np.log(p * 2.0 ** -48) - want) / tolerance(want, False))
    assert worst[2] > 5.0 and worst[3] < 0.5, worst
