"""A token model's whole use: an HMM predicts its next token, is distilled from a teacher's lists by EM, and decodes with beams; and what the
Python layer refuses on the GPU."""
import itertools

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import pc_oracle as orc
from paper_2406_00766_amd import binding as pcb
from paper_2406_00766_amd import workloads as W

pytestmark = pytest.mark.gpu


def test_beam_search_over_an_hmm_finds_the_best_sequences():
    """With as many beams as prefixes nothing is lost, so the survivors are the most probable of all sequences in order, and
    their scores the sequences' log-likelihoods (tolerance of a path: 1e-4 relative, summed over the tokens)."""
    T, V = 4, 4
    w = W.hmm(T, 32, V, 32, 1, 71, alpha_trans=0.3, alpha_emis=0.3)
    c = pcb.Circuit(w)
    n = 64
    x = np.zeros((n, T), np.int32)
    mask = np.ones((n, T), np.uint8)
    c.set_batch(x, mask)
    running = torch.full((1, n), -float("inf"), device="cuda")
    running[0, 0] = 0.0
    scores, parents, tokens = torch.empty((1, n), device="cuda"), torch.empty((1, n), dtype=torch.int32, device="cuda"), torch.empty((1, n), dtype=torch.int32, device="cuda")
    spare = torch.empty_like(c.x)
    for t in range(T):
        c.forward()
        c.backward(theta_flow=False, table_flow=False)
        a = pcb.beam(c.predict(t), running, n)
        ws = torch.empty(pcb.pc_beam_workspace_bytes(a), dtype=torch.uint8, device="cuda")
        pcb.pc_beam_select(a, ws, scores, parents, tokens)
        pcb.pc_beam_reorder([(c.x, spare)], parents, n)
        c.x.copy_(spare)
        c.x[:, t] = tokens[0]
        c.mask[:, t] = 0
        running.copy_(scores)
    every = np.array(list(itertools.product(range(V), repeat=T)), dtype=np.int32)
    ll = orc.forward(w.with_batch(every), w.theta, w.tables, every)[1]
    order = np.argsort(-ll, kind="stable")[:n]
    got = scores[0].double().cpu().numpy()
    assert np.all(np.abs(got - ll[order]) <= 1e-4 * np.abs(ll[order]) + 1e-5)
    found = c.x.cpu().numpy()
    index = {tuple(s): i for i, s in enumerate(every)}
    assert np.all(np.abs(ll[[index[tuple(s)] for s in found]] - got) <= 1e-4 * np.abs(got) + 1e-5) and len({tuple(s) for s in found}) == n
    c.close()


def test_distillation_by_em_takes_the_step_that_the_formulas_say():
    """One EM step on soft targets for the last token: new emissions = normalised flows T sum_b F q / p, from the oracle's node
    values in 64 bits.  The flows carry the path's own tolerance (1e-3 relative)."""
    T, H, V, B, top = 5, 64, 40, 33, 7
    w = W.hmm(T, H, V, 32, B, 72)
    c = pcb.Circuit(w)
    mask = np.zeros(w.x.shape, np.uint8)
    mask[:, T - 1] = 1
    c.set_batch(w.x, mask)
    rng = np.random.default_rng(5)
    ids = np.stack([rng.permutation(V)[:top] for _ in range(B)]).astype(np.int32)
    teacher = rng.normal(size=(B, top)).astype(np.float32)
    c.forward()
    c.backward(theta_flow=False, table_flow=False)
    logp = c.predict(T - 1)
    d = pcb.distill(logp, torch.from_numpy(ids).cuda(), torch.from_numpy(teacher).cuda(), normalised=True)
    loss, stats, grad = torch.empty(B, device="cuda"), torch.empty((B, 2), device="cuda"), torch.empty_like(logp)
    pcb.pc_distill_forward(d, torch.empty(max(16, pcb.pc_distill_workspace_bytes(d)), dtype=torch.uint8, device="cuda"), loss, stats)
    pcb.pc_distill_backward(d, stats, None, 1.0, grad)
    c.predict_backward(T - 1, logp, grad, scale=-1.0)
    theta = c.theta.clone()
    c.em_step()
    # the same in 64 bits: F of the last variable's input nodes, by block
    _, _, flow, _, _ = orc.backward(w, w.theta, w.tables, w.x, mask)
    F = flow.reshape(B, w.n_blocks, w.K)
    blocks = [u for u in range(w.n_blocks) if w.type[u] == W.INPUT and w.in_var[u] == T - 1]
    tables = w.tables.astype(np.float64)
    p = sum(F[:, u] @ tables[w.in_table[u]].T for u in blocks)
    q = np.exp(teacher.astype(np.float64))
    q /= q.sum(1, keepdims=True)
    dense = np.zeros((B, V))
    np.put_along_axis(dense, ids.astype(np.int64), q, 1)
    want_loss = np.sum(q * (np.log(q) - np.log(np.take_along_axis(p, ids.astype(np.int64), 1))), 1)
    assert np.all(np.abs(loss.double().cpu().numpy() - want_loss) <= 1e-3)
    new = c.tables.double().cpu().numpy().reshape(tables.shape)
    for u in blocks:
        t = w.in_table[u]
        f = tables[t] * ((dense / p).T @ F[:, u])
        want = f / f.sum(0)
        assert np.all(np.abs(new[t] - want) <= 2e-3 * want + 1e-7)
    assert torch.equal(c.theta, theta)                     # no flows there, so rows stay
    c.close()


def test_gradient_of_logits_reaches_the_tables():
    """Temperature 2, dense gradients: predict, loss, gradient and flows against differences of the loss in log tables (64 bits)."""
    K, nb, V, B, top, T = 16, 2, 12, 6, 4, 2.0
    rng = np.random.default_rng(6)
    w = rng.random((K * nb, B)).astype(np.float32)
    w /= w.sum(0)
    t = rng.random((nb, V, K)).astype(np.float32)
    t /= t.sum(1, keepdims=True)
    ids = np.stack([rng.permutation(V)[:top] for _ in range(B)])
    teacher = rng.normal(size=(B, top)).astype(np.float32)

    def objective(tables):
        p = sum(w[j * K:(j + 1) * K].T.astype(np.float64) @ tables[j].T for j in range(nb))
        z = np.log(p) / T
        z -= np.log(np.exp(z).sum(1, keepdims=True))
        q = np.exp(teacher.astype(np.float64) / T)
        q /= q.sum(1, keepdims=True)
        return float(np.sum(q * (np.log(q) - np.take_along_axis(z, ids, 1))))

    m, tables = pcb.mixture(torch.from_numpy(w).cuda(), K, V, nb), torch.from_numpy(t).cuda()
    logp = torch.empty((B, V), device="cuda")
    pcb.pc_predict(m, tables, B, logp)
    d = pcb.distill(logp, torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(teacher).cuda(), temperature=T)
    loss, stats, grad, flow = torch.empty(B, device="cuda"), torch.empty((B, 2), device="cuda"), torch.empty_like(logp), torch.zeros_like(tables)
    pcb.pc_distill_forward(d, torch.empty(max(16, pcb.pc_distill_workspace_bytes(d)), dtype=torch.uint8, device="cuda"), loss, stats)
    assert abs(float(loss.double().sum()) - objective(t.astype(np.float64))) <= 1e-4
    pcb.pc_distill_backward(d, stats, None, 1.0, grad)
    pcb.pc_predict_backward(m, tables, B, logp, grad, 1.0, flow)
    got, eps = flow.cpu().numpy(), 1e-4
    for at in [(0, 0, 0), (1, 11, 15), (0, 5, 9), (1, int(ids[2, 1]), 3)]:
        up, down = t.astype(np.float64), t.astype(np.float64)
        up[at] *= np.exp(eps)
        down[at] *= np.exp(-eps)
        assert abs((objective(up) - objective(down)) / (2 * eps) - got[at]) <= 1e-4


def test_tensors_that_do_not_fit_are_refused():
    f = lambda *s: torch.zeros(s, device="cuda")
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    m = pcb.mixture(f(64, 8), 32, 5, 2)
    d = pcb.distill(f(3, 9), i(3, 2), f(3, 2))
    a = pcb.beam(f(6, 9), f(2, 3), 4)
    u8 = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    bad = [lambda: pcb.mixture(f(64, 8).double(), 32, 5, 2), lambda: pcb.mixture(f(64, 8).t(), 32, 5, 2), lambda: pcb.mixture(f(64, 8), 32, 5, 2, rows=i(3)),
           lambda: pcb.mixture(f(64, 8), 32, 5, 2, rows=f(2)), lambda: pcb.mixture(f(1, 8).expand(64, 8), 32, 5, 2), lambda: pcb.mixture([1.0], 32, 5, 2),
           lambda: pcb.pc_predict(m, f(2, 5, 31), 8, f(8, 5)), lambda: pcb.pc_predict(m, f(2, 5, 32), 9, f(9, 5)), lambda: pcb.pc_predict(m, f(2, 5, 32), 8, f(7, 5)),
           lambda: pcb.pc_predict(m, f(2, 5, 32), 8, f(5, 8).t()), lambda: pcb.pc_predict(m, f(2, 32, 5).transpose(1, 2), 8, f(8, 5)),
           lambda: pcb.pc_predict(pcb.mixture(f(63, 8), 32, 5, 2), f(2, 5, 32), 8, f(8, 5)),
           lambda: pcb.pc_predict_backward(m, f(2, 5, 32), 8, f(8, 5), f(8, 4), 1.0, f(2, 5, 32)), lambda: pcb.pc_predict_backward(m, f(2, 5, 32), 8, f(8, 5), f(8, 5), 1.0, f(2, 5, 16)),
           lambda: pcb.distill(f(3, 9).double(), i(3, 2), f(3, 2)), lambda: pcb.distill(f(3, 9), i(3, 2).long(), f(3, 2)), lambda: pcb.distill(f(3, 9), i(3, 2), f(3, 1)),
           lambda: pcb.distill(f(3, 9), i(2, 2), f(2, 2)), lambda: pcb.distill(f(3, 9), i(3, 2), f(3, 2), teacher_lse=f(2)),
           lambda: pcb.pc_distill_forward(d, u8, f(2), f(3, 2)), lambda: pcb.pc_distill_forward(d, u8, f(3), f(3, 3)), lambda: pcb.pc_distill_backward(d, f(3, 2), f(2), 1.0, f(3, 9)),
           lambda: pcb.pc_distill_backward(d, f(3, 2), None, 1.0, f(3, 9).half()), lambda: pcb.pc_distill_backward(d, f(3, 2), None, 1.0, f(3, 8)),
           lambda: pcb.beam(f(6, 9), f(2, 2), 4), lambda: pcb.beam(f(6, 9), f(3, 2).t(), 4), lambda: pcb.beam(f(6, 9), f(2, 3), 4, done=f(2, 3)), lambda: pcb.beam(i(6, 9), f(2, 3), 4),
           lambda: pcb.pc_beam_select(a, u8[:8], f(2, 4), i(2, 4), i(2, 4)), lambda: pcb.pc_beam_select(a, u8, f(2, 3), i(2, 4), i(2, 4)), lambda: pcb.pc_beam_select(a, u8, f(2, 4), f(2, 4), i(2, 4)),
           lambda: pcb.pc_beam_reorder([], i(2, 4), 3), lambda: pcb.pc_beam_reorder([(f(6, 2), f(7, 2))], i(2, 4), 3), lambda: pcb.pc_beam_reorder([(f(6, 2), f(8, 3))], i(2, 4), 3),
           lambda: pcb.pc_beam_reorder([(f(6, 2), i(8, 2))], i(2, 4), 3), lambda: pcb.pc_beam_reorder([(f(2, 6).t(), f(8, 2))], i(2, 4), 3),
           lambda: pcb.pc_beam_reorder([(f(8, 2)[:6], f(1, 2).expand(8, 2))], i(2, 4), 3)]
    for k, call in enumerate(bad):
        with pytest.raises(pcb.PcError) as e:
            call()
        assert e.value.status_name in ("PC_ERR_ARG", "PC_ERR_WORKSPACE"), k
