"""Refusals of the calls for token models, on the CPU: every bad argument is turned down on the host, before anything is
enqueued (the addresses in these descriptors name no memory)."""
import ctypes as C

import pytest

from paper_2406_00766_amd import binding as pcb
from paper_2406_00766_amd import workloads as W

P = 1 << 20                                                # an aligned address


def status(code):
    return pcb.STATUS_NAMES[code]


def mixture(**kw):
    f = dict(K=32, n_blocks=4, n_cats=10, n_tables=4, n_rows=128, stride=64, weights=P, rows=None, table=None)
    f.update(kw)
    return pcb.pc_mixture(**f)


MIXTURE = [(dict(K=0), "PC_ERR_ARG"), (dict(K=129), "PC_ERR_ARG"), (dict(n_blocks=0), "PC_ERR_ARG"), (dict(n_cats=0), "PC_ERR_ARG"), (dict(n_cats=-4), "PC_ERR_ARG"),
           (dict(n_cats=1 << 30), "PC_ERR_TOO_LARGE"), (dict(n_tables=3), "PC_ERR_ARG"), (dict(n_tables=0), "PC_ERR_ARG"), (dict(n_rows=127), "PC_ERR_ARG"), (dict(n_rows=0, rows=P), "PC_ERR_ARG"),
           (dict(stride=15), "PC_ERR_ARG"), (dict(weights=None), "PC_ERR_ARG"), (dict(weights=P + 2), "PC_ERR_ARG"), (dict(rows=P + 1), "PC_ERR_ARG"),
           (dict(n_blocks=1 << 30, n_rows=1 << 40, n_tables=1 << 30), "PC_ERR_TOO_LARGE")]


@pytest.mark.parametrize("change,want", MIXTURE)
def test_predict_refuses_mixtures(change, want):
    m = mixture(**change)
    assert status(pcb.lib().pc_predict(C.byref(m), P, 16, P, 10, None, 0, None)) == want
    assert status(pcb.lib().pc_predict_backward(C.byref(m), P, 16, P, 10, P, 10, 1.0, 1, P, P, 1 << 30, None)) == want


@pytest.mark.parametrize("args,want", [((None, 16, P, 10), "PC_ERR_ARG"), ((P + 4, 16, P, 10), "PC_ERR_ARG"), ((P, 0, P, 10), "PC_ERR_ARG"), ((P, -1, P, 10), "PC_ERR_ARG"),
                                       ((P, 2097153, P, 10), "PC_ERR_TOO_LARGE"), ((P, 65, P, 10), "PC_ERR_ARG"), ((P, 16, None, 10), "PC_ERR_ARG"), ((P, 16, P + 1, 10), "PC_ERR_ARG"),
                                       ((P, 16, P, 9), "PC_ERR_ARG")])
def test_predict_refuses_arguments(args, want):
    m = mixture()
    assert status(pcb.lib().pc_predict(C.byref(m), *args, P, 1 << 30, None)) == want
    assert status(pcb.lib().pc_predict(None, P, 16, P, 10, None, 0, None)) == "PC_ERR_ARG"


@pytest.mark.parametrize("args", [(P, 9, P, 10, 1.0, 1, P), (P, 10, P, 9, 1.0, 1, P), (None, 10, P, 10, 1.0, 1, P), (P, 10, None, 10, 1.0, 1, P), (P, 10, P, 10, 1.0, 1, None), (P, 10, P, 10, 1.0, 1, P + 4),
                                  (P + 2, 10, P, 10, 1.0, 1, P)])
def test_predict_backward_refuses_arguments(args):
    m = mixture()
    assert status(pcb.lib().pc_predict_backward(C.byref(m), P, 16, *args, P, 1 << 30, None)) == "PC_ERR_ARG"


def test_predict_refuses_workspaces():
    m, n, L = mixture(n_blocks=64, n_tables=64, n_rows=2048), C.c_size_t(), pcb.lib()
    assert status(L.pc_predict_workspace_bytes(C.byref(m), 40, C.byref(n))) == "PC_OK" and n.value >= 2 * 40 * 10 * 4
    for ws, size, want in ((P, n.value - 1, "PC_ERR_WORKSPACE"), (None, 0, "PC_ERR_WORKSPACE"), (None, n.value, "PC_ERR_ARG"), (P + 8, n.value, "PC_ERR_ARG")):
        assert status(L.pc_predict(C.byref(m), P, 40, P, 10, ws, size, None)) == want
    assert status(L.pc_predict_workspace_bytes(None, 16, C.byref(n))) == "PC_ERR_ARG"
    assert status(L.pc_predict_workspace_bytes(C.byref(m), 16, None)) == "PC_ERR_ARG"
    m = mixture()
    assert status(L.pc_predict_workspace_bytes(C.byref(m), 16, C.byref(n))) == "PC_OK" and n.value == 0


def test_predict_backward_refuses_workspaces():
    m, n, L = mixture(stride=300), C.c_size_t(), pcb.lib()
    assert status(L.pc_predict_backward_workspace_bytes(C.byref(m), 16, C.byref(n))) == "PC_OK" and n.value == 0
    assert status(L.pc_predict_backward_workspace_bytes(C.byref(m), 300, C.byref(n))) == "PC_OK" and n.value >= 300 * 128 * 4 + 10 * 4
    for ws, size, want in ((P, n.value - 1, "PC_ERR_WORKSPACE"), (None, 0, "PC_ERR_WORKSPACE"), (None, n.value, "PC_ERR_ARG"), (P + 8, n.value, "PC_ERR_ARG")):
        assert status(L.pc_predict_backward(C.byref(m), P, 300, P, 10, P, 10, 1.0, 1, P, ws, size, None)) == want
    assert status(L.pc_predict_backward_workspace_bytes(None, 16, C.byref(n))) == "PC_ERR_ARG"
    assert status(L.pc_predict_backward_workspace_bytes(C.byref(m), 16, None)) == "PC_ERR_ARG"
    assert status(L.pc_predict_backward_workspace_bytes(C.byref(m), 301, C.byref(n))) == "PC_ERR_ARG"


def test_mixtures_of_circuits_need_a_device_and_a_variable():
    w = W.hmm(3, 2, 3, 2, 1, 52)
    h = pcb.pc_compile(w, host_only=True)
    m = pcb.pc_mixture()
    assert status(pcb.lib().pc_get_mixture(h, 0, 5, P, 1 << 30, C.byref(m))) == "PC_ERR_STATE"
    assert status(pcb.lib().pc_get_mixture(None, 0, 5, P, 1 << 30, C.byref(m))) == "PC_ERR_ARG"
    assert status(pcb.lib().pc_get_mixture(h, 0, 5, None, 1 << 30, C.byref(m))) == "PC_ERR_ARG"
    assert status(pcb.lib().pc_get_mixture(h, 0, 5, P, 1 << 30, None)) == "PC_ERR_ARG"
    pcb.pc_destroy(h)


def distill(**kw):
    f = dict(rows=6, n_cats=50, top=4, student=P, student_type=0, student_ld=50, ids=P, ids_ld=4, teacher=P, teacher_type=1, teacher_ld=4, teacher_lse=None, temperature=1.0, normalised=0)
    f.update(kw)
    return pcb.pc_distill(**f)


@pytest.mark.parametrize("change", [dict(rows=-1), dict(n_cats=0), dict(top=0), dict(top=1025, ids_ld=1025, teacher_ld=1025), dict(student_type=3), dict(teacher_type=-1), dict(temperature=0.0),
                                    dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-39), dict(normalised=1, temperature=2.0), dict(student_ld=49),
                                    dict(ids_ld=3), dict(teacher_ld=3), dict(student=None), dict(ids=None), dict(teacher=None), dict(student=P + 2), dict(teacher=P + 1), dict(ids=P + 2),
                                    dict(teacher_lse=P + 2)])
def test_distill_refuses_descriptors(change):
    d, n = distill(**change), C.c_size_t()
    assert status(pcb.lib().pc_distill_workspace_bytes(C.byref(d), C.byref(n))) == "PC_ERR_ARG"
    assert status(pcb.lib().pc_distill_forward(C.byref(d), P, 1 << 30, P, P, None)) == "PC_ERR_ARG"
    assert status(pcb.lib().pc_distill_backward(C.byref(d), P, None, 1.0, P << 4, 50, None)) == "PC_ERR_ARG"


def test_distill_refuses_arguments():
    d, L = distill(), pcb.lib()
    assert status(L.pc_distill_workspace_bytes(None, C.byref(C.c_size_t()))) == "PC_ERR_ARG"
    assert status(L.pc_distill_workspace_bytes(C.byref(d), None)) == "PC_ERR_ARG"
    for loss, stats in ((None, P), (P, None), (P + 1, P), (P, P + 2)):
        assert status(L.pc_distill_forward(C.byref(d), P, 1 << 30, loss, stats, None)) == "PC_ERR_ARG"
    far = P << 4
    for stats, out, ld in ((None, far, 50), (P, None, 50), (P, far, 49), (P + 2, far, 50), (P, far + 1, 50)):
        assert status(L.pc_distill_backward(C.byref(d), stats, None, 1.0, out, ld, None)) == "PC_ERR_ARG"
    for out, ld in ((P + 4, 50), (P, 51), (P + 6 * 50 * 4 - 4, 50), (P - 5 * 50 * 4, 50)):     # over the student's rows, but not the same
        assert status(L.pc_distill_backward(C.byref(d), P, None, 1.0, out, ld, None)) == "PC_ERR_ARG"


def test_distill_workspaces_are_checked():
    d, n, L = distill(rows=1, n_cats=50257, student_ld=50257), C.c_size_t(), pcb.lib()
    assert status(L.pc_distill_workspace_bytes(C.byref(d), C.byref(n))) == "PC_OK"
    if n.value:
        assert status(L.pc_distill_forward(C.byref(d), P, n.value - 1, P, P, None)) == "PC_ERR_WORKSPACE"
        assert status(L.pc_distill_forward(C.byref(d), None, 1 << 30, P, P, None)) == "PC_ERR_ARG"
        assert status(L.pc_distill_forward(C.byref(d), P + 8, 1 << 30, P, P, None)) == "PC_ERR_ARG"


def beam(**kw):
    f = dict(groups=3, beams=4, n_cats=50, n_out=8, scores=P, scores_type=0, scores_ld=50, normalise=0, running=None, done=None, done_token=0)
    f.update(kw)
    return pcb.pc_beam(**f)


@pytest.mark.parametrize("change,want", [(dict(groups=-1), "PC_ERR_ARG"), (dict(beams=0), "PC_ERR_ARG"), (dict(beams=65), "PC_ERR_ARG"), (dict(n_cats=0), "PC_ERR_ARG"), (dict(n_out=0), "PC_ERR_ARG"),
                                         (dict(n_out=65), "PC_ERR_ARG"), (dict(beams=1, n_cats=7, n_out=8), "PC_ERR_ARG"), (dict(scores_type=7), "PC_ERR_ARG"), (dict(scores_ld=49), "PC_ERR_ARG"),
                                         (dict(scores=None), "PC_ERR_ARG"), (dict(scores=P + 2), "PC_ERR_ARG"), (dict(running=P + 1), "PC_ERR_ARG"), (dict(done=P, done_token=50), "PC_ERR_ARG"),
                                         (dict(done=P, done_token=-1), "PC_ERR_ARG"), (dict(groups=1 << 30), "PC_ERR_TOO_LARGE")])
def test_beam_refuses_descriptors(change, want):
    a, n = beam(**change), C.c_size_t()
    assert status(pcb.lib().pc_beam_workspace_bytes(C.byref(a), C.byref(n))) == want
    assert status(pcb.lib().pc_beam_select(C.byref(a), P, 1 << 30, P, P, P, None)) == want


def test_beam_refuses_arguments():
    a, n, L = beam(), C.c_size_t(), pcb.lib()
    assert status(L.pc_beam_workspace_bytes(C.byref(a), C.byref(n))) == "PC_OK" and n.value > 0
    assert status(L.pc_beam_select(C.byref(a), P, n.value - 1, P, P, P, None)) == "PC_ERR_WORKSPACE"
    for args in ((None, n.value, P, P, P), (P + 8, n.value, P, P, P), (P, n.value, None, P, P), (P, n.value, P, None, P), (P, n.value, P, P, None), (P, n.value, P + 2, P, P)):
        assert status(L.pc_beam_select(C.byref(a), *args, None)) == "PC_ERR_ARG"


def reorder(states, n=None, parents=P, groups=2, beams=3, n_out=4):
    array = (pcb.pc_state * max(1, len(states)))(*[pcb.pc_state(*s) for s in states])
    return status(pcb.lib().pc_beam_reorder(array, len(states) if n is None else n, parents, groups, beams, n_out, None))


def test_reorder_refuses():
    ok = (P, 2 * P, 100, 100, 100)                         # src: 600 bytes, dst: 800
    assert reorder([ok], n=0) == "PC_ERR_ARG" and reorder([ok], n=17) == "PC_ERR_ARG" and reorder([ok], parents=None) == "PC_ERR_ARG" and reorder([ok], parents=P + 2) == "PC_ERR_ARG"
    assert reorder([ok], groups=-1) == "PC_ERR_ARG" and reorder([ok], beams=0) == "PC_ERR_ARG" and reorder([ok], beams=65) == "PC_ERR_ARG" and reorder([ok], n_out=65) == "PC_ERR_ARG"
    for bad in ((None, P, 100, 100, 100), (P, None, 100, 100, 100), (P, 2 * P, 0, 100, 100), (P, 2 * P, 100, 99, 100), (P, 2 * P, 100, 100, 99),
                (P, P, 100, 100, 100), (P, P + 599, 100, 100, 100), (P, P - 799, 100, 100, 100)):
        assert reorder([bad]) == "PC_ERR_ARG", bad
    assert reorder([ok, (3 * P, P + 50, 100, 100, 100)]) == "PC_ERR_ARG"       # onto another state's src
    assert reorder([ok, (3 * P, 2 * P + 750, 100, 100, 100)]) == "PC_ERR_ARG"  # onto another dst


def test_calls_without_rows_do_nothing():
    L = pcb.lib()
    d = distill(rows=0, student=None, ids=None, teacher=None)
    assert status(L.pc_distill_forward(C.byref(d), None, 0, None, None, None)) == "PC_OK"
    assert status(L.pc_distill_backward(C.byref(d), None, None, 1.0, None, 50, None)) == "PC_OK"
    a = beam(groups=0, scores=None)
    assert status(L.pc_beam_select(C.byref(a), None, 0, None, None, None, None)) == "PC_OK"
    assert reorder([(None, None, 100, 100, 100)], parents=None, groups=0) == "PC_OK"


def test_tensors_on_the_cpu_are_refused():
    torch = pytest.importorskip("torch")
    for make in (lambda: pcb.mixture(torch.zeros(32, 4), 32, 5, 1), lambda: pcb.distill(torch.zeros(2, 5), torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1)),
                 lambda: pcb.beam(torch.zeros(2, 5), torch.zeros(1, 2), 2), lambda: pcb.pc_beam_reorder([], torch.zeros((1, 1), dtype=torch.int32), 1)):
        with pytest.raises(pcb.PcError) as e:
            make()
        assert e.value.status_name == "PC_ERR_ARG"
