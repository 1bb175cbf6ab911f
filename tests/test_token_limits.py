"""Limits of the calls for token models, on the CPU: what lies just inside is accepted, what lies just outside is refused on the host (the addresses in
these descriptors name no memory, and no call here gets as far as a launch)."""
import ctypes as C

import numpy as np
import pytest

from paper_2406_00766_amd import binding as pcb
from tests.test_token_refusals import P, distill, status


@pytest.mark.parametrize("temperature,want", [(4.3e-39, "PC_OK"), (4.2e-39, "PC_ERR_ARG"), (3e-39, "PC_ERR_ARG"), (1e38, "PC_OK")])
def test_temperatures_whose_exponents_overflow_are_refused(temperature, want):
    """Exponentials are taken of (z - m) log2(e) / T: with log2(e) / T = inf the largest logit itself would give 0 * inf."""
    assert np.isfinite(np.float32(1.0) / np.float32(temperature))
    assert np.isfinite(np.float32(1.4426950408889634) * (np.float32(1.0) / np.float32(temperature))) == (want == "PC_OK")
    d, n = distill(temperature=temperature), C.c_size_t()
    assert status(pcb.lib().pc_distill_workspace_bytes(C.byref(d), C.byref(n))) == want
    if want != "PC_OK":
        assert status(pcb.lib().pc_distill_forward(C.byref(d), None, 0, P, P, None)) == want
        assert status(pcb.lib().pc_distill_backward(C.byref(d), P, None, 1.0, P << 4, 50, None)) == want
