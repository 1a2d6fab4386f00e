"""Host-side limits of the operators around the dense logits that need no GPU."""
import os

import numpy as np
import pytest

import paper_2603_25011_amd as lsr

P = 1 << 20          # an aligned address that is never dereferenced
WS = (P, 1 << 40)


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(lsr.library_path()):
        from paper_2603_25011_amd import build
        build.build()
    return lsr.load_library()


@pytest.mark.parametrize("T,taken", [(5e-39, True), (4.2e-39, False), (4e-39, False), (3e-39, False), (1.0, True), (3e38, True)])
def test_temperatures_whose_reciprocal_times_log2_e_is_no_float32_are_refused(T, taken):
    with np.errstate(over="ignore"):
        assert bool(np.isfinite(np.float32(1) / np.float32(T) * np.float32(1.44269504088896340736))) == taken
    for back in (False, True):
        assert (lsr.lsr_distill_workspace_bytes(64, 64, 500, 4, lsr.LSR_F32, T, back) > 0) == taken
    if taken:
        return
    SHAPE = 2
    for call in (lambda: lsr.lsr_top_logits(4, 500, 4, lsr.LSR_F32, T, P, 500, P, P, P, WS, stream=0),
                 lambda: lsr.lsr_distill_forward(64, 64, 500, 4, lsr.LSR_F32, T, *[P] * 9, WS, stream=0),
                 lambda: lsr.lsr_distill_backward(64, 64, 500, 4, lsr.LSR_F32, T, *[P] * 12, WS, stream=0)):
        with pytest.raises(lsr.LsrError) as e:
            call()
        assert e.value.status == SHAPE
