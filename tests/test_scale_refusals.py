"""A softmax scale that is no number is refused where a plan is made and by decode attention, on the CPU."""
import numpy as np
import pytest

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl
from tests import test_decode_refusals as td


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf")])
def test_not_finite(scale):
    w = wl.build_workload("scale", wl.ModelShape(8, 2, 128, 16, 1e4, sm_scale=scale), [[wl.unit(20), 5]], np.random.default_rng(0))
    for kw in ({}, dict(window=9, n_sink=1)):
        with pytest.raises(tb.TesseraError) as e:
            tb.Plan(w, host_only=True, **kw)
        assert e.value.status == tb.INVALID_ARG and "sm_scale" in str(e.value)
    for four in (False, True):
        assert td.attn(td.cfg(sm_scale=scale), td.desc(), four=four) == tb.INVALID_ARG and "sm_scale" in tb.last_error()


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e30])
def test_finite(scale):
    w = wl.build_workload("scale", wl.ModelShape(8, 2, 128, 16, 1e4, sm_scale=scale), [[wl.unit(20), 5]], np.random.default_rng(0))
    tb.Plan(w, host_only=True)
    assert td.attn(td.cfg(sm_scale=scale), td.desc(batch=0)) == tb.OK
