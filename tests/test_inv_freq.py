"""Frequency tables shorter than head_dim / 2 are refused wherever one is taken, before anything reads past their end."""
import numpy as np
import pytest
import torch

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl

SHAPE = wl.ModelShape(8, 2, 128, 16, 1e4)
FULL = 1e4 ** (-2.0 * np.arange(64) / 128)


def short():
    return FULL[:63]               # (a view: what lies behind it is the table's last number)


def test_plan():
    w = wl.build_workload("frequencies", SHAPE, [[wl.unit(20), 5]], np.random.default_rng(0))
    tb.Plan(w, host_only=True, inv_freq=FULL)
    with pytest.raises(ValueError, match="inv_freq"):
        tb.Plan(w, host_only=True, inv_freq=short())


def test_decode():
    with pytest.raises(ValueError, match="inv_freq"):
        tb.Decode(SHAPE, torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 4, inv_freq=short())


def test_static_shift(monkeypatch):
    calls = []
    monkeypatch.setattr(tb._lib, "tessera_rope_shift_static", lambda *a: calls.append(a) or 0)
    monkeypatch.setattr(tb, "_stream", lambda stream: None)
    pool, at = torch.zeros(2, 16, 2, 128, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="inv_freq"):
        tb.rope_shift_static(SHAPE, pool, at, at, [3], inv_freq=short())
    assert not calls
    tb.rope_shift_static(SHAPE, pool, at, at, [3], inv_freq=FULL)
    assert len(calls) == 1
