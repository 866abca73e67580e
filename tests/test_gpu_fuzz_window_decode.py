"""Random shapes, lengths, windows and positions through windowed prefill and decode attention (fixed seeds)."""
import random

import numpy as np
import pytest

from paper_2609_32999_b200 import workloads as wl
from tests import test_gpu_decode as td
from tests import test_gpu_window as tw

pytestmark = pytest.mark.gpu


def _shape(r):
    return r.choice([1, 2, 3, 4, 5, 7, 8, 9, 12, 16]), r.choice([1, 2, 3, 4, 8]), r.choice([64, 128]), r.choice([8, 16, 32, 64, 128])


def _log(r, lo, hi):
    return int(round(lo * (hi / lo) ** r.random()))


@pytest.mark.parametrize("seed", range(40))
def test_decode(seed):
    r = random.Random(seed)
    g, h, d, page = _shape(r)
    top = _log(r, 1, 5000)
    lens = [r.choice([0, 1, _log(r, 1, top), r.randint(0, top), top]) for _ in range(_log(r, 1, max(1, min(60, 60000 // top))))]
    td.Case(lens, g * h, h, d, page, seed=seed, four=seed % 2 == 1, window=r.choice([0, _log(r, 1, 2 * top)]), n_sink=r.choice([0, 1, r.randint(0, 200)]),
            q_size=r.choice([1, 1, 8])).run().check()


@pytest.mark.parametrize("seed", range(40))
def test_windowed_prefill(seed):
    r = random.Random(1000 + seed)
    g, h, d, page = _shape(r)
    top = _log(r, 2, 4000)
    lens = [r.randint(max(1, top // 3), top) for _ in range(_log(r, 1, 4))]
    rng = np.random.default_rng(seed)
    reqs = []
    for t in lens:
        if r.random() < 0.5:          # runs of 16 rows
            rows = sorted({int(x) for s in rng.integers(0, t, 1 + _log(r, 1, 300) // 16) for x in range(s, min(t, s + 16))})
        else:
            rows = sorted(rng.choice(t, min(t, _log(r, 1, 300)), replace=False))
        reqs.append([wl.unit(t, recompute=rows)])
    w = wl.build_workload("fuzz", wl.ModelShape(g * h, h, d, page, 10000.0), reqs, rng)
    tw.check(w, _log(r, 1, top), r.choice([0, 1, 4, 130, r.randint(0, 400)]), seed=seed, spoil=r.random() < 0.5)
