"""Pools that the 4-bit tier and the normalising write take beside device pools of the plan's own size: page-locked host memory, more pages."""
import pytest
import torch

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl
from tests.test_gpu_kv4 import tier
from tests.test_gpu_norm_write import workload

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("place", ["pinned", "larger"])
def test_tier(place):
    shape = wl.ModelShape(8, 2, 128, 16, 10000.0)
    store, load, at, pools, _ = tier(shape, [40, 16, 3], [5, -7, 0])
    more = 3 if place == "larger" else 0
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    k, v = (torch.randn(pools[0], 16, 2, 128, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))

    def grown(x):
        return x.cpu().pin_memory() if place == "pinned" else torch.cat([x, x.new_zeros(more, *x.shape[1:])])

    got = []
    for odd in (False, True):
        make = grown if odd else (lambda x: x)
        k_4, v_4 = (make(torch.full(tb.pool4_shape(shape, pools[1]), 7, dtype=torch.uint8, device=DEV)) for _ in range(2))
        ko, vo = (torch.full((pools[2] + (more if odd else 0), 16, 2, 128), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        store.kv_retain_kv4(make(k), make(v), k_4, v_4)
        load.kv_compose_from_kv4(k_4, v_4, ko, vo)
        torch.cuda.synchronize()
        got.append([x[:n].cpu() for x, n in ((k_4, pools[1]), (v_4, pools[1]), (ko, pools[2]), (vo, pools[2]))])
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert not (got[0][2] == 3).all()


def test_captured_units_to_page_locked_memory():
    shape = wl.ModelShape(8, 2, 128, 16, 10000.0)
    w = workload(shape)
    weight = (1 + 0.3 * torch.randn(128, device=DEV)).to(torch.bfloat16)
    got = []
    for pinned in (False, True):
        t, plan = wl.make_tensors(w, device=DEV, seed=2), tb.Plan(w)
        kc, vc = (torch.full((w.retain_pool_pages, 16, 2, 128), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        if pinned:
            kc, vc = kc.cpu().pin_memory(), vc.cpu().pin_memory()
        plan.extend_write_norm(t.k_pool, t.v_pool, t.q, t.q, t.k_new, t.v_new, weight, weight, 1e-6, kc, vc)
        torch.cuda.synchronize()
        got.append([x.cpu() for x in (t.q, t.k_pool, t.v_pool, kc, vc)])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_rows_in_host_memory():
    w = workload(wl.ModelShape(8, 2, 128, 16, 10000.0), retain=False)
    t, plan = wl.make_tensors(w, device=DEV, seed=2), tb.Plan(w)
    before = t.k_pool.clone()
    host = [x.cpu() for x in (t.q, t.k_new, t.v_new)]
    with pytest.raises(ValueError):
        plan.extend_write_norm(t.k_pool, t.v_pool, host[0], host[0], host[1], host[2])
    with pytest.raises(ValueError):
        plan.extend_write_norm(t.k_pool[:-1], t.v_pool, t.q, t.q, t.k_new, t.v_new)
    torch.cuda.synchronize()
    assert torch.equal(t.k_pool, before)
