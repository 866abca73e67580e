"""Tensors that a plan's calls refuse before the library hears of them, on the CPU: the library's functions are replaced by ones that
count their calls, and a tensor's device is what get_device() says (-1 for host memory)."""
import numpy as np
import pytest
import torch

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl

SHAPE = wl.ModelShape(8, 2, 128, 16, 1e4)


def workload(retain=False):
    w = wl.build_workload("arguments", SHAPE, [[7, wl.unit(20, "a", cached=False)], [5]], np.random.default_rng(0))
    if retain:
        w.unit_retain_page_off, w.unit_retain_pages, w.retain_pool_pages = np.array([0, 2], np.int32), np.array([1, 0], np.int32), 3
    return w


@pytest.fixture
def device_plan(monkeypatch):
    """A plan whose calls expect tensors on `device`, and the list of the calls that got through."""
    def make(w, device):
        calls = []
        for name in ("tessera_extend_write_norm", "tessera_kv_retain_kv4", "tessera_kv_compose_from_kv4"):
            monkeypatch.setattr(tb._lib, name, lambda *a, name=name: calls.append(name) or 0)
        monkeypatch.setattr(tb, "_current_device", lambda: device, raising=False)
        monkeypatch.setattr(tb, "_stream", lambda stream: None)
        plan = tb.Plan(w, host_only=True)
        plan.host_only = False
        return plan, calls
    return make


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def norm_arguments(w, retain=False):
    n, pool = w.n_q, (w.num_pool_pages, 16, 2, 128)
    a = dict(k_pool=bf16(*pool), v_pool=bf16(*pool), q=bf16(n, 8, 128), q_out=bf16(n, 8, 128), k_new_raw=bf16(n, 2, 128), v_new=bf16(n, 2, 128),
             q_weight=bf16(128), k_weight=bf16(128))
    if retain:
        a.update(k_cache=bf16(3, 16, 2, 128), v_cache=bf16(3, 16, 2, 128))
    return a


@pytest.mark.parametrize("alone", [False, True])
def test_normalising_write_of_rows_in_host_memory(device_plan, alone):
    """Rows that are all on the CPU, beside pools that claim to be on the device."""
    w = workload()
    plan, calls = device_plan(w, 0)
    a = norm_arguments(w)
    a.update(k_pool=None, v_pool=None)
    if alone:
        a.update(q=None, q_out=None, q_weight=None)
    with pytest.raises(ValueError):
        plan.extend_write_norm(**a)
    assert not calls


@pytest.mark.parametrize("change", [dict(k_pool=bf16(1, 16, 2, 128)), dict(v_pool=bf16(99, 16, 1, 128)), dict(k_pool=bf16(99, 32, 2, 64)),
                                    dict(v_pool=torch.zeros(99, 16, 2, 128)), dict(k_pool=bf16(99, 16, 128, 2).transpose(2, 3)),
                                    dict(k_pool=bf16(99 * 16, 2, 128)), dict(k_cache=bf16(2, 16, 2, 128)), dict(v_cache=bf16(3, 16, 2, 64)),
                                    dict(v_cache=torch.zeros(3, 16, 2, 128, dtype=torch.uint8))])
def test_normalising_write_pools(device_plan, change):
    w = workload(retain=True)
    plan, calls = device_plan(w, -1)
    a = norm_arguments(w, retain=True)
    with pytest.raises(ValueError) as e:
        plan.extend_write_norm(**dict(a, **change))
    assert isinstance(e.value, tb.TesseraError) and e.value.status == tb.INVALID_ARG and not calls
    plan.extend_write_norm(**a)
    plan.extend_write_norm(**dict(a, k_pool=bf16(99, 16, 2, 128)))           # more pages than the plan counts
    assert len(calls) == 2


def test_normalising_write_pools_on_another_device(device_plan):
    w = workload()
    plan, calls = device_plan(w, -1)
    a = norm_arguments(w)
    plan, calls = device_plan(w, 0)
    with pytest.raises(ValueError) as e:
        plan.extend_write_norm(**a)
    assert "k_pool" in str(e.value) and not calls


def tier_workload():
    """Units of 20 and 5 tokens out of a source pool of 9 pages into a pool of 6."""
    i = lambda *x: np.array(x, np.int32)
    return wl.Workload("tier", SHAPE, i(20, 5), i(0, 1, 2), i(20, 5), i(0, 0), i(1, 1), i(0, 0), i(0, 2, 3), i(8, 1, 4), i(0, 0, 0), i(), i(5, 0, 2), 6,
                       num_source_pages=9)


def four_bit(pages, shape=SHAPE):
    return torch.zeros(tb.pool4_shape(shape, pages), dtype=torch.uint8)


WIDE = wl.ModelShape(8, 2, 128, 32, 1e4)


@pytest.mark.parametrize("k_src,v_src,k_dst,v_dst", [
    (four_bit(6), four_bit(6), bf16(9, 16, 2, 128), bf16(9, 16, 2, 128)),                     # source and destination swapped
    (bf16(8, 16, 2, 128), bf16(9, 16, 2, 128), four_bit(6), four_bit(6)),                     # a source page too few
    (bf16(9, 16, 2, 128), bf16(9, 16, 2, 128), four_bit(6), four_bit(5)),                     # a destination page too few
    (bf16(9, 16, 2, 128), bf16(9, 16, 2, 128), four_bit(6, WIDE), four_bit(6, WIDE)),         # another page size
    (bf16(9, 16, 2, 128), bf16(9, 16, 2, 64), four_bit(6), four_bit(6)),                      # another head_dim
    (bf16(9, 16, 2, 128), bf16(9, 16, 2, 128).float(), four_bit(6), four_bit(6)),
    (bf16(9, 16, 2, 128), bf16(9, 16, 2, 128), four_bit(6), four_bit(12)[::2]),               # pages apart
    (bf16(9, 16, 2, 128), bf16(9, 16, 2, 128), bf16(6, 16, 2, 128), four_bit(6))])
def test_store_pools(device_plan, k_src, v_src, k_dst, v_dst):
    plan, calls = device_plan(tier_workload(), -1)
    with pytest.raises(ValueError) as e:
        plan.kv_retain_kv4(k_src, v_src, k_dst, v_dst)
    assert isinstance(e.value, tb.TesseraError) and e.value.status == tb.INVALID_ARG and not calls
    plan.kv_retain_kv4(bf16(9, 16, 2, 128), bf16(10, 16, 2, 128), four_bit(6), four_bit(99))
    assert calls == ["tessera_kv_retain_kv4"]


@pytest.mark.parametrize("k_src,v_src,k_dst,v_dst", [
    (bf16(6, 16, 2, 128), bf16(6, 16, 2, 128), four_bit(9), four_bit(9)),
    (four_bit(9), four_bit(8), bf16(6, 16, 2, 128), bf16(6, 16, 2, 128)),
    (four_bit(9), four_bit(9), bf16(5, 16, 2, 128), bf16(6, 16, 2, 128)),
    (four_bit(9, WIDE), four_bit(9), bf16(6, 16, 2, 128), bf16(6, 16, 2, 128)),
    (four_bit(9), four_bit(9), bf16(6, 2, 16, 128), bf16(6, 16, 2, 128)),
    (four_bit(9), four_bit(9), bf16(6, 16, 2, 128).half(), bf16(6, 16, 2, 128))])
def test_load_pools(device_plan, k_src, v_src, k_dst, v_dst):
    plan, calls = device_plan(tier_workload(), -1)
    with pytest.raises(ValueError):
        plan.kv_compose_from_kv4(k_src, v_src, k_dst, v_dst)
    assert not calls
    plan.kv_compose_from_kv4(four_bit(9), four_bit(9), bf16(6, 16, 2, 128), bf16(7, 16, 2, 128))
    assert calls == ["tessera_kv_compose_from_kv4"]


def test_tier_pools_in_plain_host_memory(device_plan):
    plan, calls = device_plan(tier_workload(), 0)
    with pytest.raises(ValueError):
        plan.kv_retain_kv4(bf16(9, 16, 2, 128), bf16(9, 16, 2, 128), four_bit(6), four_bit(6))
    with pytest.raises(ValueError):
        plan.kv_compose_from_kv4(four_bit(9), four_bit(9), bf16(6, 16, 2, 128), bf16(6, 16, 2, 128))
    assert not calls
