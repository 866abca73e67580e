"""Prefill attention with a sliding window and sinks against attention in 64 bits, over pages filled directly."""
import numpy as np
import pytest
import torch

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl
from tests import attn_ref as ar

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def batch(lens, rows, hq, h, d, page, seed=0, positions=None):
    rng = np.random.default_rng(seed)
    shape = wl.ModelShape(hq, h, d, page, 10000.0)
    reqs = [[wl.unit(t, recompute=positions if positions is not None else sorted(rng.choice(t, min(n, t), replace=False)))] for t, n in zip(lens, rows)]
    return wl.build_workload("window", shape, reqs, rng)


def rows_of(w, plan, pool, r):
    """The request's rows [T][H][D] in its pages."""
    page_off, pages, _ = plan.block_table()
    ids = torch.from_numpy(pages[page_off[r]:page_off[r + 1]].astype(np.int64)).to(DEV)
    return pool[ids].reshape(-1, *pool.shape[2:])[: int(w.seq_len[r])]


def check(w, window, n_sink, seed=1, spoil=False, scale=0.0, q_size=1.0):
    w.shape.sm_scale = scale
    plan = tb.Plan(w, window=window, n_sink=n_sink)
    t = wl.make_tensors(w, device=DEV, seed=seed)
    t.q.mul_(q_size)
    if spoil:              # what nobody sees may hold anything
        page_off, pages, _ = plan.block_table()
        B = w.shape.page_size
        for r in range(w.batch):
            pos = w.recompute_pos[w.recompute_off[r]:w.recompute_off[r + 1]].astype(np.int64)
            seen = np.zeros(len(pages[page_off[r]:page_off[r + 1]]) * B, bool)
            for p in pos:
                seen[max(0, p - window + 1):p + 1] = True
                seen[: min(n_sink, p + 1)] = True
            at = np.flatnonzero(~seen)
            slot = torch.from_numpy(pages[page_off[r] + at // B].astype(np.int64) * B + at % B).to(DEV)
            t.k_pool.view(-1, *t.k_pool.shape[2:])[slot] = float("nan")
            t.v_pool.view(-1, *t.v_pool.shape[2:])[slot] = float("inf")
    out, lse = torch.zeros_like(t.q), torch.zeros(w.n_q, w.shape.num_q_heads, device=DEV)
    plan.partial_prefill_attn(t.k_pool, t.v_pool, t.q, None, None, out, lse)
    torch.cuda.synchronize()
    assert plan.status() == 0
    for r in range(w.batch):
        a, b = int(w.recompute_off[r]), int(w.recompute_off[r + 1])
        if a == b:
            continue
        pos = torch.from_numpy(w.recompute_pos[a:b].astype(np.int64)).to(DEV)
        k, v = rows_of(w, plan, t.k_pool, r), rows_of(w, plan, t.v_pool, r)
        if spoil:
            k, v = torch.nan_to_num(k, nan=0.0), torch.nan_to_num(v, posinf=0.0)
        ar.check(out[a:b], lse[a:b], ar.attend(t.q[a:b], k, v, pos, window, n_sink, scale or None), len(k), "request %d" % r)
    return plan, t, out, lse


SHAPES = [(4, 2, 64, 16), (8, 1, 128, 64), (10, 2, 128, 8), (3, 3, 64, 128), (16, 1, 64, 32), (7, 1, 128, 128)]


@pytest.mark.parametrize("hq,h,d,page", SHAPES)
@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 3), (100, 4), (128, 128), (257, 200), (700, 0), (5000, 9)])
def test_against_64_bits(hq, h, d, page, window, n_sink):
    check(batch([901, 300, 1, 130, 2048], [120, 300, 1, 3, 64], hq, h, d, page), window, n_sink)


@pytest.mark.parametrize("window,n_sink", [(64, 4), (130, 0), (129, 300)])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
def test_keys_nobody_sees_may_hold_anything(d, page, window, n_sink):
    check(batch([3001, 640, 129], [40, 9, 1], 8, 2, d, page, seed=3), window, n_sink, spoil=True)


def test_one_row_each_and_long_gap():
    check(batch([20001], [1], 8, 2, 128, 64, positions=[20000]), 300, 5, spoil=True)
    check(batch([20001], [1], 8, 2, 128, 64, positions=[0, 1, 150, 7000, 7001, 20000]), 300, 5, spoil=True)


def test_cut_key_ranges():
    w = batch([30000, 9000], [40, 30], 8, 2, 128, 64, seed=5)
    plan = check(w, 20000, 64)[0]
    assert plan.info.n_attn_items > 2 * 2 * 2          # the key ranges were cut


@pytest.mark.parametrize("q_size,scale", [(30.0, 0.0), (1.0, 2.0), (0.0, 0.0)])
def test_score_sizes(q_size, scale):
    check(batch([1500], [200], 8, 2, 128, 64, seed=6), 333, 7, q_size=q_size, scale=scale)


def test_far_below_zero_scores():
    """A row whose first steps are masked and whose scores are then all far below zero: the weights do not vanish."""
    w = batch([2000], [1], 4, 1, 64, 16, positions=list(range(300, 332)) + [1900])
    plan = tb.Plan(w, window=90, n_sink=0)
    t = wl.make_tensors(w, device=DEV, seed=2)
    t.q.fill_(16.0)
    t.k_pool.fill_(-4.0).add_(0.25 * torch.randn(t.k_pool.shape, device=DEV).to(torch.bfloat16))
    out, lse = torch.zeros_like(t.q), torch.zeros(w.n_q, 4, device=DEV)
    plan.partial_prefill_attn(t.k_pool, t.v_pool, t.q, None, None, out, lse)
    pos = torch.from_numpy(w.recompute_pos.astype(np.int64)).to(DEV)
    ar.check(out, lse, ar.attend(t.q, rows_of(w, plan, t.k_pool, 0), rows_of(w, plan, t.v_pool, 0), pos, 90, 0), 2000)
    assert lse.max() < -400


def test_window_as_long_as_the_prompt_is_no_window():
    w = batch([1200, 77], [100, 20], 8, 2, 128, 64, seed=8)
    _, t, out, lse = check(w, 1200, 0)
    plan, o2, l2 = tb.Plan(w), torch.zeros_like(out), torch.zeros_like(lse)
    plan.partial_prefill_attn(t.k_pool, t.v_pool, t.q, None, None, o2, l2)
    assert torch.equal(out, o2) and torch.equal(lse, l2)


@pytest.mark.parametrize("page", [8, 64])
@pytest.mark.parametrize("window,n_sink", [(100, 4), (300, 200)])
def test_eight_bit_keys(page, window, n_sink):
    w = batch([901, 300, 2048], [120, 40, 64], 8, 2, 128, page, seed=9)
    plan, t = tb.Plan(w, window=window, n_sink=n_sink), wl.make_tensors(w, device=DEV, seed=4)
    k8 = (t.k_pool.float() * 32).clamp(-448, 448).to(torch.float8_e4m3fn)
    out, lse = torch.zeros_like(t.q), torch.zeros(w.n_q, 8, device=DEV)
    plan.partial_prefill_attn_k8(k8, 1 / 32, t.v_pool, t.q, 1 / 32, None, None, out, lse)
    q8 = (t.q.float() * 32).clamp(-448, 448).to(torch.float8_e4m3fn).float() / 32
    for r in range(w.batch):
        a, b = int(w.recompute_off[r]), int(w.recompute_off[r + 1])
        pos = torch.from_numpy(w.recompute_pos[a:b].astype(np.int64)).to(DEV)
        k = rows_of(w, plan, k8.view(torch.uint8), r).view(torch.float8_e4m3fn).float() / 32
        ar.check(out[a:b], lse[a:b], ar.attend(q8[a:b], k, rows_of(w, plan, t.v_pool, r), pos, window, n_sink), len(k))


def test_whole_layer_and_host_paths():
    """Compose, fresh rows and attention of a windowed plan; the host-buffer and host-tier entry points give the same bits."""
    rng = np.random.default_rng(11)
    shape = wl.ModelShape(8, 2, 128, 16, 10000.0)
    reqs = [[20, wl.unit(500, ("a", r), recompute=range(12)), 5, wl.unit(333, ("b", r), recompute=(0, 7)), 31] for r in range(5)]
    w = wl.build_workload("window-layer", shape, reqs, rng)
    outs = []
    for how in ("device", "host", "tier"):
        t = wl.make_tensors(w, device=DEV, seed=5)
        w.num_source_pages = w.num_pool_pages if how == "tier" else 0
        plan = tb.Plan(w, window=200, n_sink=4)
        out, lse = torch.zeros_like(t.q), torch.zeros(w.n_q, 8, device=DEV)
        if how == "device":
            plan.kv_compose(t.k_pool, t.v_pool)
            plan.partial_prefill_attn(t.k_pool, t.v_pool, t.q, t.k_new, t.v_new, out, lse)
            for r in range(w.batch):
                a, b = int(w.recompute_off[r]), int(w.recompute_off[r + 1])
                pos = torch.from_numpy(w.recompute_pos[a:b].astype(np.int64)).to(DEV)
                k, v = rows_of(w, plan, t.k_pool, r), rows_of(w, plan, t.v_pool, r)
                ar.check(out[a:b], lse[a:b], ar.attend(t.q[a:b], k, v, pos, 200, 4), len(k))
        elif how == "tier":
            src = t.k_pool.cpu().pin_memory(), t.v_pool.cpu().pin_memory()
            plan.composed_prefill_host_tier(*src, t.k_pool, t.v_pool, t.q, t.k_new, t.v_new, out, lse)
            torch.cuda.synchronize()
        else:
            host = [x.cpu().pin_memory() for x in (t.q, t.k_new, t.v_new, out, lse)]
            plan.composed_prefill_host(t.k_pool, t.v_pool, *host[:4], host[4])
            out, lse = host[3].to(DEV), host[4].to(DEV)
        assert plan.status() == 0
        outs.append((out.clone(), lse.clone()))
    for o, l in outs[1:]:
        assert torch.equal(outs[0][0], o) and torch.equal(outs[0][1], l)
