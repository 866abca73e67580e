"""Prefill attention with a negative softmax scale: against 64 bits, and bit for bit what negated queries give with the positive one."""
import numpy as np
import pytest
import torch

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl
from tests import attn_ref as ar
from tests import test_gpu_window as tw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("hq,h,d,page", [(4, 2, 64, 16), (8, 1, 128, 64), (10, 2, 128, 8)])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (100, 4), (257, 200)])
def test_against_64_bits(hq, h, d, page, window, n_sink):
    tw.check(tw.batch([901, 300, 1, 130], [120, 300, 1, 3], hq, h, d, page, seed=21), window, n_sink, scale=-0.11)


@pytest.mark.parametrize("window,n_sink", [(0, 0), (20000, 64)])
def test_cut_key_ranges(window, n_sink):
    plan = tw.check(tw.batch([30000, 9000], [40, 30], 8, 2, 128, 64, seed=22), window, n_sink, scale=-0.3)[0]
    assert plan.info.n_attn_items > 2 * 2 * 2          # the key ranges were cut


@pytest.mark.parametrize("window,n_sink", [(0, 0), (100, 4)])
def test_eight_bit_keys(window, n_sink):
    w = tw.batch([901, 300, 2048], [120, 40, 64], 8, 2, 128, 64, seed=23)
    w.shape.sm_scale = -0.11
    plan, t = tb.Plan(w, window=window, n_sink=n_sink), wl.make_tensors(w, device=DEV, seed=4)
    k8 = (t.k_pool.float() * 32).clamp(-448, 448).to(torch.float8_e4m3fn)
    out, lse = torch.zeros_like(t.q), torch.zeros(w.n_q, 8, device=DEV)
    plan.partial_prefill_attn_k8(k8, 1 / 32, t.v_pool, t.q, 1 / 32, None, None, out, lse)
    q8 = (t.q.float() * 32).clamp(-448, 448).to(torch.float8_e4m3fn).float() / 32
    for r in range(w.batch):
        a, b = int(w.recompute_off[r]), int(w.recompute_off[r + 1])
        pos = torch.from_numpy(w.recompute_pos[a:b].astype(np.int64)).to(DEV)
        k = tw.rows_of(w, plan, k8.view(torch.uint8), r).view(torch.float8_e4m3fn).float() / 32
        ar.check(out[a:b], lse[a:b], ar.attend(q8[a:b], k, tw.rows_of(w, plan, t.v_pool, r), pos, window, n_sink, -0.11), len(k))


@pytest.mark.parametrize("window,n_sink", [(0, 0), (100, 4)])
def test_the_sign_is_all_that_changes(window, n_sink):
    w = tw.batch([1200, 300], [200, 300], 8, 2, 128, 64, seed=24)
    t, got = wl.make_tensors(w, device=DEV, seed=5), []
    for scale, sign in ((-0.2, 1), (0.2, -1)):
        w.shape.sm_scale = scale
        out, lse = torch.zeros_like(t.q), torch.zeros(w.n_q, 8, device=DEV)
        tb.Plan(w, window=window, n_sink=n_sink).partial_prefill_attn(t.k_pool, t.v_pool, t.q * sign, None, None, out, lse)
        torch.cuda.synchronize()
        got.append((out, lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
