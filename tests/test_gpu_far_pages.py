"""Windows, norms, decode and the 4-bit tier where addresses pass 32 bits, in graphs, and with a Decode made on a busy stream.
The same pages at other places, the same call captured: the same bits."""
import dataclasses

import numpy as np
import pytest
import torch

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl
from tests.test_gpu_decode import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPE = wl.ModelShape(32, 8, 128, 64, 10000.0)
FAR16, FAR4 = 32768 + 200, 116509 + 200           # pages of SHAPE: pools of more than 2^32 bytes (and, 16-bit, 2^31 elements)


def moved(n, far):
    """Where n pages go in a pool of `far`, many more: every other to its end."""
    p = np.arange(n)
    return p if far == n else np.where(p % 2 == 0, p, far - 1 - p)


def put(small, to, far):
    big = torch.empty(far, *small.shape[1:], dtype=small.dtype, device=DEV)
    big[torch.from_numpy(to).to(DEV)] = small
    return big


def same(small, big, to):
    """Bit for bit."""
    there = big[torch.from_numpy(to).to(DEV)]
    return torch.equal(small.contiguous().view(torch.uint8), there.view(torch.uint8))


@pytest.mark.parametrize("four", [False, True])
def test_decode(four):
    c = Case([5000, 1, 64, 700, 0, 129], 32, 8, 128, 64, seed=3, four=four, window=3000, n_sink=70)
    far = FAR4 if four else FAR16
    to = moved(c.n_pages, far)
    k, v = put(c.k, to, far), put(c.v, to, far)
    table = torch.from_numpy(np.where(c.table < c.n_pages, to[np.minimum(c.table, c.n_pages - 1)], c.table).astype(np.int32)).to(DEV)
    dec = tb.Decode(SHAPE, table, c.decode.seq_lens, far, window=3000, n_sink=70)
    x = torch.randn(6, 48, 128, device=DEV).to(torch.bfloat16)
    out = []
    for d, kk, vv in ((c.decode, c.k, c.v), (dec, k, v)):
        q, o = torch.zeros_like(c.q), torch.zeros_like(c.q)
        (d.write_kv4 if four else d.write)(kk, vv, x[:, :32], q, x[:, 32:40], x[:, 40:], None, None)
        (d.attn_kv4 if four else d.attn)(kk, vv, q, o)
        out.append(o)
    assert torch.equal(*out) and out[0].isfinite().all() and out[0][0].abs().sum() > 0
    assert same(c.k, k, to) and same(c.v, v, to)


def test_tier():
    lens, per = [200, 64, 130], [4, 1, 3]
    n = len(lens)

    def plan(units, dest, pool, sources):
        return tb.Plan(wl.Workload("far", SHAPE, np.array(lens, np.int32), np.arange(n + 1, dtype=np.int32), np.array(lens, np.int32),
                                   np.array([-5, 0, 9], np.int32), np.ones(n, np.int32), np.zeros(n, np.int32),
                                   np.concatenate([[0], np.cumsum(per)]).astype(np.int32), units.astype(np.int32), np.zeros(n + 1, np.int32),
                                   np.zeros(0, np.int32), dest.astype(np.int32), pool, num_source_pages=sources))

    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    k, v = (torch.randn(8, 64, 8, 128, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    got = []
    for n16, n4 in ((8, 8), (FAR16, FAR4)):
        at16, at4 = moved(8, n16), moved(8, n4)
        kk, vv = put(k, at16, n16), put(v, at16, n16)
        k4, v4 = (torch.zeros(tb.pool4_shape(SHAPE, n4), dtype=torch.uint8, device=DEV) for _ in range(2))
        plan(at16, at4, n4, n16).kv_retain_kv4(kk, vv, k4, v4)
        for x in (kk, vv):
            x[torch.from_numpy(at16).to(DEV)] = 0
        plan(at4, at16, n16, n4).kv_compose_from_kv4(k4, v4, kk, vv)
        got.append([x[torch.from_numpy(at).to(DEV)] for x, at in ((k4, at4), (v4, at4), (kk, at16), (vv, at16))])
        del kk, vv, k4, v4
    for a, b in zip(*got):
        assert torch.equal(a, b) and a.any()


def layer(plan, t, q_raw, weight, out, lse):
    plan.kv_compose(t.k_pool, t.v_pool)
    plan.extend_write_norm(t.k_pool, t.v_pool, q_raw, t.q, t.k_new, t.v_new, weight, weight)
    plan.partial_prefill_attn(t.k_pool, t.v_pool, t.q, None, None, out, lse)


def prompts():
    rng = np.random.default_rng(1)
    w = wl.build_workload("far", SHAPE, [[20, wl.unit(600, "a"), 31, wl.unit(100, "b"), 5], [wl.unit(300, "a"), 7]], rng)
    t = wl.make_tensors(w, device=DEV, seed=2)
    return w, t, torch.randn(t.q.shape, device=DEV).to(torch.bfloat16), (1 + 0.1 * torch.randn(128, device=DEV)).to(torch.bfloat16)


def test_windowed_layer():
    w, t, q_raw, weight = prompts()
    n = w.num_pool_pages
    to = moved(n, FAR16)
    k, v = put(t.k_pool, to, FAR16), put(t.v_pool, to, FAR16)
    far = dataclasses.replace(w, unit_pages=to[w.unit_pages].astype(np.int32), free_pages=to[w.free_pages].astype(np.int32), num_pool_pages=FAR16)
    outs = []
    for x, kk, vv in ((w, t.k_pool, t.v_pool), (far, k, v)):
        t.k_pool, t.v_pool = kk, vv
        out, lse = torch.zeros_like(t.q), torch.zeros(w.n_q, 32, device=DEV)
        plan = tb.Plan(x, window=200, n_sink=4)
        layer(plan, t, q_raw, weight, out, lse)
        assert plan.status() == 0
        outs.append((out, lse))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and outs[0][0].isfinite().all() and outs[0][0].any()


def test_a_captured_windowed_layer():
    w, t, q_raw, weight = prompts()
    plan = tb.Plan(w, window=200, n_sink=4)
    out, lse = torch.zeros_like(t.q), torch.zeros(w.n_q, 32, device=DEV)
    layer(plan, t, q_raw, weight, out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(plan, t, q_raw, weight, out, lse)
    for seed in range(2):
        for x in (q_raw, t.k_new, t.v_new):
            x.copy_(torch.randn(x.shape, device=DEV).to(torch.bfloat16))
        graph.replay()
        got = out.clone(), lse.clone()
        layer(plan, t, q_raw, weight, out, lse)
        torch.cuda.synchronize()
        assert torch.equal(out, got[0]) and torch.equal(lse, got[1]) and out.isfinite().all()
    assert plan.status() == 0


@pytest.mark.parametrize("four", [False, True])
def test_two_graphs_one_after_the_other_share_a_workspace(four):
    c = Case([9000, 300, 5], 32, 8, 128, 64, seed=1, four=four)
    want = c.run().check().out.clone()
    graphs = []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.run()
            c.run()
    for g in graphs * 3:
        c.out.zero_()
        g.replay()
        assert torch.equal(c.out, want)


def test_a_decode_made_on_a_busy_stream_is_ready_for_another():
    c = Case([9000, 300], 8, 2, 128, 64, seed=2)
    size, side = c.decode.workspace.numel(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        used = torch.full((size,), 255, dtype=torch.uint8, device=DEV)       # (what the workspace may be made of)
        del used
        torch.cuda._sleep(50_000_000)
        dec = tb.Decode(c.shape, c.decode.block_table, c.decode.seq_lens, c.n_pages)
    c.decode = dec
    c.run().check()
    del dec


def test_no_decode_is_made_inside_a_capture():
    c = Case([100], 8, 2, 128, 64)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.out.zero_()
        with pytest.raises(ValueError):
            tb.Decode(c.shape, c.decode.block_table, c.decode.seq_lens, c.n_pages)


def test_q_out_right_behind_the_rows():
    """One buffer: the rows of q, then q_out; the heads of q_out in the place of a fused projection's are refused."""
    c = Case([100, 7, 64], 8, 2, 128, 16)
    x = torch.randn(6, 8, 128, device=DEV).to(torch.bfloat16)
    kv = torch.randn(3, 2, 128, device=DEV).to(torch.bfloat16)
    want = torch.empty_like(x[:3])
    c.decode.write(c.k, c.v, x[:3], want, kv, kv)
    c.decode.write(c.k, c.v, x[:3], x[3:], kv, kv)
    assert torch.equal(x[3:], want)
    with pytest.raises(tb.TesseraError):
        c.decode.write(c.k, c.v, x[1:4], x[:3], kv, kv)
