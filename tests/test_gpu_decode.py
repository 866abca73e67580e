"""Decode attention over 16-bit and 4-bit pages against attention in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl
from tests import attn_ref as ar
from tests import kv4_ref as k4

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPES = [(4, 2, 64, 16), (32, 8, 128, 64), (10, 2, 128, 8), (3, 3, 64, 128), (16, 1, 128, 32), (9, 1, 64, 8), (7, 1, 128, 128), (16, 1, 64, 64), (8, 1, 128, 16)]
LENS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 700, 0, -3, 1025, 4097]


class Case:
    """Pools with spare pages, a table in random page order, NaN and infinities wherever no request's tokens are."""

    def __init__(self, lens, hq, h, d, page, seed=0, four=False, window=0, n_sink=0, scale=0.0, wide=2, q_size=1.0):
        self.lens, self.page, self.d, self.four, self.window, self.n_sink = lens, page, d, four, window, n_sink
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.shape = wl.ModelShape(hq, h, d, page, 10000.0, sm_scale=scale)
        per = [max(0, -(-t // page)) for t in lens]
        n_pages = sum(per) + 5
        perm = rng.permutation(n_pages)
        self.table = np.full((len(lens), max(per + [0]) + wide), 2**30, np.int32)
        at = 0
        for r, n in enumerate(per):
            self.table[r, :n] = perm[at:at + n]
            at += n
        k = torch.randn(n_pages, page, h, d, generator=g, device=DEV).to(torch.bfloat16)
        v = torch.randn(n_pages, page, h, d, generator=g, device=DEV).to(torch.bfloat16)
        self.q = (q_size * torch.randn(len(lens), hq, d, generator=g, device=DEV)).to(torch.bfloat16)
        self.k, self.v = (k4.pool4(k), k4.pool4(v)) if four else (k, v)
        self.n_pages = n_pages
        seen = np.zeros(n_pages * page, bool)
        for r in range(len(lens)):
            seen[self.slots(r)] = True
        self.spoil(torch.from_numpy(np.flatnonzero(~seen)).to(DEV))
        self.decode = tb.Decode(self.shape, torch.from_numpy(self.table).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), n_pages,
                                window=window, n_sink=n_sink)
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full((len(lens), hq), 7.0, device=DEV)

    def spoil(self, slots):
        if self.four:
            page, d = self.page, self.d
            for pool in (self.k, self.v):
                pool[:, :, : page * (d // 2)].view(self.n_pages, -1, page, d // 2)[slots // page, :, slots % page] = 255
                # scale infinite, least NaN
                bad = torch.tensor([0x80, 0x7F, 0xC0, 0x7F] * 2, dtype=torch.uint8, device=DEV)
                pool[:, :, page * (d // 2):].view(self.n_pages, -1, page, 8)[slots // page, :, slots % page] = bad
        else:
            self.k.view(-1, *self.k.shape[2:])[slots] = float("nan")
            self.v.view(-1, *self.v.shape[2:])[slots] = float("inf")

    def slots(self, r):
        """Slots of the request's visible keys."""
        t = min(self.lens[r], self.table.shape[1] * self.page)
        key = np.arange(max(t, 0))
        if self.window:
            key = key[(key < self.n_sink) | (key > t - 1 - self.window)]
        page = self.table[r, key // self.page].astype(np.int64)
        ok = (page >= 0) & (page < self.n_pages)
        return page[ok] * self.page + key[ok] % self.page

    def run(self, stream=None, **kw):
        call = self.decode.attn_kv4 if self.four else self.decode.attn
        call(self.k, self.v, self.q, self.out, self.lse, stream=stream, **kw)
        return self

    def check(self, scale=None):
        torch.cuda.synchronize()
        if self.four:
            (kc, ks, km), (vc, vs, vm) = (k4.parts(x, self.page, self.d) for x in (self.k, self.v))
            kv, vv = (k4.values(x, self.page, self.d) for x in (self.k, self.v))
            # the terms the kernel sums: q times c times the scale, and the least value; p times scale times (c - 8), and p times the middle
            ka = (kc.float() * ks[..., None] + km.abs()[..., None]).reshape(kv.shape)
            va = (vs[..., None] * (vc.float() - 8).abs()).reshape(vv.shape)
            # (with at most 4 queries a KV head the first half's codes come as bytes less the second's: c0 + 16 c1 - 16 c1, and -8, the middle)
            taken_off = torch.zeros_like(vc, dtype=torch.float32)
            if self.q.shape[1] <= 4 * ks.shape[2]:
                taken_off[..., 0, :] = 32 * vc[..., 1, :].float()
            vsum = (vs[..., None] * (vc.float() + taken_off + 8) + (vm + 8 * vs).abs()[..., None]).reshape(vv.shape)
        else:
            kv, vv, ka, va, vsum = self.k, self.v, None, None, None
        for r in range(len(self.lens)):
            at = torch.from_numpy(self.slots(r)).to(DEV)
            if len(at) == 0:
                assert (self.out[r] == 0).all() and (self.lse[r] == -torch.inf).all(), r
                continue
            row = lambda x: None if x is None else x.reshape(-1, *x.shape[2:])[at]
            pos = torch.tensor([len(at) - 1], device=DEV)
            want = ar.attend(self.q[r:r + 1], row(kv), row(vv), pos, scale=scale, k_size=row(ka), v_size=row(va), v_sum=row(vsum))
            ar.check(self.out[r:r + 1], self.lse[r:r + 1], want, len(at), "request %d of %d keys" % (r, len(at)))
        return self


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("hq,h,d,page", SHAPES)
def test_against_64_bits(hq, h, d, page, four):
    Case(LENS, hq, h, d, page, four=four).run().check()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("hq,h,d,page", [(4, 2, 64, 16), (32, 8, 128, 64), (16, 1, 128, 8)])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (64, 4), (100, 130), (500, 3), (2**31 - 1, 0), (5, 2**31 - 1)])
def test_window(hq, h, d, page, window, n_sink, four):
    Case(LENS, hq, h, d, page, seed=1, four=four, window=window, n_sink=n_sink).run().check()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("lens", [[20011], [9000, 1, 30000], [64] * 148, [65] * 149, [1] * 1100, [3, 0] * 300 + [5000]])
def test_shares(lens, four):
    """One long request, as many units as blocks, one more, batches of more requests than a block has threads."""
    Case(lens, 8, 2, 128, 64, seed=2, four=four, wide=1).run().check()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("q_size,scale", [(40.0, 0.0), (1.0, 3.0), (0.0, 0.0)])
def test_score_sizes(q_size, scale, four):
    c = Case([1, 100, 3000], 8, 2, 128, 64, seed=3, four=four, q_size=q_size, scale=scale)
    c.run().check(scale or None)


@pytest.mark.parametrize("hq,h,d,page", [(8, 2, 128, 64), (16, 2, 64, 16), (12, 1, 128, 8)])
@pytest.mark.parametrize("size", [1e-25, 1e-6, 1.0, 1e6, 1e20, 1e33])
def test_sizes_of_4_bit_values(size, hq, h, d, page):
    """Values of any size, and a request whose values grow and shrink by far between tiles."""
    c = Case([1, 90, 700, 40], hq, h, d, page, seed=21, four=True)
    v = size * torch.randn(c.n_pages, page, h, d, device=DEV)
    keep = c.v.clone()
    for r, grow in ((2, [1, 1e-9, 1e4, 1e-3, 1e15]), (3, [1e-6, 1])):
        for i, f in enumerate(grow):
            at = torch.from_numpy(c.slots(r)[i * 130:(i + 1) * 130 if i + 1 < len(grow) else None]).to(DEV)
            v.view(-1, h, d)[at] *= min(f, 1e37 / size / 16)
    new, page_of = k4.pool4(v.to(torch.bfloat16)), torch.from_numpy(np.concatenate([c.slots(r) for r in range(4)])).to(DEV)
    split = lambda x: (x[:, :, : page * (d // 2)].view(c.n_pages, h, page, d // 2), x[:, :, page * (d // 2):].view(c.n_pages, h, page, 8))
    for a, b in zip(split(keep), split(new)):
        a[page_of // page, :, page_of % page] = b[page_of // page, :, page_of % page]
    c.v.copy_(keep)
    c.run().check()


def test_4_bit_rows_of_one_value_and_of_nan():
    c = Case([200, 77, 64], 8, 2, 128, 16, seed=22, four=True)
    d, page = 128, 16
    par = c.v[:, :, page * (d // 2):].view(c.n_pages, 2, page, 8)
    at = torch.from_numpy(c.slots(0)).to(DEV)
    par[at // page, :, at % page] = torch.tensor([0, 0, 0x80, 0x7E, 0, 0, 0x80, 0xBF], dtype=torch.uint8, device=DEV)      # scales 0, leasts 2^126 and -1
    par = c.k[:, :, page * (d // 2):].view(c.n_pages, 2, page, 8)
    bad = int(c.slots(1)[50])
    par[bad // page, 1, bad % page] = torch.tensor([0xC0, 0x7F] * 4, dtype=torch.uint8, device=DEV)
    c.run()
    torch.cuda.synchronize()
    # weights of 200 equal values sum to far more than 4 before they are divided by: 4 times 2^126 is no fp32 number any more
    assert c.out[0, :, :64].isinf().all() and (c.out[0, :, 64:] == -1).all()
    par = c.v[:, :, page * (d // 2):].view(c.n_pages, 2, page, 8)
    par[at // page, :, at % page] = torch.tensor([0, 0, 0x80, 0x71, 0, 0, 0x80, 0xBF], dtype=torch.uint8, device=DEV)      # 2^100
    c.run()
    assert (c.out[0, :, :64].float() == 2.0 ** 100).all() and (c.out[0, :, 64:] == -1).all()
    assert c.out[1, 4:].isnan().all() and c.lse[1, 4:].isnan().all() and c.out[1, :4].isfinite().all() and c.lse[1, :4].isfinite().all()
    assert c.out[2].isfinite().all()


@pytest.mark.parametrize("q_size", [1e-30, 1e-4, 1e4])
def test_sizes_of_queries_over_4_bit_keys(q_size):
    c = Case([1, 90, 700], 8, 2, 128, 64, seed=23, four=True, q_size=q_size, scale=0.088 / q_size if q_size > 1 else 0.0)
    c.q[1, 3, 5:] = 0
    c.q[2, 2] *= 2.0 ** torch.linspace(-40, 0, 128, device=DEV)
    c.run().check(0.088 / q_size if q_size > 1 else None)


@pytest.mark.parametrize("four", [False, True])
def test_negative_scale(four):
    Case([1, 33, 1000], 8, 2, 128, 64, seed=24, four=four, scale=-0.3, window=300, n_sink=5).run().check(-0.3)


@pytest.mark.parametrize("four", [False, True])
def test_pages_outside_the_pool_and_lengths_past_the_table(four):
    c = Case([300, 130, 64, 200], 8, 2, 128, 16, seed=4, four=four, wide=0)
    c.table[0, 3], c.table[0, 7], c.table[1, :], c.table[2, 0] = -1, c.n_pages, 2**31 - 1, -2**31
    c.lens[3] = 100000                             # more than the table has room for
    c.table[3, 13:] = -7
    c.decode.block_table.copy_(torch.from_numpy(c.table))
    c.decode.seq_lens.copy_(torch.tensor(c.lens, dtype=torch.int32))
    c.run().check()


@pytest.mark.parametrize("four", [False, True])
def test_a_length_past_a_full_table(four):
    c = Case([208, 96], 8, 2, 128, 16, seed=14, four=four, wide=0)       # (both requests' last pages are full, the second's table is not)
    c.lens = [100000, 97]
    c.decode.seq_lens.copy_(torch.tensor(c.lens, dtype=torch.int32))
    c.run().check()


@pytest.mark.parametrize("four", [False, True])
def test_same_bits_again_and_without_lse(four):
    c = Case([5000, 33, 700], 32, 8, 128, 64, seed=5, four=four).run()
    first = c.out.clone(), c.lse.clone()
    c.out.zero_()
    call = c.decode.attn_kv4 if four else c.decode.attn
    call(c.k, c.v, c.q, c.out)
    assert torch.equal(first[0], c.out)


@pytest.mark.parametrize("four", [False, True])
def test_streams_with_a_decode_each(four):
    cases = [Case([9000, 500 + 100 * i], 8, 2, 128, 64, seed=6 + i, four=four) for i in range(3)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(10):
        for c, s in zip(cases, streams):
            c.run(stream=s)
    for c in cases:
        c.check()


@pytest.mark.parametrize("four", [False, True])
def test_a_captured_step_follows_lengths_and_table(four):
    """Write and attention of a step in one graph, replayed while requests grow, end and begin."""
    lens = [1, 63, 64, 300, 0, 2000]
    c = Case([t + 8 if t else 0 for t in lens], 8, 2, 128, 16, seed=9, four=four)
    c.lens = list(lens)
    q, k, v = (torch.randn(6, n, 128, device=DEV).to(torch.bfloat16) for n in (8, 2, 2))
    weight = (1 + 0.1 * torch.randn(128, device=DEV)).to(torch.bfloat16)

    def step():
        write = c.decode.write_kv4 if four else c.decode.write
        write(c.k, c.v, q, c.q, k, v, weight, weight)
        c.run()

    c.decode.seq_lens.zero_()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(5):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device=DEV).to(torch.bfloat16))
        if n == 3:
            c.lens[1] = 0                           # ended
        c.lens = [t + 1 if t else 0 for t in c.lens]
        c.decode.seq_lens.copy_(torch.tensor(c.lens, dtype=torch.int32))
        graph.replay()
        c.check()


@pytest.mark.parametrize("four", [False, True])
def test_decode_after_a_composed_prompt(four):
    """Plan -> compose -> fresh rows with norms -> prefill attention -> (4-bit copy) -> decode steps, each against 64 bits."""
    rng = np.random.default_rng(3)
    shape = wl.ModelShape(8, 2, 128, 16, 10000.0)
    w = wl.build_workload("then-decode", shape, [[20, wl.unit(300, "a"), 31], [wl.unit(100, "b"), 7]], rng, spare_pages=9)
    t = wl.make_tensors(w, device=DEV, seed=1)
    weight = (1 + 0.1 * torch.randn(128, device=DEV)).to(torch.bfloat16)
    plan = tb.Plan(w, window=64, n_sink=4)
    plan.kv_compose(t.k_pool, t.v_pool)
    plan.extend_write_norm(t.k_pool, t.v_pool, t.q, t.q, t.k_new, t.v_new, weight, weight)
    out, lse = torch.zeros_like(t.q), torch.zeros(w.n_q, 8, device=DEV)
    plan.partial_prefill_attn(t.k_pool, t.v_pool, t.q, None, None, out, lse)
    page_off, pages, _ = plan.block_table()
    assert plan.status() == 0
    table = torch.zeros(2, 30, dtype=torch.int32)
    spare = iter(set(w.free_pages.tolist()) - set(pages.tolist()))
    for r in range(2):
        mine = pages[page_off[r]:page_off[r + 1]].tolist() + [next(spare), next(spare)]
        table[r, : len(mine)] = torch.tensor(mine, dtype=torch.int32)
    lens = torch.from_numpy(w.seq_len).to(DEV)
    for r in range(2):
        a, b = int(w.recompute_off[r]), int(w.recompute_off[r + 1])
        ids = torch.from_numpy(pages[page_off[r]:page_off[r + 1]].astype(np.int64)).to(DEV)
        kr, vr = (x[ids].reshape(-1, 2, 128)[: int(w.seq_len[r])] for x in (t.k_pool, t.v_pool))
        pos = torch.from_numpy(w.recompute_pos[a:b].astype(np.int64)).to(DEV)
        ar.check(out[a:b], lse[a:b], ar.attend(t.q[a:b], kr, vr, pos, 64, 4), len(kr), "prefill %d" % r)
    c = Case([1, 1], 8, 2, 128, 16)
    c.four, c.n_pages, c.window, c.n_sink, c.table = four, w.num_pool_pages, 64, 4, table.numpy()
    if four:                                        # the finished prompt's pages go to the 4-bit pool, page for page
        c.k, c.v = (torch.zeros(tb.pool4_shape(shape, w.num_pool_pages), dtype=torch.uint8, device=DEV) for _ in range(2))
        units = [wl.unit(int(x)) for x in w.seq_len]
        back = wl.build_workload("retain", shape, [[u] for u in units], rng, shuffle_pages=False)
        back.unit_pages, back.free_pages, back.num_source_pages, back.num_pool_pages = pages, pages, w.num_pool_pages, w.num_pool_pages
        tb.Plan(back).kv_retain_kv4(t.k_pool, t.v_pool, c.k, c.v, fuse_rope=False)
    else:
        c.k, c.v = t.k_pool, t.v_pool
    c.decode = tb.Decode(shape, table.to(DEV), lens, w.num_pool_pages, window=64, n_sink=4)
    c.out, c.lse = torch.zeros(2, 8, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 8, device=DEV)
    for _ in range(20):
        lens += 1
        fused = torch.randn(2, 12 * 128, device=DEV).to(torch.bfloat16)      # one projection: q, k and v side by side
        heads = fused.view(2, 12, 128)
        c.q = torch.empty(2, 8, 128, dtype=torch.bfloat16, device=DEV)
        write = c.decode.write_kv4 if four else c.decode.write
        write(c.k, c.v, heads[:, :8], c.q, heads[:, 8:10], heads[:, 10:], weight, weight)
        c.run()
        c.lens = lens.tolist()
        c.check()


def test_arguments():
    c = Case([10, 20], 8, 2, 128, 16)
    d = c.decode
    with pytest.raises(ValueError):
        d.attn(c.k, c.v, c.q.float(), c.out)
    with pytest.raises(ValueError):
        d.attn(c.k[:-1], c.v, c.q, c.out)
    with pytest.raises(ValueError):
        d.attn(c.k, c.v, c.q, c.out, c.lse.double())
    with pytest.raises(ValueError):
        d.attn_kv4(c.k, c.v, c.q, c.out)
    with pytest.raises(ValueError):
        d.write(c.k, c.v, c.q, c.out, c.k[0, :2], c.v[0, :2].expand(2, 2, 128).transpose(0, 1))
    with pytest.raises(ValueError):
        d.write(c.k, c.v, c.q, c.out, c.k[0, :1].expand(2, 2, 128), c.v[0, :2])
    with pytest.raises(ValueError):
        tb.Decode(c.shape, d.block_table.long(), d.seq_lens, c.n_pages)
    with pytest.raises(tb.TesseraError):
        d.workspace = d.workspace[:1024]
        d.attn(c.k, c.v, c.q, c.out)
