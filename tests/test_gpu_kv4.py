"""The 4-bit tier: codes, scales and least values bit for bit, and what comes back."""
import numpy as np
import pytest
import torch

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl
from tests import kv4_ref as k4
from tests.test_gpu_norm_write import near, turned

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPES = [(4, 2, 64, 16, 0), (32, 8, 128, 64, 0), (2, 1, 128, 8, 1), (3, 3, 64, 128, 1), (10, 5, 128, 32, 0)]


def tier(shape, lens, moved, seed=0, offset=0):
    """Plans that store units of these lengths and bring them back `moved` further on; slots of their tokens in the three pools."""
    rng = np.random.default_rng(seed)
    B, n = shape.page_size, len(lens)
    src_per, per = [-(-(x + offset) // B) for x in lens], [-(-x // B) for x in lens]
    pages = [rng.permutation(sum(src_per) + 2)[: sum(src_per)], rng.permutation(sum(per) + 2)[: sum(per)], rng.permutation(sum(per) + 4)[: sum(per)]]
    zeros = np.zeros(n, np.int32)

    def plan(units, counts, dest, pool, sources, cached, off):
        w = wl.Workload("tier", shape, np.array(lens, np.int32), np.arange(n + 1, dtype=np.int32), np.array(lens, np.int32), cached.astype(np.int32),
                        np.ones(n, np.int32), zeros, np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), units.astype(np.int32),
                        np.zeros(n + 1, np.int32), np.zeros(0, np.int32), dest.astype(np.int32), pool, unit_src_offset=np.full(n, off, np.int32),
                        num_source_pages=sources)
        return tb.Plan(w)

    store = plan(pages[0], src_per, pages[1], sum(per) + 2, sum(src_per) + 2, zeros, offset)
    load = plan(pages[1], per, pages[2], sum(per) + 4, sum(per) + 2, -np.array(moved), 0)
    u, i = np.repeat(np.arange(n), lens), np.concatenate([np.arange(x) for x in lens])

    def slots(pg, counts, off):
        first = np.concatenate([[0], np.cumsum(counts)])[u]
        return torch.from_numpy(pg[first + (i + off) // B].astype(np.int64) * B + (i + off) % B).to(DEV)

    at = slots(pages[0], src_per, offset), slots(pages[1], per, 0), slots(pages[2], per, 0)
    return store, load, at, (sum(src_per) + 2, sum(per) + 2, sum(per) + 4), torch.from_numpy(np.array(moved)[u]).to(DEV)


def rows_equal(four, want, slots, page, d, untouched=0xA5):
    n, h, _ = four.shape
    expect = torch.full_like(four, untouched)
    split = lambda x: (x[:, :, : page * (d // 2)].view(n, h, page, d // 2), x[:, :, page * (d // 2):].view(n, h, page, 8))
    src = split(k4.pool4(want))
    for a, c in zip(split(expect), src):
        a[slots // page, :, slots % page] = c[slots // page, :, slots % page]
    # (NaN: any NaN will do)
    a, b = split(four), split(expect)
    assert torch.equal(a[0], b[0])
    fa, fb = (x[1].contiguous().view(torch.bfloat16) for x in (a, b))
    assert ((fa == fb) | (fa.isnan() & fb.isnan())).all()


def strange(x):
    """Rows that are awkward to quantise, in the first tokens of a pool [slots][H][D]."""
    h, d = x.shape[1:]
    x[0] = 0
    x[1] = 5.5
    x[2] = torch.arange(d, device=x.device) * 1.0                       # many exact ties
    x[3] = (torch.arange(d, device=x.device) % 31) * 0.5 - 3.0
    x[4, :, 3] = float("nan")
    x[5, :, d - 1] = float("inf")
    x[6, :, 0] = float("-inf")
    x[7, :, 1], x[7, :, 2] = 3e38, -3e38                                # range above fp32's
    x[8] = torch.randn(h, d, device=x.device).to(x.dtype) * 2e38 / 4
    x[9] = torch.randn(h, d, device=x.device).to(x.dtype) * 3e-30       # scales around the smallest that is kept
    x[10] = torch.randn(h, d, device=x.device).to(x.dtype) * 1e-40
    x[11] = 1000 + torch.randn(h, d, device=x.device).to(x.dtype)
    x[12, :, : d // 2] = 1e30
    x[13] = -x[2]
    x[14] = (torch.arange(d, device=x.device) % 16) * 2.0 ** -96


@pytest.mark.parametrize("hq,h,d,page,pairing", SHAPES)
@pytest.mark.parametrize("offset", [0, 5])
def test_store_and_load(hq, h, d, page, pairing, offset):
    shape = wl.ModelShape(hq, h, d, page, 10000.0, rope_pairing=pairing)
    lens = [page, 1, 37, 3 * page + 1, 100, page - 1]
    store, load, at, pools, moved = tier(shape, lens, [0, 1, -100, 30000, 7, 512], offset=offset)
    k, v = (torch.randn(pools[0], page, h, d, device=DEV).to(torch.bfloat16) for _ in range(2))
    kk, vv = k.view(-1, h, d), v.view(-1, h, d)
    sp = torch.randn(len(at[0]), h, d, device=DEV).to(torch.bfloat16)
    strange(sp)
    vv[at[0]] = sp
    kk[at[0][:4]] = sp[:4]
    k_4, v_4 = (torch.full(tb.pool4_shape(shape, pools[1]), 0xA5, dtype=torch.uint8, device=DEV) for _ in range(2))
    store.kv_retain_kv4(k, v, k_4, v_4, fuse_rope=False)
    torch.cuda.synchronize()
    for four, x in ((k_4, kk), (v_4, vv)):
        mid = torch.zeros(pools[1] * page, h, d, dtype=torch.bfloat16, device=DEV)
        mid[at[1]] = x[at[0]]
        rows_equal(four, mid.view(pools[1], page, h, d), at[1], page, d)
    ko, vo = (torch.full((pools[2], page, h, d), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    load.kv_compose_from_kv4(k_4, v_4, ko, vo)
    val_k, val_v = (k4.values(x, page, d).reshape(-1, h, d)[at[1]] for x in (k_4, v_4))
    # one rounding to fp32 (scale c + least; the product is exact), one to bf16; the range of fp32 ends inside some strange rows
    got = vo.view(-1, h, d)[at[2]]
    ok = val_v.isfinite()
    assert torch.equal(got.isfinite() | ~ok, torch.ones_like(ok))
    assert torch.equal(got[ok], val_v[ok].float().to(torch.bfloat16))
    assert got[~ok].isnan().all()
    want, size = turned(val_k, moved, 10000.0, pairing)
    near(ko.view(-1, h, d)[at[2]], want, size + val_k.abs().amax(-1, keepdim=True), d)
    still = moved == 0
    assert torch.equal(ko.view(-1, h, d)[at[2]][still], val_k[still].float().to(torch.bfloat16))
    left = torch.ones(pools[2] * page, dtype=torch.bool, device=DEV)
    left[at[2]] = False
    assert (ko.view(-1, h, d)[left] == 3).all() and (vo.view(-1, h, d)[left] == 3).all()


@pytest.mark.parametrize("hq,h,d,page,pairing", SHAPES)
def test_store_rotated(hq, h, d, page, pairing):
    """With the rotation a store keeps the quantised form of the rows that a 16-bit copy of the same plan would hold."""
    shape = wl.ModelShape(hq, h, d, page, 10000.0, rope_pairing=pairing)
    _, load, at, pools, moved = tier(shape, [page + 3, 40], [900, -3])
    k, v = (torch.randn(pools[1], page, h, d, device=DEV).to(torch.bfloat16) for _ in range(2))
    k2, v2 = torch.zeros(pools[2], page, h, d, dtype=torch.bfloat16, device=DEV), torch.zeros(pools[2], page, h, d, dtype=torch.bfloat16, device=DEV)
    load.kv_compose_from(k, v, k2, v2)
    k_4, v_4 = (torch.full(tb.pool4_shape(shape, pools[2]), 0xA5, dtype=torch.uint8, device=DEV) for _ in range(2))
    load.kv_retain_kv4(k, v, k_4, v_4)
    rows_equal(k_4, k2, at[2], page, d)
    rows_equal(v_4, v2, at[2], page, d)


def test_refusals():
    shape = wl.ModelShape(4, 2, 64, 16, 10000.0)
    w = wl.build_workload("here", shape, [[wl.unit(40)]], np.random.default_rng(0))
    x = torch.zeros(8, 16, 2, 64, dtype=torch.bfloat16, device=DEV)
    f = torch.zeros(tb.pool4_shape(shape, 8), dtype=torch.uint8, device=DEV)
    for call in (lambda p: p.kv_retain_kv4(x, x, f, f), lambda p: p.kv_compose_from_kv4(f, f, x, x)):
        with pytest.raises(tb.TesseraError) as e:
            call(tb.Plan(w))                        # no separate source pool
        assert e.value.status == tb.INVALID_ARG
        with pytest.raises(tb.TesseraError):
            call(tb.Plan(w, host_only=True))
    w.num_source_pages = 8
    with pytest.raises(tb.TesseraError):
        tb.Plan(w).kv_retain_kv4(x, None, f, f)
    with pytest.raises(tb.TesseraError):
        tb.Plan(w).kv_retain_kv4(x, x, f.view(-1)[8:], f)
