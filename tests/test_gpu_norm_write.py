"""Fresh rows with per-head norms: values against 64 bits, slots and everything around them bit for bit."""
import numpy as np
import pytest
import torch

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl
from tests import kv4_ref as k4

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP32 = 2.0 ** -8, 2.0 ** -24


def turned(x, pos, theta, pairing):
    """[n][heads][D] in 64 bits, and the size of the two terms of every element."""
    d = x.shape[-1]
    ang = pos.double()[:, None] * theta ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / d)
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    a, b = (x[..., : d // 2], x[..., d // 2:]) if pairing == 0 else (x[..., 0::2], x[..., 1::2])
    parts = [(a * c - b * s, (a * c).abs() + (b * s).abs()), (b * c + a * s, (b * c).abs() + (a * s).abs())]
    join = (lambda u, v: torch.cat([u, v], -1)) if pairing == 0 else (lambda u, v: torch.stack([u, v], -1).reshape(x.shape))
    return join(parts[0][0], parts[1][0]), join(parts[0][1], parts[1][1])


def normed(x, w, eps):
    x = x.double()
    return x if w is None else x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()


def near(got, want, size, d):
    """One rounding to bf16; in fp32 before it the sum of D squares (under a root: half its error), the reciprocal root (2 steps), two
    products, the table's rounding, two products and a sum of the rotation."""
    tol = BF16 * want.abs() * 1.01 + (d / 2 + 12) * FP32 * size + 1e-37
    assert ((got.double() - want).abs() <= tol).all()


def workload(shape, seed=0, retain=True):
    rng = np.random.default_rng(seed)
    reqs = [[17, wl.unit(70, "a", cached=False), 9, wl.unit(50, "b", recompute=(0, 3, 49))], [wl.unit(33, "c", cached=False)], [1], [5, wl.unit(200, "d", recompute=range(11))]]
    w = wl.build_workload("norm", shape, reqs, rng)
    if retain:             # the two missed units are captured into a cache pool of their own
        per = [-(-int(n) // shape.page_size) if c else 0 for n, c in zip(w.unit_len, np.diff(w.unit_page_off) == 0)]
        w.unit_retain_page_off = np.concatenate([[0], np.cumsum(per)]).astype(np.int32)
        w.unit_retain_pages = rng.permutation(sum(per) + 2)[: sum(per)].astype(np.int32)
        w.retain_pool_pages = sum(per) + 2
    return w


@pytest.mark.parametrize("norms", ["both", "q", "k", "none"])
@pytest.mark.parametrize("hq,h,d,page,pairing", [(4, 2, 64, 16, 0), (32, 8, 128, 64, 0), (10, 2, 128, 8, 1), (3, 3, 64, 128, 1), (80, 5, 128, 32, 0)])
def test_extend(hq, h, d, page, pairing, norms):
    shape = wl.ModelShape(hq, h, d, page, 10000.0, rope_pairing=pairing)
    w = workload(shape)
    t = wl.make_tensors(w, device=DEV, seed=2)
    t.q.mul_(5)
    t.k_new.mul_(0.01)
    t.q[3, 0] = 0                                    # a head of zeros: eps keeps it
    qw = (1 + 0.3 * torch.randn(d, device=DEV)).to(torch.bfloat16) if norms in ("both", "q") else None
    kw = (1 + 0.3 * torch.randn(d, device=DEV)).to(torch.bfloat16) if norms in ("both", "k") else None
    eps, plan = 1e-5, tb.Plan(w)
    k0, v0 = t.k_pool.clone(), t.v_pool.clone()
    kc, vc = (torch.full((w.retain_pool_pages, page, h, d), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q_out = torch.full_like(t.q, 9.0)
    plan.extend_write_norm(t.k_pool, t.v_pool, t.q, q_out, t.k_new, t.v_new, qw, kw, eps, kc, vc)
    torch.cuda.synchronize()
    page_off, pages, _ = plan.block_table()
    req = np.repeat(np.arange(w.batch), np.diff(w.recompute_off))
    p = w.recompute_pos.astype(np.int64)
    slot = torch.from_numpy(pages[page_off[req] + p // page].astype(np.int64) * page + p % page).to(DEV)
    pos = torch.from_numpy(p).to(DEV)
    near(q_out, *turned(normed(t.q, qw, eps), pos, 10000.0, pairing), d)
    near(t.k_pool.view(-1, h, d)[slot], *turned(normed(t.k_new, kw, eps), pos, 10000.0, pairing), d)
    assert torch.equal(t.v_pool.view(-1, h, d)[slot], t.v_new)
    for now, before in ((t.k_pool, k0), (t.v_pool, v0)):
        now, before = now.view(-1, h, d).clone(), before.view(-1, h, d)
        now[slot] = before[slot]
        assert torch.equal(now, before)
    if norms == "none":             # the plain write's bits, q where it was told to go
        q2, k2, v2, kc2, vc2 = t.q.clone(), k0.clone(), v0.clone(), torch.full_like(kc, 3.0), torch.full_like(vc, 3.0)
        plan.extend_write(k2, v2, q2, t.k_new, t.v_new, kc2, vc2)
        for a, b in ((q2, q_out), (k2, t.k_pool), (v2, t.v_pool), (kc2, kc), (vc2, vc)):
            assert torch.equal(a, b)
    # captured: the key before rotation
    left = torch.ones(w.retain_pool_pages * page, dtype=torch.bool, device=DEV)
    for r in range(w.batch):
        for u in range(w.unit_off[r], w.unit_off[r + 1]):
            lo, hi = w.unit_retain_page_off[u], w.unit_retain_page_off[u + 1]
            if lo == hi:
                continue
            i = np.arange(int(w.unit_len[u]))
            at = torch.from_numpy(w.unit_retain_pages[lo + i // page].astype(np.int64) * page + i % page).to(DEV)
            rows = torch.from_numpy(w.recompute_off[r] + np.searchsorted(p[w.recompute_off[r]:w.recompute_off[r + 1]], int(w.unit_target_pos[u]) + i)).to(DEV)
            want = normed(t.k_new[rows], kw, eps)
            near(kc.view(-1, h, d)[at], want, want.abs(), d)
            assert torch.equal(vc.view(-1, h, d)[at], t.v_new[rows])
            left[at] = False
    assert (kc.view(-1, h, d)[left] == 3).all() and (vc.view(-1, h, d)[left] == 3).all()


def test_extend_in_place_and_from_a_fused_projection():
    shape = wl.ModelShape(8, 2, 128, 16, 10000.0)
    w = workload(shape, retain=False)
    t = wl.make_tensors(w, device=DEV, seed=3)
    weight = (1 + 0.3 * torch.randn(128, device=DEV)).to(torch.bfloat16)
    plan, q_out = tb.Plan(w), torch.empty_like(t.q)
    plan.extend_write_norm(t.k_pool, t.v_pool, t.q, q_out, t.k_new, t.v_new, weight, weight)
    fused = torch.cat([t.q, t.k_new, t.v_new], 1).contiguous()
    k2, v2, q2, q3 = torch.zeros_like(t.k_pool).copy_(t.k_pool), t.v_pool.clone(), torch.empty_like(t.q), t.q.clone()
    plan.extend_write_norm(k2, v2, fused[:, :8], q2, fused[:, 8:10], fused[:, 10:], weight, weight)
    plan.extend_write_norm(k2, v2, q3, q3, t.k_new, t.v_new, weight, weight)
    plan.extend_write_norm(k2, v2, None, None, t.k_new, t.v_new, None, weight)
    for a, b in ((q_out, q2), (q_out, q3), (t.k_pool, k2), (t.v_pool, v2)):
        assert torch.equal(a, b)


def decode_case(shape, lens, seed=0, wide=0):
    rng = np.random.default_rng(seed)
    per = [max(0, -(-x // shape.page_size)) for x in lens]
    n = sum(per) + 3
    perm = rng.permutation(n)
    table = np.full((len(lens), max(per) + wide), -1, np.int32)
    at = 0
    for r, c in enumerate(per):
        table[r, :c] = perm[at:at + c]
        at += c
    return n, table


@pytest.mark.parametrize("hq,h,d,page,pairing", [(4, 2, 64, 16, 0), (32, 8, 128, 64, 0), (10, 2, 128, 8, 1), (3, 3, 64, 128, 1), (16, 1, 128, 32, 0), (128, 8, 128, 64, 0)])
@pytest.mark.parametrize("norms", [True, False])
def test_step(hq, h, d, page, pairing, norms):
    shape = wl.ModelShape(hq, h, d, page, 500000.0, rope_pairing=pairing)
    lens = [1, 0, 17, 64, 65, -5, 1000, 90, 333]
    n, table = decode_case(shape, lens)
    table[7, (90 - 1) // page] = n + 4               # the new token's page is not in the pool
    lens.append(10 ** 6)                             # nor in the table
    table = np.concatenate([table, np.zeros((1, table.shape[1]), np.int32)])
    b = len(lens)
    dec = tb.Decode(shape, torch.from_numpy(table).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), n)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(5)
    draw = lambda heads: torch.randn(b, heads, d, generator=gen, device=DEV).to(torch.bfloat16)
    q, k, v = 4 * draw(hq), draw(h), draw(h)
    qw, kw = ((1 + 0.2 * draw(1)[0, 0]) if norms else None for _ in range(2))
    kp, vp = (torch.full((n, page, h, d), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q_out = torch.full_like(q, 9.0)
    dec.write(kp, vp, q, q_out, k, v, qw, kw, 1e-6)
    torch.cuda.synchronize()
    fine = [r for r in range(b) if 0 < lens[r] <= table.shape[1] * page and 0 <= table[r, (lens[r] - 1) // page] < n]
    assert fine == [0, 2, 3, 4, 6, 8]
    pos = torch.tensor([lens[r] - 1 for r in fine], device=DEV)
    slot = torch.tensor([int(table[r, (lens[r] - 1) // page]) * page + (lens[r] - 1) % page for r in fine], device=DEV)
    near(q_out[fine], *turned(normed(q[fine], qw, 1e-6), pos, 500000.0, pairing), d)
    near(kp.view(-1, h, d)[slot], *turned(normed(k[fine], kw, 1e-6), pos, 500000.0, pairing), d)
    assert torch.equal(vp.view(-1, h, d)[slot], v[fine])
    rest = [r for r in range(b) if r not in fine]
    assert (q_out[rest] == 9).all()
    left = torch.ones(n * page, dtype=torch.bool, device=DEV)
    left[slot] = False
    assert (kp.view(-1, h, d)[left] == 3).all() and (vp.view(-1, h, d)[left] == 3).all()
    # 4-bit pools keep the quantised form of these very rows, and nothing else changes
    k_4, v_4 = (torch.full(tb.pool4_shape(shape, n), 0xA5, dtype=torch.uint8, device=DEV) for _ in range(2))
    q2 = torch.full_like(q, 9.0)
    dec.write_kv4(k_4, v_4, q, q2, k, v, qw, kw, 1e-6)
    assert torch.equal(q2, q_out)
    for four, sixteen in ((k_4, kp), (v_4, vp)):
        want = torch.full_like(four, 0xA5)
        full = k4.pool4(sixteen)
        split = lambda x: (x[:, :, : page * (d // 2)].view(n, h, page, d // 2), x[:, :, page * (d // 2):].view(n, h, page, 8))
        for a, c in zip(split(want), split(full)):
            a[slot // page, :, slot % page] = c[slot // page, :, slot % page]
        assert torch.equal(four, want)


def test_far_positions():
    shape = wl.ModelShape(4, 1, 128, 128, 10000.0)
    lens = [1048576, 999999]
    table = np.zeros((2, 8192), np.int32)
    table[1] = 1
    dec = tb.Decode(shape, torch.from_numpy(table).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), 2)
    q, k, v = (torch.randn(2, n, 128, device=DEV).to(torch.bfloat16) for n in (4, 1, 1))
    kp, vp, q_out = torch.zeros(2, 128, 1, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 128, 1, 128, dtype=torch.bfloat16, device=DEV), torch.empty_like(q)
    dec.write(kp, vp, q, q_out, k, v)
    pos = torch.tensor(lens, device=DEV) - 1
    near(q_out, *turned(q.double(), pos, 10000.0, 0), 128)
