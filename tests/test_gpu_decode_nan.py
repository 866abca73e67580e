"""Decode attention where every score of a row is NaN: out and lse are NaN; lse = -inf stays with requests that see no key."""
import pytest
import torch

from tests.test_gpu_decode import DEV, Case

pytestmark = pytest.mark.gpu
NAN4 = [0xC0, 0x7F] * 4               # a 4-bit row's numbers, all NaN


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("hq,h,d", [(8, 2, 128), (10, 2, 128), (16, 1, 64)])
@pytest.mark.parametrize("lens", [[77, 0, 5], [300, 0, 40], [20011, 0, 90], [64] * 150 + [0, 3]])
def test_a_query_of_nan(lens, hq, h, d, four):
    """Pairs that a warp has to itself, that a block's warps join, and that blocks join."""
    c = Case(lens, hq, h, d, 64, seed=31, four=four)
    g, empty = hq // h, lens.index(0)
    c.q[0, 1, 3] = float("nan")
    c.q[0, g * (h - 1):, 5] = float("nan")                # all queries of the last KV head
    bad = torch.zeros(len(lens), hq, dtype=torch.bool, device=DEV)
    bad[0, 1] = True
    bad[0, g * (h - 1):] = True
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.lse.isnan(), bad)
    assert torch.equal(c.out.isnan(), bad[..., None].expand_as(c.out))
    none = torch.zeros_like(bad)
    none[empty] = True
    assert torch.equal(c.lse == -torch.inf, none) and (c.out[empty] == 0).all()


@pytest.mark.parametrize("four", [False, True])
def test_a_lone_key_of_nan(four):
    c = Case([1, 0, 1], 8, 2, 128, 16, seed=32, four=four)
    slot = int(c.slots(0)[0])
    if four:
        c.k[:, :, 16 * 64:].view(c.n_pages, 2, 16, 8)[slot // 16, 1, slot % 16] = torch.tensor(NAN4, dtype=torch.uint8, device=DEV)
    else:
        c.k.view(-1, 2, 128)[slot, 1, 7] = float("nan")
    c.run()
    torch.cuda.synchronize()
    assert c.lse[0, 4:].isnan().all() and c.out[0, 4:].isnan().all()
    assert c.lse[0, :4].isfinite().all() and c.out[0, :4].isfinite().all() and c.lse[2].isfinite().all()
    assert (c.lse[1] == -torch.inf).all() and (c.out[1] == 0).all()
