"""Batches whose tiles of keys pass 64 bits are refused as those that pass 32 are, on the CPU."""
import pytest

from paper_2609_32999_b200 import binding as tb
from tests import test_decode_refusals as td


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("heads,batch,pages", [(128, 2**30, 2**26), (4096, 2**26, 2**25), (4096, 2**31 - 1, 2**26), (4096, 2**31 - 1, 0), (1, 2**30, 2)])
def test_too_many_tiles(heads, batch, pages, four):
    c, d = td.cfg(num_q_heads=heads, num_kv_heads=heads), td.desc(batch=batch, max_pages=pages)
    assert td.attn(c, d, four=four) == tb.UNSUPPORTED_SHAPE and "tiles" in tb.last_error()
    assert td.write(c, d, td.rows(), four=four) == tb.UNSUPPORTED_SHAPE


def test_the_largest_batch_is_not():
    """(2^31 - 1 tiles and no device address that anything could follow: the null pool is what is refused)"""
    c, d = td.cfg(num_q_heads=1, num_kv_heads=1), td.desc(batch=2**31 - 1, max_pages=0)
    assert td.attn(c, d, k=None) == tb.INVALID_ARG and "k_pool" in tb.last_error()
