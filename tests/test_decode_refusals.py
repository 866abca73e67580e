"""What the decode and fresh-row entry points refuse, on the CPU: every check comes before the first use of a device."""
import ctypes

import numpy as np
import pytest

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl

P = 1 << 20          # stands for a device address; no call below gets as far as using it


def cfg(**kw):
    f = dict(num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, rope_theta=1e4, inv_freq=None, rope_pairing=0, sm_scale=0.0)
    f.update(kw)
    return tb.ModelCfg(*f.values())


def desc(**kw):
    f = dict(batch=3, max_pages=4, block_table=P, seq_len=P, num_pool_pages=100, window=0, n_sink=0)
    f.update(kw)
    return tb.DecodeDesc(*f.values())


def rows(**kw):
    f = dict(q=P, k=P, v=P, q_out=2 * P, q_row=0, k_row=0, v_row=0, q_weight=P, k_weight=P, eps=1e-6)
    f.update(kw)
    return tb.FreshRows(*f.values())


def attn(c, d, k=P, v=P, q=P, out=P, ws=P, size=1 << 30, four=False):
    call = tb._lib.tessera_decode_attn_kv4 if four else tb._lib.tessera_decode_attn
    return call(ctypes.byref(c), ctypes.byref(d), k, v, q, out, None, ws, size, None)


def write(c, d, r, k=P, v=P, four=False):
    call = tb._lib.tessera_decode_write_kv4 if four else tb._lib.tessera_decode_write
    return call(ctypes.byref(c), ctypes.byref(d), k, v, ctypes.byref(r), None)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("kw", [dict(num_q_heads=0), dict(num_q_heads=9), dict(num_q_heads=34), dict(num_kv_heads=0), dict(head_dim=96), dict(page_size=4),
                                dict(page_size=48), dict(page_size=256)])
def test_shapes(kw, four):
    assert attn(cfg(**kw), desc(), four=four) == tb.UNSUPPORTED_SHAPE
    assert write(cfg(**kw), desc(), rows(), four=four) == tb.UNSUPPORTED_SHAPE


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("kw,code", [(dict(batch=-1), tb.INVALID_ARG), (dict(max_pages=-1), tb.INVALID_ARG), (dict(num_pool_pages=-1), tb.INVALID_ARG),
                                     (dict(window=-1), tb.INVALID_ARG), (dict(n_sink=-1), tb.INVALID_ARG), (dict(seq_len=None), tb.INVALID_ARG),
                                     (dict(block_table=None), tb.INVALID_ARG), (dict(num_pool_pages=2**28), tb.UNSUPPORTED_SHAPE),
                                     (dict(max_pages=2**27), tb.UNSUPPORTED_SHAPE), (dict(batch=2**30, max_pages=1024), tb.UNSUPPORTED_SHAPE)])
def test_descriptions(kw, code, four):
    assert attn(cfg(), desc(**kw), four=four) == code
    assert write(cfg(), desc(**kw), rows(), four=four) == code
    assert tb.last_error()


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(q=None), dict(out=None), dict(k=P + 8), dict(v=P + 2), dict(q=P + 4), dict(out=P + 8)])
def test_attention_pointers(kw):
    assert attn(cfg(), desc(), **kw) == tb.INVALID_ARG


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(q_out=None), dict(q=P + 8), dict(k=P + 2), dict(v=P + 8), dict(q_out=P + 8), dict(q_weight=P + 2),
                                dict(k_weight=P + 4), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(q_row=1016), dict(q_row=1028),
                                dict(k_row=255), dict(v_row=248), dict(k_row=-256), dict(q_out=P, q_row=1536)])
def test_rows(kw):
    assert write(cfg(), desc(), rows(**kw)) == tb.INVALID_ARG
    w = wl.build_workload("rows", wl.ModelShape(8, 2, 128, 16, 1e4), [[3]], np.random.default_rng(0))
    plan = tb.Plan(w, host_only=True)
    assert tb._lib.tessera_extend_write_norm(plan._h, P, P, ctypes.byref(rows(**kw)), None, None, None) == tb.INVALID_ARG       # (host only)


@pytest.mark.parametrize("kw", [dict(q_out=P + 4096), dict(q_out=P + 6128, k=4 * P, v=4 * P), dict(q=3 * P, q_out=P - 6144 + 16), dict(q=3 * P, q_out=P + 1024),
                                dict(q=3 * P, q_out=P + 1536, v_row=512), dict(q_out=P)])
def test_q_out_over_rows_that_are_read(kw):
    """3 rows of 8 + 2 x 2 heads of 128: q 6 144 bytes, k and v 1 536."""
    assert write(cfg(), desc(), rows(**kw)) == tb.INVALID_ARG and "overlaps" in tb.last_error()


def test_rotation():
    assert write(cfg(rope_pairing=2), desc(), rows()) == tb.UNSUPPORTED_SHAPE
    assert write(cfg(rope_theta=0.0), desc(), rows()) == tb.INVALID_ARG


def test_an_empty_batch_is_nothing():
    empty = desc(batch=0, block_table=None, seq_len=None)
    assert attn(cfg(), empty, k=None, v=None, q=None, out=None, ws=None, size=0) == tb.OK
    assert write(cfg(), empty, rows(), k=None, v=None) == tb.OK


def test_null_structures():
    assert tb._lib.tessera_decode_attn(None, None, P, P, P, P, None, P, 0, None) == tb.INVALID_ARG
    assert tb._lib.tessera_decode_write(ctypes.byref(cfg()), ctypes.byref(desc()), P, P, None, None) == tb.INVALID_ARG
    assert tb._lib.tessera_decode_workspace_bytes(None, None) == tb.INVALID_ARG
    n = ctypes.c_int64()
    assert tb._lib.tessera_decode_workspace_bytes(ctypes.byref(cfg(head_dim=32)), ctypes.byref(n)) == tb.UNSUPPORTED_SHAPE
    assert tb._lib.tessera_extend_write_norm(None, P, P, ctypes.byref(rows()), None, None, None) == tb.INVALID_ARG
    for name in ("tessera_kv_retain_kv4", "tessera_kv_compose_from_kv4"):
        assert getattr(tb._lib, name)(None, P, P, P, P, 0, None) == tb.INVALID_ARG
