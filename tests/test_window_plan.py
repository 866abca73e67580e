"""Placement with a sliding window, on the CPU: counts, refusals, and the work list against a walk over all keys."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2609_32999_b200 import binding as tb
from paper_2609_32999_b200 import workloads as wl

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_32999_b200", "csrc")


def scattered(T, rows, g=4, seed=0, page=16):
    rng = np.random.default_rng(seed)
    shape = wl.ModelShape(2 * g, 2, 64, page, 10000.0)
    u = wl.unit(T, recompute=sorted(rng.choice(T, rows, replace=False)))
    return wl.build_workload("window", shape, [[u]], rng)


def visible(p, window, n_sink):
    return [k for k in range(p + 1) if window == 0 or k < n_sink or k > p - window]


@pytest.mark.parametrize("window,n_sink", [(0, 0), (1, 0), (1, 1), (7, 300), (128, 4), (129, 128), (500, 129), (2**31 - 1, 0), (5, 2**31 - 1)])
def test_pair_count(window, n_sink):
    w = scattered(700, 45)
    info = tb.Plan(w, host_only=True, window=window, n_sink=n_sink).info
    want = sum(len(visible(int(p), window, n_sink)) for p in w.recompute_pos)
    assert info.qk_pairs == want
    assert info.attn_flops == 4 * 64 * 8 * want
    assert info.attn_mma_pairs >= want * 8


def test_no_window_is_the_plain_plan():
    w = wl.config(5, requests_override=3)
    a, b = tb.Plan(w, host_only=True), tb.Plan(w, host_only=True, window=0, n_sink=7)
    for name, _ in a.info._fields_:
        assert getattr(a.info, name) == getattr(b.info, name)


@pytest.mark.parametrize("window,n_sink", [(-1, 0), (4, -1), (0, -1)])
def test_refusals(window, n_sink):
    with pytest.raises(tb.TesseraError) as e:
        tb.Plan(scattered(64, 8), host_only=True, window=window, n_sink=n_sink)
    assert e.value.status == tb.INVALID_ARG


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    """The library's own host sources linked with a stand-in for the CUDA runtime and a view of the work list."""
    tmp = tmp_path_factory.mktemp("window")
    src, so = tmp / "tiles.cpp", str(tmp / "libwindow.so")
    src.write_text('#include "plan.h"\nextern "C" __attribute__((visibility("default"))) int view_tiles(const tessera_plan *p, int32_t *out, int room) {'
                   'for (int i = 0; i < (int)p->tiles.size() && i < room; ++i) { out[3 * i] = p->tiles[i].q_begin; out[3 * i + 1] = p->tiles[i].n_tok; '
                   'out[3 * i + 2] = p->tiles[i].kv_len; } return (int)p->tiles.size(); }\n')
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-fvisibility=hidden", "-Wl,-Bsymbolic", "-Wl,--no-undefined",
                           "-I", os.path.join(cuda, "include"), "-I", CSRC, "-I", os.path.join(os.path.dirname(HERE), "include"), "-x", "c++",
                           *[os.path.join(CSRC, f) for f in ("api.cu", "plan.cu", "blob_pool.cu")], os.path.join(HERE, "fake_cuda.cpp"),
                           os.path.join(HERE, "plan_view.cpp"), str(src), "-o", so])
    lib = ctypes.CDLL(so)
    lib.view_work.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int]
    lib.view_tiles.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int]
    lib.tessera_plan_create_windowed.argtypes = tb._lib.tessera_plan_create_windowed.argtypes
    lib.tessera_plan_destroy.argtypes = [ctypes.c_void_p]

    def run(w, window, n_sink):
        arr = [np.ascontiguousarray(getattr(w, f), dtype=np.int32) for f in
               ("seq_len", "unit_off", "unit_len", "unit_cached_pos", "unit_cached_stride", "unit_target_pos", "unit_page_off", "unit_pages",
                "recompute_off", "recompute_pos", "free_pages")]
        ptr = [a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)) for a in arr]
        cfg = tb.ModelCfg(w.shape.num_q_heads, w.shape.num_kv_heads, w.shape.head_dim, w.shape.page_size, 1e4, None, 0, 0.0)
        desc = tb.ComposeDesc(len(arr[0]), *ptr, len(arr[10]), None, 0, None, None, None, 0)
        h = ctypes.c_void_p()
        rc = lib.tessera_plan_create_windowed(ctypes.byref(cfg), ctypes.byref(desc), int(w.num_pool_pages), window, n_sink, 1, ctypes.byref(h), None)
        assert rc == 0
        n = lib.view_work(h, 0, None, 0)
        work = np.zeros((n, 12), np.int32)
        lib.view_work(h, 0, work.ctypes.data_as(ctypes.c_void_p), n)
        t = lib.view_tiles(h, None, 0)
        tiles = np.zeros((t, 3), np.int32)
        lib.view_tiles(h, tiles.ctypes.data_as(ctypes.c_void_p), t)
        lib.tessera_plan_destroy(h)
        return work, tiles

    return run


@pytest.mark.parametrize("T,rows,window,n_sink", [(3000, 200, 64, 0), (3000, 200, 700, 130), (5000, 40, 9, 3), (900, 900, 128, 1), (2000, 60, 1, 0),
                                                  (40000, 16, 30000, 4), (129, 1, 1, 0), (1, 1, 1, 1)])
def test_steps_cover_what_rows_see(planner, T, rows, window, n_sink):
    """Every (row, head, visible key) is in exactly one part of one item; between its sinks and its window an item has no key
    that none of its rows sees, apart from the edges of its steps."""
    w = scattered(T, rows, seed=T)
    items, tiles = planner(w, window, n_sink)
    g = w.shape.num_q_heads // w.shape.num_kv_heads
    count = np.zeros((rows, w.shape.num_kv_heads, T), np.int8)
    for it in items:
        if it[0] < 0:
            continue
        gap, sink_steps = it[11], it[10]
        steps = [v if v < sink_steps else v + gap for v in range(it[3], it[4])]
        seen = set()
        for t in (it[0], it[1]):
            if t < 0:
                continue
            q0, n, kv_len = tiles[t]
            assert n * g <= 128
            for j in range(q0, q0 + n):
                p = int(w.recompute_pos[j])
                vis = np.array(visible(p, window, n_sink))
                for s in steps:
                    if s * 128 < kv_len:
                        hit = vis[(vis >= s * 128) & (vis < (s + 1) * 128)]
                        count[j, it[2], hit] += 1
                        seen.update(hit.tolist())
        if steps:              # no key between the item's first and last that none of its rows sees, but for the sinks' side
            rows_of = [int(w.recompute_pos[j]) for t in (it[0], it[1]) if t >= 0 for j in range(tiles[t][0], tiles[t][0] + tiles[t][1])]
            lo = max(0, min(rows_of) - window + 1)
            inside = [k for s in steps for k in range(s * 128, (s + 1) * 128) if lo <= k <= max(rows_of)]
            assert set(inside) <= seen | {k for k in range(T) if k < n_sink}
    for j in range(rows):
        want = np.zeros(T, np.int8)
        want[visible(int(w.recompute_pos[j]), window, n_sink)] = 1
        assert (count[j] == want).all()
