"""Sparse attention without a GPU: what the calls refuse, before anything is enqueued, and the workspaces they ask for."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2602_14516_amd as A
import paper_2602_14516_amd.binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WORKSPACE, RANGE = 0, -1, -2, -3, -4


def shape_cache(Hq=8, Hkv=2, d=128, P=16, pages=1000):
    c = A.KVCache(Hq, Hkv, d, P, None, None, 0.1)
    c.num_pages_hint = pages
    return c


def test_selection_workspaces():
    ws = A.select_pages_workspace_bytes
    # keys of 64 pages for one group of two heads, and the groups' codes of 4 d bytes
    assert ws(shape_cache(), [16 * 50], [1], 51, 4) == 2 * 64 * 4 + 2 * 4 * 128
    # nothing to choose: all pages fit the budget
    assert ws(shape_cache(), [16 * 50], [1], 51, 51) == 2 * 4 * 128
    assert ws(shape_cache(), [16 * 50], [0], 51, 4) == 256
    # bounded, however many the rows
    assert ws(shape_cache(Hkv=8), [16 * 60000] * 300, [64] * 300, 60004, 128) <= (64 << 20) + 300 * 64 * 8 * 512
    for bad in (dict(budget=0), dict(budget=2, last_pages=2), dict(budget=4, first_pages=-1), dict(budget=4, last_pages=0), dict(budget=4, group_tokens=0),
                dict(budget=3, group_tokens=18), dict(budget=9, group_tokens=33), dict(budget=1 << 26)):
        kw = dict(first_pages=1, last_pages=1, group_tokens=1, **bad) if not set(bad) & {"first_pages", "last_pages", "group_tokens"} else bad
        assert ws(shape_cache(), [800], [1], 51, **kw) == 0, bad
    assert ws(shape_cache(d=96), [800], [1], 51, 4) == 0 and ws(shape_cache(), [800], [1], 50, 4) == 0


def test_attention_workspaces():
    ws = A.sparse_attn_workspace_bytes
    assert ws(shape_cache(), [800] * 300, [1] * 300, 51, 4) == 256                 # enough items: nothing is cut
    one = ws(shape_cache(), [80000], [1], 5001, 128)
    pieces = one // (2 * 16 * 130 * 4)
    assert one == pieces * 2 * 16 * 130 * 4 and 4 <= pieces <= 16                  # 2 048 keys in pieces of 128 at least
    assert ws(shape_cache(), [800], [1], 51, 0) == 0 and ws(shape_cache(), [800], [1], 51, 4, group_tokens=0) == 0
    assert ws(shape_cache(), [800], [1], 51, 4, group_tokens=33) == 0 and ws(shape_cache(), [800], [1], 51, 4, group_tokens=32) > 0
    assert A.num_groups([0, 1, 8, 9], 8) == 4 and A.num_groups([5, 0, 2]) == 7


def structs():
    c = shape_cache().c_struct()
    c.k_pool = c.v_pool = 256
    b, keep = B._batch([20], [4], None, None, max_pages=2)
    b.d_block_table = 256
    return c, b, keep


@pytest.mark.skipif(os.environ.get("AMPD_HOST_ONLY") == "1", reason="entry points of the GPU half")
def test_rotation_refusals_come_before_anything_is_enqueued():
    row = 8 * 128

    def call(change):
        c, b, keep = structs()
        ro = B._Rope(128, 0, 256, None, 1.0, 0)
        rows = B._Rows(256, 256, 256, row, 256, 256)
        bounds = B._Bounds(256, 256)
        x = dict(c=c, b=b, ro=ro, rows=rows, bounds=bounds, out=512, rop=None)
        change(x)
        return B._packed.ampd_rope_kv_append(ctypes.byref(x["c"]), ctypes.byref(x["b"]), None if x["rop"] else ctypes.byref(x["ro"]), ctypes.byref(x["rows"]),
                                             x["out"], ctypes.byref(x["bounds"]), None)

    def put(which, field, value):
        return lambda x: setattr(x[which], field, value)

    for change, status in ((put("ro", "rotary_dim", 8), UNSUPPORTED), (put("ro", "rotary_dim", 144), UNSUPPORTED), (put("ro", "rotary_dim", 40), UNSUPPORTED),
                           (put("ro", "interleaved", 2), INVALID), (put("ro", "scale", 0.0), INVALID), (put("ro", "scale", float("nan")), INVALID),
                           (put("ro", "reserved", 1), INVALID), (put("ro", "inv_freq", None), INVALID), (put("rows", "k", None), INVALID),
                           (put("rows", "v", 264), INVALID), (put("rows", "q_stride", row - 8), INVALID), (put("rows", "k_stride", 260), INVALID),
                           (put("rows", "v_stride", -256), INVALID), (put("bounds", "codes", 264), INVALID), (put("bounds", "scale", None), INVALID),
                           (put("c", "v_pool", None), INVALID), (put("c", "head_dim", 96), UNSUPPORTED), (lambda x: x.update(out=None), INVALID),
                           (lambda x: x.update(out=520), INVALID), (lambda x: x.update(rop=1), INVALID),
                           (lambda x: (setattr(x["rows"], "q_stride", 2 * row), x.update(out=256)), INVALID)):
        assert call(change) == status
    c, b, keep = structs()
    mirror = np.array([[0, 1000]], np.int32)
    b.h_block_table = mirror.ctypes.data
    assert B._packed.ampd_page_bounds_update(ctypes.byref(c), ctypes.byref(b), ctypes.byref(B._Bounds(256, 256)), None) == RANGE
    assert B._packed.ampd_page_bounds_update(ctypes.byref(c), ctypes.byref(structs()[1]), None, None) == INVALID


@pytest.mark.skipif(os.environ.get("AMPD_HOST_ONLY") == "1", reason="entry points of the GPU half")
def test_selection_and_attention_refusals_come_before_anything_is_enqueued():
    def select(q=256, out=256, ws=256, nbytes=1 << 20, table=256, **kw):
        c, b, keep = structs()
        c.k_pool = c.v_pool = None                          # a selection reads no pool
        b.d_block_table = table
        s = B._Selection(kw.get("budget", 4), kw.get("first", 1), kw.get("last", 1), kw.get("group", 1), (ctypes.c_int32 * 4)(*([kw.get("reserved", 0)] * 4)))
        return B._packed.ampd_select_pages(ctypes.byref(c), ctypes.byref(b), ctypes.byref(B._Bounds(256, 256)), ctypes.byref(s), q, out, ws, nbytes, None)

    for kw, status in ((dict(q=None), INVALID), (dict(q=264), INVALID), (dict(out=None), INVALID), (dict(out=258), INVALID), (dict(ws=None), WORKSPACE),
                       (dict(ws=128), WORKSPACE), (dict(nbytes=255), WORKSPACE), (dict(table=None), INVALID), (dict(budget=1), INVALID),
                       (dict(reserved=1), INVALID), (dict(group=33, budget=9), UNSUPPORTED)):
        assert select(**kw) == status, kw

    def sparse(q=256, out=256, sel=256, ws=256, nbytes=1 << 20, budget=4, group=1, pool=256):
        c, b, keep = structs()
        c.k_pool = pool
        return B._packed.ampd_sparse_attn(ctypes.byref(c), ctypes.byref(b), sel, budget, group, q, out, ws, nbytes, None)

    for kw, status in ((dict(q=None), INVALID), (dict(q=264), INVALID), (dict(out=None), INVALID), (dict(sel=None), INVALID), (dict(sel=258), INVALID),
                       (dict(ws=None), WORKSPACE), (dict(ws=64), WORKSPACE), (dict(nbytes=8), WORKSPACE), (dict(budget=0), INVALID), (dict(group=0), INVALID),
                       (dict(group=33), UNSUPPORTED), (dict(budget=1 << 27), UNSUPPORTED), (dict(pool=None), INVALID)):
        assert sparse(**kw) == status, kw


def test_tensors_of_another_kind_are_refused():
    """Types, shapes, strides and places that the library would read as something else."""
    P, Hq, Hkv, d, n = 16, 8, 2, 64, 4
    bf = torch.bfloat16
    pools = [torch.zeros((9, Hkv, P, d), dtype=bf) for _ in range(2)]
    good = dict(table=torch.zeros((1, 3), dtype=torch.int32), q=torch.zeros((n, Hq, d), dtype=bf), k=torch.zeros((n, Hkv, d), dtype=bf), f=torch.ones(32),
                codes=torch.zeros((9, Hkv, 2, d), dtype=torch.int8), scale=torch.ones((9, Hkv)), sel=torch.zeros((n, Hkv, 4), dtype=torch.int32), k_pool=pools[0],
                positions=None, q_out=None, out=None, lengths=([20], [n]))

    def calls(**kw):
        x = dict(good, **kw)
        cache = A.KVCache(Hq, Hkv, d, P, x["k_pool"], pools[1], 0.1)
        b = A.PageBounds(x["codes"], x["scale"])
        return {"rope": lambda: A.rope_kv_append(cache, *x["lengths"], x["table"], A.Rope(x["f"]), x["q"], x["k"], x["k"], q_out=x["q_out"], positions=x["positions"], bounds=b),
                "bounds": lambda: A.page_bounds_update(cache, *x["lengths"], x["table"], b),
                "select": lambda: A.select_pages(cache, *x["lengths"], x["table"], b, x["q"], 4, out=x["out"], workspace=torch.zeros(4096, dtype=torch.uint8)),
                "sparse": lambda: A.sparse_attn(cache, *x["lengths"], x["table"], x["sel"], x["q"], out=x["out"], workspace=torch.zeros(4096, dtype=torch.uint8))}

    def refused(ops, match, **kw):
        for op in ops:
            kw2 = dict(kw)
            if "out" not in kw2 and op in ("select", "sparse"):
                kw2["out"] = torch.zeros((n, Hkv, 4), dtype=torch.int32) if op == "select" else torch.zeros((n, Hq, d), dtype=bf)
            if "q_out" not in kw2 and op == "rope":
                kw2["q_out"] = torch.zeros((n, Hq, d), dtype=bf)
            with pytest.raises(ValueError, match=match):
                calls(**kw2)[op]()

    every = ("rope", "bounds", "select", "sparse")
    refused(every, "device memory")                                                # all on the CPU
    refused(every, "block_table", table=torch.zeros((1, 3), dtype=torch.int64))
    refused(every, "block_table", table=torch.zeros((2, 3), dtype=torch.int32))
    refused(every, "block_table", table=torch.zeros((1, 6), dtype=torch.int32)[:, ::2])
    refused(every, "two vectors", lengths=([20, 1], [n]))
    refused(("rope", "bounds", "sparse"), "k_pool", k_pool=pools[0].float())
    refused(("rope", "bounds", "sparse"), "k_pool", k_pool=pools[0].transpose(1, 2))
    refused(("rope", "bounds", "select"), "bounds", codes=torch.zeros((9, Hkv, 2, d), dtype=torch.uint8))
    refused(("rope", "bounds", "select"), "bounds", codes=torch.zeros((8, Hkv, 2, d), dtype=torch.int8))
    refused(("rope", "bounds", "select"), "bounds", scale=torch.ones((9, Hkv), dtype=torch.float64))
    refused(("rope", "select", "sparse"), "q", q=torch.zeros((n, Hq, d)))
    refused(("rope", "select", "sparse"), "q", q=torch.zeros((n + 1, Hq, d), dtype=bf))
    refused(("select", "sparse"), "q", q=torch.zeros((n, 2 * Hq, d), dtype=bf)[:, ::2])
    refused(("rope",), "next to each other", q=torch.zeros((n, 2 * Hq, d), dtype=bf)[:, ::2])
    refused(("rope",), "k_new", k=torch.zeros((n, Hkv, 2 * d), dtype=bf))
    refused(("rope",), "inv_freq", f=torch.ones((2, 16)))
    refused(("rope",), "positions", positions=torch.zeros(n, dtype=torch.int64))
    refused(("rope",), "q_out", q_out=torch.zeros((n, Hq, d)))
    refused(("sparse",), "selected", sel=torch.zeros((n, Hkv, 4), dtype=torch.int64))
    refused(("sparse",), "selected", sel=torch.zeros((n, Hkv + 1, 4), dtype=torch.int32))
    refused(("select",), "out", out=torch.zeros((n, Hkv, 5), dtype=torch.int32))
    refused(("sparse",), "out", out=torch.zeros((n, Hq, d)))


@pytest.mark.skipif(os.environ.get("AMPD_HOST_ONLY") == "1", reason="this is the test that sets it")
@pytest.mark.timeout(600)
def test_host_half_runs_clean_under_sanitizers():
    from test_host_sanitizers import _preload_in_use
    from paper_2602_14516_amd.build import build_host_sanitized
    host_lib, _, runtime = build_host_sanitized(address=not _preload_in_use())
    env = dict(os.environ, AMPD_LIB_PATH=host_lib, AMPD_HOST_ONLY="1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1",
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0")
    if runtime:
        env["LD_PRELOAD"] = runtime
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", os.path.abspath(__file__)]
    res = subprocess.run(cmd, cwd=ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=580)
    assert res.returncode == 0 and "runtime error:" not in res.stdout and " passed" in res.stdout, res.stdout[-4000:]
