"""The sparse-attention operators on the device against their 64-bit definitions: pages, scales, bounds and page choices bit by bit, rotated
queries and attention within bounds that follow from the formats."""
import numpy as np
import pytest
import torch

import oracle
import paper_2602_14516_amd as A
import workloads as W
from oracle import sparse as S
from sparse_util import BF16_HALF_STEP, Pool, check_attention, dev_bits, host_bits, normal_bits

pytestmark = pytest.mark.gpu

GEOMETRIES = [(8, 2, 128, 16), (8, 2, 64, 16), (4, 4, 64, 32), (8, 1, 128, 32), (6, 3, 128, 64), (32, 8, 64, 64)]


def inv_freq(rotary, base=10000.0):
    return (base ** (-np.arange(0, rotary, 2) / rotary)).astype(np.float32)


def case(name):
    print("case:", name, flush=True)


# ---- rotate and append ---------------------------------------------------------------------------------------------------------


def rope_call(p, C, L, f, q, k, v, **kw):
    return A.rope_kv_append(p.cache, C, L, p.table, A.Rope(torch.from_numpy(f).cuda(), interleaved=kw.pop("interleaved", False), scale=kw.pop("scale", 1.0)),
                            None if q is None else dev_bits(q), dev_bits(k), dev_bits(v), **kw)


def check_queries(got, q, pos, f, interleaved, scale):
    """Each product of 32-bit factors and their difference is off by 2^-24 of its size, the angle's two factors by as much each."""
    ref = S.rope_reference(q, pos, f, interleaved, scale)
    x = np.abs(oracle.bf16_to_f64(q)).max(axis=2, keepdims=True) * scale
    tol = BF16_HALF_STEP * np.abs(ref) + 2 * x * 6 * 2.0 ** -24
    assert (np.abs(W.bf16_bits_to_f64(host_bits(got)) - ref) <= tol * (1 + 2.0 ** -8)).all()


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "8bit"])
@pytest.mark.parametrize("Hq,Hkv,d,P", GEOMETRIES)
def test_rotate_and_append(Hq, Hkv, d, P, fp8):
    # initial rows, rows that end and begin inside pages and at their edges, one token, none
    C, L = np.array([0, 5, P, 2 * P - 1, 40, 3 * P + 1, 0], np.int32), np.array([1, 1, P, 2, 0, 2 * P + 3, P - 1], np.int32)
    for rotary, interleaved, bounds in ((d, False, True), (d, True, False), (d // 2, False, False), (16, True, True)):
        case(f"rope {Hq}/{Hkv}/{d}/{P} 8bit={fp8} rotary={rotary} interleaved={interleaved} bounds={bounds}")
        p = Pool(rotary + interleaved, C, L, Hq, Hkv, d, P, fp8)
        n, f = int(L.sum()), inv_freq(rotary)
        q, k, v = normal_bits(p.g, n, Hq, d), normal_bits(p.g, n, Hkv, d, mult=3.0), normal_bits(p.g, n, Hkv, d, mult=0.5)
        pos = np.concatenate([np.arange(c, c + m) for c, m in zip(C, L)])
        got = rope_call(p, C, L, f, q, k, v, interleaved=interleaved, bounds=p.bounds if bounds else None)
        torch.cuda.synchronize()
        check_queries(got, q, pos, f, interleaved, 1.0)
        p.append(C, L, S.f64_to_bf16_bits(S.rope_reference(k, pos, f, interleaved)), v)
        p.assert_pools_equal()
        if bounds:
            p.set_bounds(C, L)
        p.assert_bounds_equal()
        # the same call once more changes nothing
        again = rope_call(p, C, L, f, q, k, v, interleaved=interleaved, bounds=p.bounds if bounds else None)
        torch.cuda.synchronize()
        assert torch.equal(again, got)
        p.assert_pools_equal()
        p.assert_bounds_equal()


def test_rotation_at_given_positions_and_scale():
    case("rope positions")
    C, L = np.array([3, 30], np.int32), np.array([20, 1], np.int32)
    p = Pool(5, C, L, 4, 2, 128, 16)
    n, f = 21, inv_freq(128, 500000.0)
    q, k, v = normal_bits(p.g, n, 4, 128), normal_bits(p.g, n, 2, 128), normal_bits(p.g, n, 2, 128)
    pos = p.g.integers(-2 ** 31, 2 ** 31, n).astype(np.int32)
    pos[:4] = (0, -1, 1048575, 2 ** 31 - 1)
    got = rope_call(p, C, L, f, q, k, v, scale=1.25, positions=torch.from_numpy(pos).cuda())
    check_queries(got, q, pos, f, False, 1.25)
    p.append(C, L, S.f64_to_bf16_bits(S.rope_reference(k, pos, f, False, 1.25)), v)
    p.assert_pools_equal()


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "8bit"])
def test_rotation_of_views_and_in_place(fp8):
    case("rope views")
    C, L, Hq, Hkv, d, P = np.array([9, 0], np.int32), np.array([4, 17], np.int32), 8, 2, 64, 16
    n, f = 21, inv_freq(64)
    g = np.random.default_rng(3)
    x = normal_bits(g, n, Hq + 2 * Hkv, d)
    a, b, c = (Pool(3, C, L, Hq, Hkv, d, P, fp8) for _ in range(3))
    want = rope_call(a, C, L, f, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])
    qkv, rope = dev_bits(x), A.Rope(torch.from_numpy(f).cuda())
    got = A.rope_kv_append(b.cache, C, L, b.table, rope, qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:])
    q = dev_bits(x[:, :Hq])
    same = A.rope_kv_append(c.cache, C, L, c.table, rope, q, qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], q_out=q)
    assert same is q and torch.equal(got, want) and torch.equal(q, want)
    assert np.array_equal(host_bits(qkv), x)
    for t in (b, c):
        assert torch.equal(t.cache.k_pool.view(torch.uint8), a.cache.k_pool.view(torch.uint8)) and torch.equal(t.cache.v_pool.view(torch.uint8), a.cache.v_pool.view(torch.uint8))
    none = Pool(3, C, L, Hq, Hkv, d, P, fp8)
    assert A.rope_kv_append(none.cache, C, L, none.table, rope, None, qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]) is None
    assert torch.equal(none.cache.k_pool.view(torch.uint8), a.cache.k_pool.view(torch.uint8))


def test_a_page_without_a_place_in_the_pool_is_left_out():
    """Ids outside the pool write nothing, and the queries of their tokens are rotated all the same."""
    case("rope page range")
    C, L = np.array([0, 0], np.int32), np.array([16, 20], np.int32)
    p, full = (Pool(8, C, L, 4, 2, 64, 16) for _ in range(2))
    n, f = 36, inv_freq(64)
    q, k, v = normal_bits(p.g, n, 4, 64), normal_bits(p.g, n, 2, 64), normal_bits(p.g, n, 2, 64)
    bad = p.bt.copy()
    bad[0, 0], bad[1, 1] = p.n, -7
    before = p.k.copy()
    got = A.rope_kv_append(p.cache, C, L, torch.from_numpy(bad).cuda(), A.Rope(torch.from_numpy(f).cuda()), dev_bits(q), dev_bits(k), dev_bits(v), bounds=p.bounds)
    A.page_bounds_update(p.cache, C, L, torch.from_numpy(bad).cuda(), p.bounds)
    assert torch.equal(got, rope_call(full, C, L, f, q, k, v))
    page = int(p.bt[1, 0])
    rest = [i for i in range(p.n) if i != page]
    now = host_bits(p.cache.k_pool)
    assert np.array_equal(now[rest], before[rest]) and np.array_equal(now[page], host_bits(full.cache.k_pool)[page])
    assert (p.bounds.codes.cpu().numpy()[rest] == 99).all()


def test_many_rows_take_several_launches():
    case("rope 300 rows")
    g = np.random.default_rng(11)
    C, L = g.integers(0, 40, 300).astype(np.int32), g.integers(0, 3, 300).astype(np.int32)
    p = Pool(11, C, L, 4, 2, 64, 16, True)
    n, f = int(L.sum()), inv_freq(64)
    q, k, v = normal_bits(p.g, n, 4, 64), normal_bits(p.g, n, 2, 64), normal_bits(p.g, n, 2, 64)
    pos = np.concatenate([np.arange(c, c + m) for c, m in zip(C, L)])
    got = rope_call(p, C, L, f, q, k, v, bounds=p.bounds)
    check_queries(got, q, pos, f, False, 1.0)
    p.append(C, L, S.f64_to_bf16_bits(S.rope_reference(k, pos, f)), v)
    p.set_bounds(C, L)
    p.assert_pools_equal()
    p.assert_bounds_equal()


# ---- bounds --------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "8bit"])
@pytest.mark.parametrize("Hq,Hkv,d,P", GEOMETRIES)
@pytest.mark.parametrize("mult", [1.0, 2.0 ** -44, 2.0 ** 90])
def test_bounds_of_pages(Hq, Hkv, d, P, fp8, mult):
    case(f"bounds {Hq}/{Hkv}/{d}/{P} 8bit={fp8} mult={mult}")
    T = np.array([1, P, P + 1, 7 * P - 3, 0], np.int32)
    p = Pool(21, T, np.zeros_like(T), Hq, Hkv, d, P, fp8, mult=mult)
    for C, L in ((np.zeros_like(T), T), (np.array([0, P - 1, P, 3 * P + 2, 0], np.int32), np.array([1, 0, 1, 1, 0], np.int32))):
        A.page_bounds_update(p.cache, C, L, p.table, p.bounds)
        p.set_bounds(C, L)
        p.assert_bounds_equal()


def test_bounds_of_extreme_keys():
    """Whole pages of one value: zero, the smallest and the largest numbers, the exponent's borders, one sign."""
    case("bounds extremes")
    values = np.array([0.0, -0.0, 2.0 ** -133, -2.0 ** -126, 127.0, -127.5, 2.0 ** 103, -3.3e38, 1.984375, -1.9921875], np.float32)
    P, d = 16, 64
    T = np.full(1, P * len(values), np.int32)
    p = Pool(1, T, [0], 2, 1, d, P, spare=0)
    for j, x in enumerate(values):
        p.k[p.bt[0, j]] = W.f32_to_bf16_bits(np.full((1, P, d), x, np.float32))
        p.k[p.bt[0, j], 0, 3, 5] = W.f32_to_bf16_bits(np.float32([2.0 ** -130]))[0]
    p.upload()
    A.page_bounds_update(p.cache, [0], T, p.table, p.bounds)
    p.set_bounds([0], T)
    p.assert_bounds_equal()


# ---- selection -----------------------------------------------------------------------------------------------------------------


def random_bounds(g, n, Hkv, d, spread=127, scales=2):
    codes = g.integers(-spread, spread + 1, (n, Hkv, 2, d)).astype(np.int8)
    return codes, np.exp2(g.integers(-scales, 1, (n, Hkv))).astype(np.float32)


def check_selection(codes, scale, bt, C, L, q, Hq, P, budget, first, last, g, n=None):
    Hkv, d = codes.shape[1], codes.shape[3]
    cache = A.KVCache(Hq, Hkv, d, P, None, None, 1.0)
    b = A.PageBounds(torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda())
    got = A.select_pages(cache, C, L, torch.from_numpy(bt).cuda(), b, dev_bits(q), budget, first_pages=first, last_pages=last, group_tokens=g)
    want = S.select_reference(codes, scale, bt, C, L, q, P, budget, first, last, g)
    got = got.cpu().numpy()
    assert np.array_equal(got, want), np.argwhere((got != want).any(axis=2))[:5].tolist()


def table(g, T, P, n):
    bt = np.full((len(T), max(1, max(-(-int(t) // P) for t in T))), -1, np.int32)
    for r, t in enumerate(T):
        k = -(-int(t) // P)
        bt[r, :k] = g.integers(0, n, k)
    return bt


@pytest.mark.parametrize("Hq,Hkv,d,P", GEOMETRIES + [(64, 1, 128, 16), (128, 8, 64, 32), (12, 12, 64, 16), (45, 9, 128, 16)])
def test_selection_of_single_tokens(Hq, Hkv, d, P):
    """One token over none to thousands of pages; rows without a token among them."""
    case(f"select {Hq}/{Hkv}/{d}/{P}")
    g = np.random.default_rng(31)
    C = np.array([0, 1, P - 1, P, 9 * P + 3, 300, 130 * P, 129 * P - 1, 1500 * P + 5], np.int32)
    L = np.array([1, 1, 1, 1, 1, 0, 1, 1, 1], np.int32)
    codes, scale = random_bounds(g, 200, Hkv, d)
    q = normal_bits(g, int(L.sum()), Hq, d)
    for budget, first, last in ((3, 1, 2), (8, 0, 1), (20, 2, 4), (129, 1, 1)):
        check_selection(codes, scale, table(g, C + L, P, 200), C, L, q, Hq, P, budget, first, last, 1)


@pytest.mark.parametrize("Hq,Hkv,d,P", GEOMETRIES)
@pytest.mark.parametrize("g_tok", [1, 3, 8, 32])
def test_selection_of_groups(Hq, Hkv, d, P, g_tok):
    if g_tok * (Hq // Hkv) > 128:
        pytest.skip("more rows than a group may have")
    case(f"select groups of {g_tok} {Hq}/{Hkv}/{d}/{P}")
    g = np.random.default_rng(37)
    C, L = np.array([0, 70 * P + 5, 13, 333 * P], np.int32), np.array([5 * P, 70, 1, 2 * g_tok + 1], np.int32)
    codes, scale = random_bounds(g, 150, Hkv, d)
    q = normal_bits(g, int(L.sum()), Hq, d)
    tail = -(-(g_tok - 1) // P)
    for budget, first, last in ((2 + tail, 0, 1), (12 + tail, 1, 2), (70, 2, 3)):
        check_selection(codes, scale, table(g, C + L, P, 150), C, L, q, Hq, P, budget, first, last, g_tok)


@pytest.mark.parametrize("pages", [1023, 1030, 2560, 2570, 4096, 4200, 16384, 16500, 40000])
def test_selection_over_long_rows(pages):
    """Rows on either side of what each form of the choice holds in registers; scores with many equals among them."""
    case(f"select over {pages} pages")
    g = np.random.default_rng(pages)
    P, Hkv, d = 16, 1, 64
    C, L = np.array([pages * P - 1, 5 * P], np.int32), np.array([1, 1], np.int32)
    for spread in (127, 1):
        codes, scale = random_bounds(g, 1000 if spread > 1 else 30, Hkv, d, spread, 2 if spread > 1 else 0)
        q = normal_bits(g, 2, 2, d)
        for budget in (40, 700):
            check_selection(codes, scale, table(g, C + L, P, len(codes)), C, L, q, 2, P, budget, 1, 2, 1)


def test_selection_among_equal_scores_takes_the_lowest_pages():
    case("select ties")
    P, Hkv, d, n = 16, 2, 64, 1000
    g = np.random.default_rng(2)
    codes, scale = np.full((n, Hkv, 2, d), 5, np.int8), np.ones((n, Hkv), np.float32)
    C, L = np.array([999 * P], np.int32), np.array([1], np.int32)
    bt = g.permutation(n).astype(np.int32)[None]
    for q in (normal_bits(g, 1, 4, d), np.zeros((1, 4, d), np.uint16), np.full((1, 4, d), 0x8000, np.uint16)):
        check_selection(codes, scale, bt, C, L, q, 4, P, 33, 1, 2, 1)
    # two values, the border inside the larger one, and inside the smaller one
    codes[bt[0, ::3]] = 9
    q = W.f32_to_bf16_bits(np.abs(g.standard_normal((1, 4, d))).astype(np.float32))
    for budget in (100, 334, 500, 900):
        check_selection(codes, scale, bt, C, L, q, 4, P, budget, 1, 2, 1)


@pytest.mark.parametrize("pages", [70, 1000, 2400, 4000, 9000, 17000])
def test_selection_among_pages_of_one_score(pages):
    """In every form of the choice: a row whose scores are one value, next to rows whose scores are two and many."""
    case(f"select among {pages} pages of one score")
    P, Hkv, d, n = 16, 4, 64, 64
    g = np.random.default_rng(pages)
    codes, scale = random_bounds(g, n, Hkv, d)
    codes[:20], scale[:20] = 5, 1.0
    codes[20], scale[20] = 9, 1.0
    C, L = np.array([pages * P - 1, pages * P - 1, pages * P - 1], np.int32), np.ones(3, np.int32)
    bt = np.stack([g.integers(0, 20, pages), g.integers(0, 21, pages), g.integers(0, n, pages)]).astype(np.int32)
    q = normal_bits(g, 3, 8, d)
    for budget in (9, 60):
        check_selection(codes, scale, bt, C, L, q, 8, P, budget, 1, 2, 1)


@pytest.mark.parametrize("pages", [300, 2400, 20000])
def test_selection_over_pages_whose_bounds_were_never_set(pages):
    """Any bits in a page's scale: what is chosen among those pages is open, but it is a list of the row's pages, and nothing else is written."""
    case(f"select over {pages} pages of any scale")
    P, Hkv, d, n = 16, 2, 64, 500
    g = np.random.default_rng(pages)
    C, L, budget = np.array([pages * P - 1, 40 * P], np.int32), np.ones(2, np.int32), 24
    bt = torch.from_numpy(table(g, C + L, P, n)).cuda()
    q = dev_bits(normal_bits(g, 2, 2, d))
    cache = A.KVCache(2, Hkv, d, P, None, None, 1.0)
    for low, high in ((0, 2 ** 32), (0x7fffff00, 0x80000000), (0x7f800000, 0x80000000), (0xffffff00, 2 ** 32)):
        codes = torch.from_numpy(random_bounds(g, n, Hkv, d)[0]).cuda()
        scale = g.integers(low, high, (n, Hkv), dtype=np.uint32).view(np.float32)
        out = torch.full((4, Hkv, budget), -7, dtype=torch.int32, device="cuda")
        A.select_pages(cache, C, L, bt, A.PageBounds(codes, torch.from_numpy(scale).cuda()), q, budget, out=out[1:3])
        out = out.cpu().numpy()
        assert (out[[0, 3]] == -7).all()
        for r in (0, 1):
            assert (np.diff(out[1 + r], axis=1) > 0).all() and (out[1 + r, :, 0] == 0).all() and (out[1 + r, :, -1] == C[r] // P).all()


@pytest.mark.parametrize("mult", [1e-38, 1e-30, 1.0, 127.0, 1e30, 3e38])
def test_selection_does_not_depend_on_the_size_of_the_queries(mult):
    case(f"select q x {mult}")
    g = np.random.default_rng(6)
    codes, scale = random_bounds(g, 90, 2, 64)
    C, L = np.array([80 * 16], np.int32), np.array([1], np.int32)
    q = W.f32_to_bf16_bits((np.clip(g.standard_normal((1, 4, 64)), -1, 1) * mult).astype(np.float32))
    check_selection(codes, scale, table(g, C + L, 16, 90), C, L, q, 4, 16, 12, 1, 2, 1)


def test_selection_of_more_scores_than_one_launch_holds():
    case("select chunks")
    g = np.random.default_rng(41)
    P, Hkv, d = 16, 2, 64
    C, L = np.concatenate([np.full(130, 40, np.int32), [50000 * P, 20000 * P]]).astype(np.int32), np.concatenate([np.ones(130, np.int32), [200, 30]]).astype(np.int32)
    codes, scale = random_bounds(g, 500, Hkv, d)
    q = normal_bits(g, int(L.sum()), 2, d)
    cache = A.KVCache(2, Hkv, d, P, None, None, 1.0)
    cache.num_pages_hint = 500
    bt = table(g, C + L, P, 500)
    ws = A.select_pages_workspace_bytes(cache, C, L, bt.shape[1], 24, last_pages=2)
    assert ws < 80 << 20                               # 230 tokens over up to 50 000 pages would take 170 MB
    check_selection(codes, scale, bt, C, L, q, 2, P, 24, 1, 2, 1)


# ---- attention over listed pages -----------------------------------------------------------------------------------------------


def check_sparse(p, C, L, sel, q, g_tok, **kw):
    T = C + L
    got = A.sparse_attn(p.cache, C, L, p.table, torch.from_numpy(sel).cuda(), dev_bits(q), group_tokens=g_tok, **kw)
    ref, mag, dots = S.sparse_attn_reference(p.rows("k", T), p.rows("v", T), C, L, sel, q, p.P, p.cache.softmax_scale, g_tok)
    check_attention(W.bf16_bits_to_f64(host_bits(got)), ref, mag, dots)
    return got


def random_lists(g, C, L, P, Hkv, budget, g_tok, holes=0.2):
    """Pages of each group in any order, with holes."""
    groups = S.groups_of(C, L, g_tok)
    sel = np.full((len(groups), Hkv, budget), -1, np.int32)
    for i, (r, t0, m, _) in enumerate(groups):
        pages = (int(C[r]) + t0 + m - 1) // P + 1
        for h in range(Hkv):
            k = min(budget, pages)
            x = g.permutation(pages)[:k]
            x[g.random(k) < holes] = -1
            sel[i, h, g.permutation(budget)[:k]] = x
    return sel


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "8bit"])
@pytest.mark.parametrize("Hq,Hkv,d,P", GEOMETRIES + [(64, 1, 64, 16), (40, 2, 128, 16), (16, 1, 128, 64)])
def test_sparse_attention_of_single_tokens(Hq, Hkv, d, P, fp8):
    case(f"sparse {Hq}/{Hkv}/{d}/{P} 8bit={fp8}")
    C, L = np.array([0, 1, P - 1, P, 3 * P + 5, 17, 40 * P - 1], np.int32), np.array([1, 1, 1, 1, 1, 0, 1], np.int32)
    p = Pool(51, C + L, np.zeros_like(C), Hq, Hkv, d, P, fp8)
    for budget in (1, 2, 7, 40):
        check_sparse(p, C, L, random_lists(p.g, C, L, P, Hkv, budget, 1), normal_bits(p.g, int(L.sum()), Hq, d), 1)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "8bit"])
@pytest.mark.parametrize("Hq,Hkv,d,P", GEOMETRIES)
@pytest.mark.parametrize("g_tok", [3, 8, 32])
def test_sparse_attention_of_groups(Hq, Hkv, d, P, g_tok, fp8):
    if g_tok * (Hq // Hkv) > 128:
        pytest.skip("more rows than a group may have")
    case(f"sparse groups of {g_tok} {Hq}/{Hkv}/{d}/{P} 8bit={fp8}")
    C, L = np.array([0, 9 * P + 5, 13], np.int32), np.array([3 * P + 1, 41, 1], np.int32)
    p = Pool(53, C + L, np.zeros_like(C), Hq, Hkv, d, P, fp8)
    for budget in (1, 5, 14):
        check_sparse(p, C, L, random_lists(p.g, C, L, P, Hkv, budget, g_tok), normal_bits(p.g, int(L.sum()), Hq, d), g_tok)


@pytest.mark.parametrize("g_tok", [1, 8])
def test_lists_of_nothing_duplicates_and_pages_that_are_not_there(g_tok):
    """Empty lists give zeros; entries behind the group's own page and below zero are ignored; a page listed twice counts twice; pages
    that the table places outside the pool are ignored."""
    case(f"sparse odd lists {g_tok}")
    P, Hq, Hkv, d = 16, 8, 2, 64
    C, L = np.array([100, 0, 37], np.int32), np.array([1, 1, 11], np.int32)
    p = Pool(55, C + L, np.zeros_like(C), Hq, Hkv, d, P)
    n, q = len(S.groups_of(C, L, g_tok)), normal_bits(p.g, 13, Hq, d)
    none = check_sparse(p, C, L, np.full((n, Hkv, 5), -1, np.int32), q, g_tok)
    assert not none.float().any()
    sel = random_lists(p.g, C, L, P, Hkv, 6, g_tok, 0.0)
    sel[:, :, 3] = sel[:, :, 0]
    sel[:, 1, 1] = 2 ** 31 - 1
    sel[:, 1, 2] = -2 ** 31
    check_sparse(p, C, L, sel, q, g_tok)
    only = np.full((n, Hkv, 2), -1, np.int32)
    only[:, :, 1] = 0
    want = check_sparse(p, C, L, only, q, g_tok)
    only[:, :, 0] = 1                                        # page 1 of rows 0 and 2 is nowhere now
    table_ = p.table.clone()
    table_[:, 1] = torch.tensor([p.n, -1, -5], device="cuda")
    got = A.sparse_attn(p.cache, C, L, table_, torch.from_numpy(only).cuda(), dev_bits(q), group_tokens=g_tok)
    assert torch.equal(got, want)


@pytest.mark.parametrize("rows,budget", [(1, 600), (2, 129), (40, 9), (70, 12), (130, 5), (260, 3)])
def test_lists_in_pieces_and_whole(rows, budget):
    """Few rows: the list is cut and joined; many: whole; more rows than a launch takes."""
    case(f"sparse {rows} rows x {budget} pages")
    P, Hq, Hkv, d = 16, 8, 2, 128
    g = np.random.default_rng(rows)
    C, L = g.integers(0, min(budget, 60) * P, rows).astype(np.int32), np.ones(rows, np.int32)
    C[0] = min(budget, 600) * P - 1
    p = Pool(57, C + L, np.zeros_like(C), Hq, Hkv, d, P)
    check_sparse(p, C, L, random_lists(p.g, C, L, P, Hkv, budget, 1), normal_bits(p.g, rows, Hq, d), 1)


def test_groups_as_large_workgroups():
    """128 to 256 items go as workgroups of 8 waves, 32 query rows each."""
    case("sparse groups of 8 waves")
    P, Hq, Hkv, d = 16, 8, 2, 128
    C, L = np.array([300, 0], np.int32), np.array([261, 260], np.int32)
    p = Pool(58, C + L, np.zeros_like(C), Hq, Hkv, d, P)
    assert 128 <= A.num_groups(L, 8) * Hkv <= 256
    check_sparse(p, C, L, random_lists(p.g, C, L, P, Hkv, 19, 8), normal_bits(p.g, int(L.sum()), Hq, d), 8)


def test_logits_far_apart_and_a_page_that_outweighs_the_rest():
    case("sparse large logits")
    P, Hq, Hkv, d = 16, 8, 2, 64
    C, L = np.array([400, 900], np.int32), np.array([1, 6], np.int32)
    p = Pool(59, C + L, np.zeros_like(C), Hq, Hkv, d, P, mult=20.0)
    for g_tok in (1, 6):
        check_sparse(p, C, L, random_lists(p.g, C, L, P, Hkv, 30, g_tok), normal_bits(p.g, 7, Hq, d, mult=8.0), g_tok)


def test_pools_past_four_gigabytes():
    """Byte offsets of pages need more than 32 bits."""
    case("sparse 64-bit offsets")
    P, Hq, Hkv, d = 16, 8, 2, 128
    C, L = np.array([5 * P + 3], np.int32), np.array([1], np.int32)
    p = Pool(61, C, L, Hq, Hkv, d, P)
    pages = 700000                                           # of 8 KiB
    big = [torch.zeros((pages, Hkv, P, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    top = np.arange(pages - p.n, pages)
    for t, src in zip(big, (p.cache.k_pool, p.cache.v_pool)):
        t[pages - p.n:] = src
    bounds = A.PageBounds(torch.zeros((pages, Hkv, 2, d), dtype=torch.int8, device="cuda"), torch.ones((pages, Hkv), device="cuda"))
    cache = A.KVCache(Hq, Hkv, d, P, *big, p.cache.softmax_scale)
    bt = torch.from_numpy(top[p.bt].astype(np.int32)).cuda()
    f = inv_freq(128)
    q, k, v = normal_bits(p.g, 1, Hq, d), normal_bits(p.g, 1, Hkv, d), normal_bits(p.g, 1, Hkv, d)
    qr = A.rope_kv_append(cache, C, L, bt, A.Rope(torch.from_numpy(f).cuda()), dev_bits(q), dev_bits(k), dev_bits(v), bounds=bounds)
    A.page_bounds_update(cache, [0], C + L, bt, bounds)
    sel = A.select_pages(cache, C, L, bt, bounds, qr, 4)
    out = A.sparse_attn(cache, C, L, bt, sel, qr)
    qs = rope_call(p, C, L, f, q, k, v, bounds=p.bounds)
    A.page_bounds_update(p.cache, [0], C + L, p.table, p.bounds)
    assert torch.equal(sel, A.select_pages(p.cache, C, L, p.table, p.bounds, qs, 4))
    assert torch.equal(out, A.sparse_attn(p.cache, C, L, p.table, sel, qs))
    assert not big[0][:pages - p.n].any()


def test_a_row_of_the_longest_length():
    """2^30 tokens, nearly all on one page of the pool: the last page, alone or next to a page that is not there, is attended as in a short
    row, and the selection finds the three pages that stand out and the lowest of the others."""
    case("sparse longest row")
    P, d = 16, 64
    C, L = np.array([2 ** 30 - 1], np.int32), np.array([1], np.int32)
    p = Pool(67, [2 * P], [0], 2, 1, d, P)
    q = dev_bits(normal_bits(p.g, 1, 2, d))
    last = 2 ** 30 // P - 1
    bt = torch.full((1, last + 1), int(p.bt[0, 0]), dtype=torch.int32, device="cuda")
    bt[0, last] = int(p.bt[0, 1])
    for g_tok in (1, 20):
        for there in ([last, -1], [-1, last], [last], [-1, -1, last, -1]):
            sel = torch.tensor(there, dtype=torch.int32, device="cuda")[None, None]
            got = A.sparse_attn(p.cache, C, L, bt, sel, q, group_tokens=g_tok)
            short = torch.where(sel < 0, sel, torch.ones_like(sel))
            assert torch.equal(got, A.sparse_attn(p.cache, [2 * P - 1], L, p.table, short, q, group_tokens=g_tok)), there
    codes, scale = torch.ones((p.n, 1, 2, d), dtype=torch.int8, device="cuda"), torch.ones((p.n, 1), device="cuda")
    other = int(np.setdiff1d(np.arange(p.n), p.bt[0])[0])
    codes[other] = 3
    high = [5, 2 ** 25 + 1, last - 1]
    bt[0, high] = other
    chosen = A.select_pages(p.cache, C, L, bt, A.PageBounds(codes, scale), q.abs(), 6)
    assert chosen.flatten().tolist() == [0, 1, 5, 2 ** 25 + 1, last - 1, last]


# ---- the operators together ----------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "8bit"])
def test_a_session_prefills_and_decodes_with_chosen_pages(fp8):
    """Rounds of a prefill in groups and decode steps through one pool, as a worker would run them: pages, bounds and choices follow the
    definitions bit by bit, attention the chosen pages; a budget of all pages gives dense attention."""
    case(f"session 8bit={fp8}")
    P, Hq, Hkv, d, f = 16, 8, 2, 64, inv_freq(64)
    T = np.array([0, 0], np.int32)
    p = Pool(71, T, [700, 500], Hq, Hkv, d, P, fp8)
    for step, L in enumerate(((200, 3), (1, 1), (1, 1), (90, 160), (1, 1), (0, 1))):
        C, L = T.copy(), np.array(L, np.int32)
        n, g_tok = int(L.sum()), 8 if max(L) > 1 else 1
        q, k, v = normal_bits(p.g, n, Hq, d), normal_bits(p.g, n, Hkv, d), normal_bits(p.g, n, Hkv, d)
        pos = np.concatenate([np.arange(c, c + m) for c, m in zip(C, L)])
        qr = rope_call(p, C, L, f, q, k, v, bounds=p.bounds)
        p.append(C, L, S.f64_to_bf16_bits(S.rope_reference(k, pos, f)), v)
        p.set_bounds(C, L)
        p.assert_pools_equal()
        p.assert_bounds_equal()
        qb = host_bits(qr)
        for budget in (6, 64):
            sel = A.select_pages(p.cache, C, L, p.table, p.bounds, qr, budget, last_pages=2, group_tokens=g_tok)
            assert np.array_equal(sel.cpu().numpy(), S.select_reference(p.codes, p.bscale, p.bt, C, L, qb, P, budget, 1, 2, g_tok)), (step, budget)
            out = check_sparse(p, C, L, sel.cpu().numpy(), qb, g_tok)
        dense = A.paged_attn(p.cache, C, L, p.table, qr)
        # both are within 2 * 2^-8 of the sum of p |v| of the same number, |v| < 6 here (rounded probabilities; the output's rounding)
        assert (out.float() - dense.float()).abs().max() <= 2 * 2 * 2.0 ** -8 * 6
        T = T + L


def test_calls_on_a_stream_of_their_own_and_without_outputs_given():
    case("sparse streams")
    P, Hq, Hkv, d = 16, 8, 2, 128
    C, L = np.array([1000, 500], np.int32), np.array([1, 1], np.int32)
    p = Pool(73, C + L, np.zeros_like(C), Hq, Hkv, d, P)
    q = dev_bits(normal_bits(p.g, 2, Hq, d))
    A.page_bounds_update(p.cache, [0, 0], C + L, p.table, p.bounds)
    sel = A.select_pages(p.cache, C, L, p.table, p.bounds, q, 16)
    out = A.sparse_attn(p.cache, C, L, p.table, sel, q)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:                                        # two at once, with workspaces of their own
        a = A.select_pages(p.cache, C, L, p.table, p.bounds, q, 16, stream=s)
        got.append((a, A.sparse_attn(p.cache, C, L, p.table, a, q, stream=s)))
    for s in streams:
        s.synchronize()
    for a, b in got:
        assert torch.equal(a, sel) and torch.equal(b, out)


def test_a_captured_step_replays():
    """A decode step in a graph, replayed over changing queries with eager work between the replays."""
    case("sparse graph")
    P, Hq, Hkv, d, f = 16, 8, 2, 128, inv_freq(128)
    C, L = np.array([3000, 77], np.int32), np.array([1, 1], np.int32)
    p = Pool(75, C, L, Hq, Hkv, d, P, spare=5)
    A.page_bounds_update(p.cache, np.zeros_like(C), C, p.table, p.bounds)
    rope = A.Rope(torch.from_numpy(f).cuda())
    q, k, v = (dev_bits(normal_bits(p.g, 2, h, d)) for h in (Hq, Hkv, Hkv))
    qr, out, sel = torch.empty_like(q), torch.empty_like(q), torch.empty((2, Hkv, 24), dtype=torch.int32, device="cuda")
    ws = [torch.empty(max(256, n), dtype=torch.uint8, device="cuda") for n in (
        A.select_pages_workspace_bytes(p.cache, C, L, p.bt.shape[1], 24), A.sparse_attn_workspace_bytes(p.cache, C, L, p.bt.shape[1], 24))]

    def step():
        A.rope_kv_append(p.cache, C, L, p.table, rope, q, k, v, q_out=qr, bounds=p.bounds)
        A.select_pages(p.cache, C, L, p.table, p.bounds, qr, 24, out=sel, workspace=ws[0])
        A.sparse_attn(p.cache, C, L, p.table, sel, qr, out=out, workspace=ws[1])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        q.copy_(dev_bits(normal_bits(p.g, 2, Hq, d)))
        k.copy_(dev_bits(normal_bits(p.g, 2, Hkv, d)))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (qr, sel, out, p.bounds.codes, p.cache.k_pool.view(torch.int16))]
        for t in (qr, out):
            t.zero_()
        sel.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (qr, sel, out, p.bounds.codes, p.cache.k_pool.view(torch.int16))):
            assert torch.equal(a, b), i


def test_empty_batches():
    case("sparse nothing")
    p = Pool(77, [20], [0], 8, 2, 64, 16)
    z = np.zeros(1, np.int32)
    q, kv = torch.empty((0, 8, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert A.rope_kv_append(p.cache, [20], z, p.table, A.Rope(torch.ones(32, device="cuda")), q, kv, kv).shape == (0, 8, 64)
    A.page_bounds_update(p.cache, [20], z, p.table, p.bounds)
    sel = A.select_pages(p.cache, [20], z, p.table, p.bounds, q, 4)
    assert sel.shape == (0, 2, 4) and A.sparse_attn(p.cache, [20], z, p.table, sel, q).shape == (0, 8, 64)
    none = torch.empty((0, 3), dtype=torch.int32, device="cuda")              # no requests at all
    assert A.rope_kv_append(p.cache, [], [], none, A.Rope(torch.ones(32, device="cuda")), q, kv, kv).shape == (0, 8, 64)
    A.page_bounds_update(p.cache, [], [], none, p.bounds)
    sel = A.select_pages(p.cache, [], [], none, p.bounds, q, 4)
    assert sel.shape == (0, 2, 4) and A.sparse_attn(p.cache, [], [], none, sel, q).shape == (0, 8, 64)
    p.assert_pools_equal()
    p.assert_bounds_equal()


# ---- the two ways through the binding ------------------------------------------------------------------------------------------


def session(fp8=False):
    P, Hq, Hkv, d = 16, 8, 2, 64
    C, L = np.array([60, 33], np.int32), np.array([1, 9], np.int32)
    p = Pool(81, C, L, Hq, Hkv, d, P, fp8)
    A.page_bounds_update(p.cache, np.zeros_like(C), C, p.table, p.bounds)
    x = dev_bits(normal_bits(p.g, 10, Hq + 2 * Hkv, d))
    out = dict(q_out=torch.empty((10, Hq, d), dtype=torch.bfloat16, device="cuda"), sel=torch.empty((A.num_groups(L, 4), Hkv, 4), dtype=torch.int32, device="cuda"),
               out=torch.empty((10, Hq, d), dtype=torch.bfloat16, device="cuda"), ws=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    calls = [lambda C=C: A.rope_kv_append(p.cache, C, L, p.table, A.Rope(torch.from_numpy(inv_freq(64)).cuda()), x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:],
                                          q_out=out["q_out"], bounds=p.bounds),
             lambda C=C: A.page_bounds_update(p.cache, C, L, p.table, p.bounds),
             lambda C=C: A.select_pages(p.cache, C, L, p.table, p.bounds, out["q_out"], 4, group_tokens=4, out=out["sel"], workspace=out["ws"]),
             lambda C=C: A.sparse_attn(p.cache, C, L, p.table, out["sel"], out["q_out"], group_tokens=4, out=out["out"], workspace=out["ws"])]
    return p, out, calls


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "8bit"])
def test_usual_calls_take_the_extension_and_others_the_general_path(fp8, monkeypatch):
    case(f"sparse marshalling 8bit={fp8}")
    import paper_2602_14516_amd.binding as B
    results = []
    for general in (False, True):
        p, out, calls = session(fp8)
        taken = []
        real = B._fast_sparse
        monkeypatch.setattr(B, "_fast_sparse", lambda *a: taken.append(None if general else real(*a)) or taken[-1])
        for f in calls:
            f()
        assert taken == [None if general else 0] * 4
        monkeypatch.setattr(B, "_fast_sparse", real)
        # lengths of another kind: the general path
        for f in calls:
            f(C=[60, 33])
        torch.cuda.synchronize()
        results.append([t.clone() for t in (out["q_out"], out["sel"], out["out"], p.bounds.codes, p.bounds.scale, p.cache.k_pool, p.cache.v_pool)])
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.uint8) if a.is_floating_point() else a, b.view(torch.uint8) if b.is_floating_point() else b)


def test_what_the_library_would_read_as_something_else_is_refused_on_the_device_too():
    case("sparse refusals")
    p, out, calls = session()
    for f in calls:
        f()
    C, L = np.array([60, 33], np.int32), np.array([1, 9], np.int32)
    q, sel = out["q_out"], out["sel"]
    rope, kv = A.Rope(torch.ones(32, device="cuda")), q[:, :2]
    good = dict(q_out=out["out"], bounds=p.bounds)
    with pytest.raises(ValueError, match="q_out"):
        A.rope_kv_append(p.cache, C, L, p.table, rope, q, kv, kv, q_out=out["out"][:9])
    with pytest.raises(ValueError, match="device memory"):
        A.rope_kv_append(p.cache, C, L, p.table, rope, q, kv, kv, positions=torch.zeros(10, dtype=torch.int32), **good)
    with pytest.raises(ValueError, match="next to each other"):
        A.rope_kv_append(p.cache, C, L, p.table, rope, torch.empty((10, 64, 8), dtype=torch.bfloat16, device="cuda").transpose(1, 2), kv, kv, **good)
    with pytest.raises(ValueError, match="k_pool"):
        A.sparse_attn(A.KVCache(8, 2, 64, 16, p.cache.k_pool[:, :, :8], p.cache.v_pool, 0.1), C, L, p.table, sel, q, group_tokens=4, out=out["out"], workspace=out["ws"])
    with pytest.raises(ValueError, match="selected"):
        A.sparse_attn(p.cache, C, L, p.table, sel, q, group_tokens=1, out=out["out"], workspace=out["ws"])
    with pytest.raises(ValueError, match="device memory"):
        A.select_pages(p.cache, C, L, p.table, p.bounds, q, 4, group_tokens=4, out=sel, workspace=torch.empty(1 << 20, dtype=torch.uint8))
    for f, status in ((lambda: A.rope_kv_append(p.cache, C, L, p.table, A.Rope(torch.ones(20, device="cuda")), q, kv, kv, **good), -2),
                      (lambda: A.rope_kv_append(p.cache, C, L, p.table, A.Rope(torch.ones(32, device="cuda"), scale=-1.0), q, kv, kv, **good), -1),
                      (lambda: A.select_pages(p.cache, C, L, p.table, p.bounds, q, 4, group_tokens=4, out=sel, workspace=out["ws"][:256]), -3),
                      (lambda: A.select_pages(p.cache, C, L, p.table, p.bounds, q, 4, group_tokens=4, out=sel, workspace=out["ws"][1:]), -3),
                      (lambda: A.select_pages(p.cache, C, L, p.table, p.bounds, q, 4, group_tokens=4, last_pages=4, out=sel, workspace=out["ws"]), -1),
                      (lambda: A.sparse_attn(p.cache, C, L, p.table[:, :2].contiguous(), sel, q, group_tokens=4, out=out["out"], workspace=out["ws"]), -1)):
        with pytest.raises(A.AmpdError) as e:
            f()
        assert e.value.status == status


def test_results_and_workspaces_a_raw_stream_or_a_view_cannot_have():
    """A raw handle of another stream names no memory to allocate results from; a workspace's bytes lie next to each other."""
    case("sparse raw streams and workspace views")
    p, out, calls = session()
    for f in calls:
        f()
    C, L = np.array([60, 33], np.int32), np.array([1, 9], np.int32)
    q, sel, raw = out["q_out"], out["sel"], torch.cuda.Stream().cuda_stream
    rope, kv = A.Rope(torch.ones(32, device="cuda")), q[:, :2]
    with pytest.raises(ValueError, match="pass q_out="):
        A.rope_kv_append(p.cache, C, L, p.table, rope, q, kv, kv, stream=raw)
    with pytest.raises(ValueError, match="pass out="):
        A.select_pages(p.cache, C, L, p.table, p.bounds, q, 4, group_tokens=4, workspace=out["ws"], stream=raw)
    with pytest.raises(ValueError, match="pass workspace="):
        A.sparse_attn(p.cache, C, L, p.table, sel, q, group_tokens=4, out=out["out"], stream=raw)
    view = torch.empty(1, dtype=torch.uint8, device="cuda").expand(1 << 20)
    for stream in (None, torch.cuda.current_stream()):
        with pytest.raises(ValueError, match="workspace"):
            A.select_pages(p.cache, C, L, p.table, p.bounds, q, 4, group_tokens=4, out=sel, workspace=view, stream=stream)
        with pytest.raises(ValueError, match="workspace"):
            A.sparse_attn(p.cache, C, L, p.table, sel, q, group_tokens=4, out=out["out"], workspace=view, stream=stream)
