"""The workspace of a page selection stays at 64 MiB, or at what one group needs, however the batch looks; what is cut for it selects the
same pages."""
import numpy as np
import pytest
import torch

import paper_2602_14516_amd as A
from test_gpu_sparse import normal_bits, random_bounds, table
from oracle import sparse as S
from sparse_util import dev_bits

LIMIT = 64 << 20


def cache(Hq, Hkv, d, P):
    c = A.KVCache(Hq, Hkv, d, P, None, None, 1.0)
    c.num_pages_hint = 1000
    return c


def bytes_of(Hkv, d, P, C, L, budget, group=1, G=1):
    pages = max(-(-(c + n) // P) for c, n in zip(C, L))
    return A.select_pages_workspace_bytes(cache(Hkv * G, Hkv, d, P), C, L, pages, budget, group_tokens=group)


def test_queries_codes_count_and_only_where_they_are_made():
    code = 4 * 128                                                                 # of a group and KV head
    # every page fits the budget: nothing is scored, and a group's codes are all that is asked for
    assert bytes_of(8, 128, 16, [0] * 90, [30000] * 90, 4096) == 8 * code
    # single tokens quantise their queries on the way
    assert bytes_of(8, 128, 16, [16 * 60 - 1] * 90, [1] * 90, 8) == 90 * 8 * 64 * 4 + 8 * code
    assert bytes_of(8, 128, 16, [16 * 60] * 3, [1, 16, 1], 8) == 18 * 8 * (64 * 4 + code)
    for C, L, budget in (([0] * 64, [2000] * 64, 64), ([0] * 16, [4096] * 16, 128), ([500] * 96 + [0], [1] * 96 + [60000], 16),
                         ([0] * 8 + [40000], [16000] * 8 + [1], 1001)):
        assert 0 < bytes_of(8, 128, 16, C, L, budget) <= LIMIT


def test_any_batch_stays_within_the_limit_or_a_group():
    g = np.random.default_rng(5)
    for _ in range(300):
        Hkv, d, P, group = int(g.choice([1, 2, 8, 40])), int(g.choice([64, 128])), int(g.choice([16, 32, 64])), int(g.choice([1, 2, 16]))
        n = int(g.integers(1, 200))
        C, L = (2 ** g.uniform(0, 20, n)).astype(np.int32), (2 ** g.uniform(0, g.uniform(1, 17), n)).astype(np.int32)
        budget = int(2 ** g.uniform(3, 14))
        ws = bytes_of(Hkv, d, P, C, L, budget, group)
        pages = int((-(-(C + L) // P)).max())
        a_group = Hkv * (4 * d + 4 * (-(-pages // 64) * 64))
        assert 256 <= ws <= max(LIMIT, a_group) + 8 * Hkv * d


@pytest.mark.gpu
@pytest.mark.parametrize("group", [1, 2])
def test_a_batch_in_several_launches_selects_what_its_parts_select(group):
    """More groups than one launch has room for, next to rows without scores and to rows of one group."""
    print(f"case: groups of {group}", flush=True)
    g = np.random.default_rng(group)
    P, Hkv, d, n, budget = 16, 8, 128, 400, 12
    C = np.array([0, 100 * P, 5 * P, 90 * P, 0, 64 * P], np.int32)
    L = np.array([20, 1, 12000 * group, 1, 150, 300], np.int32)
    codes, scale = random_bounds(g, n, Hkv, d)
    b = A.PageBounds(torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda())
    bt = table(g, C + L, P, n)
    q = normal_bits(g, int(L.sum()), Hkv, d)
    dq, c = dev_bits(q), cache(Hkv, Hkv, d, P)
    ws = A.select_pages_workspace_bytes(c, C, L, bt.shape[1], budget, group_tokens=group)
    assert 32 << 20 < ws <= LIMIT + 8 * Hkv * d
    room = torch.full((ws + 4096,), 171, dtype=torch.uint8, device="cuda")
    got = A.select_pages(c, C, L, torch.from_numpy(bt).cuda(), b, dq, budget, group_tokens=group, workspace=room[:ws])
    assert (room[ws:] == 171).all()
    parts, at = [], 0
    for r in range(len(C)):
        for i in range(0, int(L[r]), 1000 * group):
            m = min(1000 * group, int(L[r]) - i)
            parts.append(A.select_pages(c, [int(C[r]) + i], [m], torch.from_numpy(bt[r:r + 1]).cuda(), b, dq[at:at + m], budget, group_tokens=group))
            at += m
    assert torch.equal(got, torch.cat(parts))
    few = [0, 1, 3, 4]                                             # and the short rows as defined
    rows = np.concatenate([np.arange(L[:r].sum(), L[:r].sum() + L[r]) for r in few])
    first = np.concatenate([[0], np.cumsum(-(-L // group))])
    lists = np.concatenate([np.arange(first[r], first[r + 1]) for r in few])
    want = S.select_reference(codes, scale, bt[few], C[few], L[few], q[rows], P, budget, 1, 1, group)
    assert np.array_equal(got.cpu().numpy()[lists], want)
