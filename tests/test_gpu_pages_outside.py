"""Page choices where the block table names pages outside the pool: they come behind all others, whatever the first page's bounds are."""
import numpy as np
import pytest

from test_gpu_sparse import check_selection, random_bounds, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group_tokens", [1, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("pages", [60, 700, 3000])
def test_pages_outside_the_pool_are_chosen_last(pages, d, group_tokens):
    print(f"case: {pages} pages, d {d}, groups of {group_tokens}", flush=True)
    g = np.random.default_rng(pages)
    P, Hq, Hkv, n = 16, 4, 2, 200
    codes, scale = random_bounds(g, n, Hkv, d)
    codes[0, :, 0], codes[0, :, 1], scale[0] = 127, -127, 4.0                   # no page scores above the first
    C, L = np.full(4, pages * P - 1, np.int32), np.full(4, group_tokens + 1, np.int32)
    bt = table(g, C + L, P, n)
    q = np.uint16(0x3F80) + g.integers(0, 2 ** 7, (int(L.sum()), Hq, d)).astype(np.uint16)
    for r, share in enumerate((0.1, 0.5, 0.98, 1.0)):
        out = g.random(bt.shape[1]) < share
        bt[r, out] = g.choice(np.array([-1, -2 ** 31, n, 2 ** 31 - 1], np.int32), int(out.sum()))
    for budget in (8, 50):
        check_selection(codes, scale, bt, C, L, q, Hq, P, budget, 1, 2, group_tokens)
