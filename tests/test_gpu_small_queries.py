"""Page choices of queries whose largest magnitude has no leading one (below 2^-126), or lies just above: rounded to whole numbers by the
definition's exponent."""
import numpy as np
import pytest

from test_gpu_sparse import check_selection, random_bounds, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group_tokens", [1, 3])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("largest", [0x01, 0x02, 0x3F, 0x40, 0x7E, 0x7F, 0x80, 0xFE, 0xFF, 0x100])
def test_queries_next_to_zero(largest, d, group_tokens):
    print(f"case: largest query bits {largest:#x}, d {d}, groups of {group_tokens}", flush=True)
    g = np.random.default_rng(largest)
    P, Hq, Hkv, rows = 16, 4, 2, 48
    codes, scale = random_bounds(g, 300, Hkv, d)
    C, L = np.full(rows, 90 * P, np.int32), np.full(rows, 2 * group_tokens - 1, np.int32)
    n = int(L.sum())
    q = g.integers(0, largest + 1, (n, Hq, d)).astype(np.uint16)
    q[:, ::Hq // Hkv, 5] = largest                               # the largest of every group and KV head
    q |= (g.integers(0, 2, q.shape) << 15).astype(np.uint16)
    check_selection(codes, scale, table(g, C + L, P, 300), C, L, q, Hq, P, 24, 1, 2, group_tokens)
