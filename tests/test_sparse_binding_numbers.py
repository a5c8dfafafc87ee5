"""Numbers that do not fit the library's 32 bits, and groups of no tokens, are refused in the binding: cut to 32 bits they would be others."""
import pytest
import torch

import paper_2602_14516_amd as A


def calls(budget=4, first_pages=1, last_pages=1, group_tokens=1):
    P, Hq, Hkv, d, n = 16, 8, 2, 64, 4
    bf = torch.bfloat16
    pool = torch.zeros((9, Hkv, P, d), dtype=bf)
    cache = A.KVCache(Hq, Hkv, d, P, pool, pool, 0.1)
    batch = ([20], [n], torch.zeros((1, 3), dtype=torch.int32))
    b = A.PageBounds(torch.zeros((9, Hkv, 2, d), dtype=torch.int8), torch.ones((9, Hkv)))
    q, ws = torch.zeros((n, Hq, d), dtype=bf), torch.zeros(8192, dtype=torch.uint8)
    choice = dict(first_pages=first_pages, last_pages=last_pages, group_tokens=group_tokens)
    return {"select": lambda: A.select_pages(cache, *batch, b, q, budget, out=torch.zeros((n, Hkv, 4), dtype=torch.int32), workspace=ws, **choice),
            "select_bytes": lambda: A.select_pages_workspace_bytes(cache, [20], [n], 3, budget, **choice),
            "sparse": lambda: A.sparse_attn(cache, *batch, torch.zeros((n, Hkv, 4), dtype=torch.int32), q, group_tokens=group_tokens, out=torch.zeros((n, Hq, d), dtype=bf),
                                            workspace=ws),
            "sparse_bytes": lambda: A.sparse_attn_workspace_bytes(cache, [20], [n], 3, budget, group_tokens=group_tokens),
            "groups": lambda: A.num_groups([n], group_tokens)}


@pytest.mark.parametrize("name", ["budget", "first_pages", "last_pages", "group_tokens"])
@pytest.mark.parametrize("by", [2 ** 32, -2 ** 32, 2 ** 63])
def test_numbers_past_32_bits(name, by):
    value = (4 if name == "budget" else 1) + by                    # (its low 32 bits are a valid call's)
    ops = ["select", "select_bytes"] + {"budget": ["sparse_bytes"], "group_tokens": ["sparse", "sparse_bytes", "groups"]}.get(name, [])
    for op in ops:
        with pytest.raises(ValueError, match="32 bits"):
            calls(**{name: value})[op]()


@pytest.mark.parametrize("group_tokens", [0, -1])
def test_groups_of_no_tokens(group_tokens):
    for op in ("select", "sparse", "groups"):
        with pytest.raises(ValueError, match="group_tokens"):
            calls(group_tokens=group_tokens)[op]()
