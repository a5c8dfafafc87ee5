"""How attention over listed pages cuts lists and sizes its workgroups: when there are few lists, only long ones are cut, into as many pieces as fill the
chip, and the result is the same on either side of every border."""
import numpy as np
import pytest
import torch

import paper_2602_14516_amd as A
from oracle import sparse as S
from sparse_util import Pool, check_attention, dev_bits, host_bits, normal_bits
import workloads as W


def workspace(items, keys, d=128, rows=4):
    """`items` lists of `keys` keys: new tokens of a request, one KV head."""
    c = A.KVCache(rows, 1, d, 64, None, None, 0.1)
    c.num_pages_hint = 10 ** 6
    return A.sparse_attn_workspace_bytes(c, [1 << 20], [items], (1 << 14) + 10, keys // 64)


def pieces(items, keys, d=128, rows=4):
    n = workspace(items, keys, d, rows) / (items * (16 if rows <= 16 else 32) * (d + 2) * 4)
    return int(n) if n >= 1 else 1


def test_short_lists_are_never_cut():
    assert all(workspace(n, 512, d) == 256 for n in (1, 16, 33, 96, 120, 128, 200, 257, 300, 500) for d in (64, 128))


def test_long_lists_are_cut_while_whole_ones_would_leave_the_chip_idle():
    # 128 lists on 256 CUs are no longer left whole where 120 are cut
    assert [pieces(n, 8192) for n in (8, 32, 33, 64, 120, 128, 129, 256)] == [16, 16, 7, 4, 2, 2, 1, 1]
    assert [pieces(n, 8192) for n in (257, 341, 342, 512, 513)] == [3, 3, 1, 1, 1]
    assert pieces(300, 2048) == 3 and pieces(300, 2048, rows=32) == 1 and pieces(300, 4096, rows=32) == 3 and pieces(300, 2048, d=64) == 1
    assert pieces(1, 1 << 20) == 512 and pieces(64, 1 << 20) == 4


@pytest.mark.gpu
@pytest.mark.parametrize("d,fp8", [(128, False), (64, True)], ids=["bf16", "8bit"])
@pytest.mark.parametrize("n", [8, 9, 32, 33, 64, 65, 85, 86])
def test_attention_on_either_side_of_the_borders(n, d, fp8):
    print(f"case: {n} rows of 4 KV heads, d {d}, 8 bits: {fp8}", flush=True)
    P, G, Hkv = 64, 4, 4
    for keys in (512, 2048, 4096):
        budget = keys // P
        C = np.full(n, keys + P - 2, np.int32)
        few = min(n, max(1, 20000 // int(C[0])))                                   # rows share the pages of a few
        p = Pool(n + keys, C[:few] + 1, 0 * C[:few], G * Hkv, Hkv, d, P, fp8)
        rows = np.arange(n) % few
        q = normal_bits(p.g, n, G * Hkv, d)
        sel = np.sort(np.stack([[p.g.permutation(budget + 1)[:budget] for _ in range(Hkv)] for _ in range(n)])).astype(np.int32)
        got = A.sparse_attn(p.cache, C, np.ones(n, np.int32), p.table[torch.from_numpy(rows).cuda()].contiguous(), torch.from_numpy(sel).cuda(), dev_bits(q))
        some = np.unique(np.concatenate([[0, n - 1], p.g.integers(0, n, 10)]))
        k, v = p.rows("k", C[:few] + 1), p.rows("v", C[:few] + 1)
        ref, mag, dots = S.sparse_attn_reference([k[r] for r in rows[some]], [v[r] for r in rows[some]], C[some], np.ones(len(some), np.int32), sel[some], q[some], P,
                                                 p.cache.softmax_scale, 1)
        check_attention(W.bf16_bits_to_f64(host_bits(got))[some], ref, mag, dots)
        # every other row as in a call of its own rows
        for r in np.setdiff1d(np.arange(n), some)[:4]:
            alone = A.sparse_attn(p.cache, C[:1], [1], p.table[rows[r]:rows[r] + 1].contiguous(), torch.from_numpy(sel[r:r + 1]).cuda(), dev_bits(q[r:r + 1]))
            assert (alone[0].float() - got[int(r)].float()).abs().max() <= 2.0 ** -7 * got[int(r)].float().abs().max()
