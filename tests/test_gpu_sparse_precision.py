"""Attention over listed pages keeps the probabilities' bits: over few keys whose values cancel, outputs are off by the rounding of the output
and what 32-bit arithmetic loses, not by a rounding of the probabilities to 16 bits."""
import numpy as np
import pytest
import torch

import paper_2602_14516_amd as A
import workloads as W
from oracle import sparse as S
from sparse_util import BF16_HALF_STEP, Pool, dev_bits, host_bits, normal_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "8bit"])
@pytest.mark.parametrize("rows", [8, 30, 150], ids=lambda r: f"{r}rows")
@pytest.mark.parametrize("Hq,Hkv,d,P,g_tok", [(8, 2, 128, 16, 1), (8, 2, 64, 32, 1), (8, 2, 128, 16, 8), (4, 4, 64, 64, 20), (32, 4, 128, 16, 1)])
def test_probabilities_are_not_rounded_to_16_bits(Hq, Hkv, d, P, g_tok, rows, fp8):
    print(f"case: {Hq}/{Hkv}/{d}/{P}, groups of {g_tok}, {rows} rows, 8 bits: {fp8}", flush=True)
    C, L = np.full(rows, 3 * P + 5, np.int32), np.full(rows, g_tok, np.int32)
    p = Pool(rows + d, C + L, 0 * C, Hq, Hkv, d, P, fp8)
    q = normal_bits(p.g, int(L.sum()), Hq, d)
    sel = np.tile(np.array([1, 3, -1, -1], np.int32), (rows, Hkv, 1))            # 2 pages of P keys, the second in part
    got = A.sparse_attn(p.cache, C, L, p.table, torch.from_numpy(sel).cuda(), dev_bits(q), group_tokens=g_tok)
    ref, mag, dots = S.sparse_attn_reference(p.rows("k", C + L), p.rows("v", C + L), C, L, sel, q, P, p.cache.softmax_scale, g_tok)
    # each relative to the probability: its logit (128 products in 32 bits, the reference it is taken against as many), the argument of exp2 and its
    # result, two parts of 8 bits (2^-15), and sums of at most 2 P terms in 32 bits, twice
    p_off = 2 * 128 * 2.0 ** -24 * dots + 3 * 2.0 ** -23 * dots + 2.0 ** -22 + 2.0 ** -15 + 2 * 2 * P * 2.0 ** -24
    bound = mag * p_off[..., None] * (1 + 2.0 ** -8) + BF16_HALF_STEP * np.abs(ref) + 1e-30
    worst = float((np.abs(W.bf16_bits_to_f64(host_bits(got)) - ref) / bound).max())
    assert worst <= 1.0, f"{worst:.2f} of the bound"
