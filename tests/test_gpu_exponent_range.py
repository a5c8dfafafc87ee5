"""8-bit pages whose power-of-two scale rises over the whole range of exponents, -40 to 119: pools and scales of every way into the cache
against the definition, byte by byte."""
import numpy as np
import pytest
import torch

import paper_2602_14516_amd as A
import workloads as W
from sparse_util import Pool, dev_bits, normal_bits

pytestmark = pytest.mark.gpu

# exponents that the new tokens ask for; from -40 they are 60 and 126 to 159 above the old one
RISES = (20, 86, 87, 88, 89, 100, 118, 119)


def rising(seed, Hkv, d, P, L, fp8=True):
    """Rows whose last page holds 1 to 5 tokens, the first rows' of zeros, the others' of the smallest numbers that their exponent -40 keeps;
    L new tokens each, of the exponents in turn: largest magnitudes 448 * 2^e, exactly in the first of them."""
    n = 2 * len(RISES)
    C = np.array([P + 1 + r % 5 for r in range(n)], np.int32)
    p = Pool(seed, np.zeros(n, np.int32), C + L, 8, Hkv, d, P, fp8)
    old = [normal_bits(p.g, 2, int(c), Hkv, d, mult=2.0 ** -34 if r >= len(RISES) else 0.0) for r, c in enumerate(C)]
    k, v = (np.concatenate([x[i] for x in old]) for i in range(2))
    p.append(np.zeros_like(C), C, k, v)
    p.upload()
    inc = np.full(n, L, np.int32)
    new = p.g.uniform(-1.0, 1.0, (2, n, L, Hkv, d))
    new[:, :, 0, :, 3] = 1.0
    new *= 448.0 * 2.0 ** np.array(RISES * 2, np.float64)[None, :, None, None, None]
    bits = W.f32_to_bf16_bits(new.astype(np.float32)).reshape(2, n * L, Hkv, d)
    return p, C, inc, bits[0], bits[1]


@pytest.mark.parametrize("L", [1, 3])
@pytest.mark.parametrize("Hkv,d,P", [(2, 128, 16), (4, 64, 32), (2, 128, 64)])
@pytest.mark.parametrize("way", ["append", "attention", "rotate", "rotate_with_bounds"])
def test_old_codes_follow_an_exponent_that_rises_by_any_amount(way, Hkv, d, P, L):
    print(f"case: {way} {Hkv}/{d}/{P}, {L} tokens", flush=True)
    p, C, inc, k, v = rising(3, Hkv, d, P, L)
    q = normal_bits(p.g, int(inc.sum()), 8, d)
    if way == "append":
        A.kv_append(p.cache, C, inc, p.table, dev_bits(k), dev_bits(v))
    elif way == "attention":
        A.mixed_batch_attn(p.cache, C, inc, p.table, dev_bits(q), dev_bits(k), dev_bits(v))
    else:
        still = A.Rope(torch.zeros(d // 2, device="cuda"))          # (angles of 0: keys of the largest magnitude stay what they are)
        A.rope_kv_append(p.cache, C, inc, p.table, still, dev_bits(q), dev_bits(k), dev_bits(v), bounds=p.bounds if way == "rotate_with_bounds" else None)
    torch.cuda.synchronize()
    p.append(C, inc, k, v)
    p.assert_pools_equal()
    if way == "rotate_with_bounds":
        p.set_bounds(C, inc)
        p.assert_bounds_equal()


@pytest.mark.parametrize("way", ["append", "attention", "rotate"])
def test_numbers_above_the_largest_scale_saturate(way):
    """Finite bf16 numbers from 448 * 2^119 up to the largest, in a fresh page and in one that holds tokens."""
    print(f"case: {way}, largest numbers", flush=True)
    Hkv, d, P = 2, 64, 16
    C, inc = np.array([0, 3, 16, 30], np.int32), np.array([2, 1, 3, 4], np.int32)
    p = Pool(9, C, inc, 4, Hkv, d, P, True)
    m = int(inc.sum())
    bits = np.uint16(0x7F60) + p.g.integers(0, 0x20, (2, m, Hkv, d)).astype(np.uint16)
    bits |= (p.g.integers(0, 2, bits.shape) << 15).astype(np.uint16)
    k, v = bits
    if way == "append":
        A.kv_append(p.cache, C, inc, p.table, dev_bits(k), dev_bits(v))
    elif way == "attention":
        A.mixed_batch_attn(p.cache, C, inc, p.table, dev_bits(normal_bits(p.g, m, 4, d)), dev_bits(k), dev_bits(v))
    else:
        A.rope_kv_append(p.cache, C, inc, p.table, A.Rope(torch.zeros(d // 2, device="cuda")), None, dev_bits(k), dev_bits(v))
    torch.cuda.synchronize()
    p.append(C, inc, k, v)
    p.assert_pools_equal()
