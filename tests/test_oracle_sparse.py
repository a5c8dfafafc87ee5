"""Pins of the 64-bit definitions behind the sparse-attention operators: closed forms, brute force, and the properties that the
operators are used for."""
import math

import numpy as np
import pytest

import oracle
import workloads as W
from oracle import sparse as S


def bits(x):
    return W.f32_to_bf16_bits(np.asarray(x, np.float32))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_depends_on_distance_alone(interleaved):
    g = np.random.default_rng(1)
    d, h = 64, 16
    f = (10000.0 ** (-np.arange(h) / h)).astype(np.float32)
    x, y = g.standard_normal((1, 1, d)), g.standard_normal((1, 1, d))
    for a, b in ((0, 0), (5, 3), (1000003, 1000001)):
        rx, ry = S.rope_reference(x, [a], f, interleaved), S.rope_reference(y, [b], f, interleaved)
        assert np.array_equal(rx[..., 2 * h:], x[..., 2 * h:])
        assert abs(np.linalg.norm(rx) - np.linalg.norm(x)) < 1e-12
        near, far = (rx * ry).sum(), (S.rope_reference(x, [a + 77], f, interleaved) * S.rope_reference(y, [b + 77], f, interleaved)).sum()
        assert abs(near - far) < 1e-8
    one = np.zeros((1, 1, d))
    one[0, 0, 0] = 1.0
    r = S.rope_reference(one, [1], np.ones(h, np.float32), interleaved)[0, 0]
    assert abs(r[0] - math.cos(1.0)) < 1e-15 and abs(r[1 if interleaved else h] - math.sin(1.0)) < 1e-15


def test_bounds_hold_every_key_and_their_exponent_is_the_smallest():
    g = np.random.default_rng(2)
    for mult in (1e-30, 2.0 ** -41, 1e-3, 1.0, 127.0, 127.5, 1e20):
        k = oracle.bf16_to_f64(bits(g.standard_normal((16, 64)) * mult))
        codes, scale = S.page_bounds(k)
        hi, lo = codes[0] * float(scale), codes[1] * float(scale)
        assert (k <= hi).all() and (k >= lo).all()
        e = int(math.log2(scale))
        amax = np.abs(k).max()
        assert amax <= 127 * 2.0 ** e and (e == -40 or amax > 127 * 2.0 ** (e - 1))
        assert (hi - k.max(axis=0) <= scale).all() and (k.min(axis=0) - lo <= scale).all()     # (< before the difference is rounded)
    assert S.bounds_exponent(127.0) == 0 and S.bounds_exponent(127.5) == 1 and S.bounds_exponent(0.0) == -40


def test_scores_bound_the_sum_of_logits_up_to_the_rounding_of_the_queries():
    g = np.random.default_rng(3)
    for rows in (1, 4, 128):
        q, k = g.standard_normal((rows, 64)), g.standard_normal((5, 16, 64))
        codes, scale = zip(*(S.page_bounds(x) for x in k))
        s = S.page_scores(q, np.stack(codes), np.array(scale, np.float32)).astype(np.float64)
        f = math.ceil(math.log2(np.abs(q).max() / 127))
        for j in range(5):
            best = np.einsum("rd,td->rt", q, k[j]).max(axis=1).sum()
            # each query is off by half a step in each of 64 channels
            assert s[j] * 2.0 ** f >= best - rows * 64 * 0.5 * 2.0 ** f * np.abs(codes[j]).max() * scale[j]


def test_selection_is_the_brute_force_choice():
    g = np.random.default_rng(4)
    P, Hkv, G, d, n = 16, 2, 2, 64, 20
    codes = g.integers(-127, 128, (n, Hkv, 2, d)).astype(np.int8)
    codes[7] = codes[5]                                                    # equal pages: the lower index wins
    scale = np.ones((n, Hkv), np.float32)
    bt = np.arange(n, dtype=np.int32)[None]
    q = bits(g.standard_normal((1, Hkv * G, d)))
    sel = S.select_reference(codes, scale, bt, [n * P - 1], [1], q, P, 6, 1, 2, 1)[0]
    for h in range(Hkv):
        s = S.page_scores(oracle.bf16_to_f64(q)[0, h * G:(h + 1) * G], codes[:, h], scale[:, h])
        order = sorted(range(1, n - 2), key=lambda j: (-s[j], j))[:3]
        assert sel[h].tolist() == sorted([0, n - 2, n - 1] + order)
    assert S.select_reference(codes, scale, bt, [3 * P], [2], np.repeat(q, 2, 0), P, 8, 1, 2, 2)[0, 0].tolist() == [0, 1, 2, 3] + [-1] * 4


def test_attention_over_all_pages_is_attention():
    b = W.make_batch([33, 0, 15], [5, 9, 1], 4, 2, 64, 16, seed=9)
    off = b.row_offsets
    ref = np.concatenate(oracle.attn_oracle(b.k_pool, b.v_pool, b.block_table, b.ctx_len, b.incr_len, b.q, b.k_new, b.v_new, b.P, b.scale))
    rows = [[np.concatenate([oracle.bf16_to_f64(oracle.gather_request_kv(pool, b.block_table[r], int(b.ctx_len[r]), b.P)),
                             oracle.bf16_to_f64(new[off[r]:off[r + 1]])]) for r in range(3)] for pool, new in ((b.k_pool, b.k_new), (b.v_pool, b.v_new))]
    for g in (1, 4):
        n = len(S.groups_of(b.ctx_len, b.incr_len, g))
        every = np.tile(np.arange(5, dtype=np.int32), (n, 2, 1))
        out, mag, _ = S.sparse_attn_reference(*rows, b.ctx_len, b.incr_len, every, b.q, b.P, b.scale, g)
        assert np.abs(out - ref).max() < 1e-12 and (mag >= np.abs(out) - 1e-12).all()
        none, _, _ = S.sparse_attn_reference(*rows, b.ctx_len, b.incr_len, np.full_like(every, -1), b.q, b.P, b.scale, g)
        assert not none.any()
