"""Helpers for the tests of the sparse-attention operators: a cache on the device with a mirror on the host, filled through the append."""
import numpy as np
import torch

import oracle
import paper_2602_14516_amd as A
import workloads as W
from oracle import sparse as S

BF16_HALF_STEP = 2.0 ** -8            # a rounding to bf16, relative to the value


def dev_bits(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda().view(torch.bfloat16)


def host_bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def normal_bits(g, *shape, mult=1.0):
    return W.f32_to_bf16_bits((g.standard_normal(shape) * mult).astype(np.float32))


class Pool:
    """A cache whose pages hold `tokens` of each row, everything else NaN; the host mirror follows by the oracle's append."""

    def __init__(self, seed, tokens, room, Hq, Hkv, d, P, fp8=False, mult=1.0, spare=3):
        self.g = np.random.default_rng(seed)
        self.Hq, self.Hkv, self.d, self.P, self.fp8 = Hq, Hkv, d, P, fp8
        self.tokens = np.asarray(tokens, np.int32)
        pages_of = (self.tokens + np.asarray(room, np.int32) + P - 1) // P
        self.n = int(pages_of.sum()) + spare
        perm = self.g.permutation(self.n).astype(np.int32)
        self.bt = np.full((len(self.tokens), max(1, int(pages_of.max(initial=0)))), -1, np.int32)
        o = 0
        for r, k in enumerate(pages_of):
            self.bt[r, :k] = perm[o:o + k]
            o += int(k)
        shape = (self.n, Hkv, P, d)
        if fp8:
            self.k, self.v = np.full(shape, 0x7F, np.uint8), np.full(shape, 0x7F, np.uint8)
            self.ks, self.vs = np.full(shape[:2], np.nan, np.float32), np.full(shape[:2], np.nan, np.float32)
        else:
            self.k, self.v = np.full(shape, W.batches.NAN_BF16), np.full(shape, W.batches.NAN_BF16)
            self.ks = self.vs = None
        n = int(self.tokens.sum())
        self.append(np.zeros_like(self.tokens), self.tokens, normal_bits(self.g, n, Hkv, d, mult=mult), normal_bits(self.g, n, Hkv, d))
        self.codes = np.full((self.n, Hkv, 2, d), 99, np.int8)                   # (a mark: bounds that no call set)
        self.bscale = np.full((self.n, Hkv), np.nan, np.float32)
        self.upload()

    def append(self, C, L, k_bits, v_bits):
        if self.fp8:
            self.k, self.ks = oracle.fp8_append_reference(self.k, self.ks, self.bt, C, L, k_bits, self.P)
            self.v, self.vs = oracle.fp8_append_reference(self.v, self.vs, self.bt, C, L, v_bits, self.P)
        else:
            self.k, self.v = oracle.kv_append_reference(self.k, self.v, self.bt, C, L, k_bits, v_bits, self.P)

    def upload(self):
        if self.fp8:
            k, v = torch.from_numpy(self.k.copy()).cuda(), torch.from_numpy(self.v.copy()).cuda()
            ks, vs = torch.from_numpy(self.ks.copy()).cuda(), torch.from_numpy(self.vs.copy()).cuda()
        else:
            k, v, ks, vs = dev_bits(self.k), dev_bits(self.v), None, None
        self.cache = A.KVCache(self.Hq, self.Hkv, self.d, self.P, k, v, float(self.d) ** -0.5, ks, vs, 1 if self.fp8 else 0)
        self.table = torch.from_numpy(self.bt).cuda()
        self.bounds = A.PageBounds(torch.from_numpy(self.codes.copy()).cuda(), torch.from_numpy(self.bscale.copy()).cuda())

    def set_bounds(self, C, L):
        self.codes, self.bscale = S.page_bounds_reference(self.codes, self.bscale, self.k, self.ks, self.bt, C, L, self.P)

    def assert_pools_equal(self):
        """Every byte of the pools, written or not."""
        c = self.cache
        if self.fp8:
            pairs = [(c.k_pool.cpu().numpy(), self.k), (c.v_pool.cpu().numpy(), self.v), (c.k_scale.cpu().numpy().view(np.uint32), self.ks.view(np.uint32)),
                     (c.v_scale.cpu().numpy().view(np.uint32), self.vs.view(np.uint32))]
        else:
            pairs = [(host_bits(c.k_pool), self.k), (host_bits(c.v_pool), self.v)]
        for name, (got, want) in zip(("K", "V", "K scales", "V scales"), pairs):
            assert np.array_equal(got, want), f"{name}: {np.argwhere(got != want)[:5].tolist()}"

    def assert_bounds_equal(self):
        got, scale = self.bounds.codes.cpu().numpy(), self.bounds.scale.cpu().numpy()
        assert np.array_equal(scale.view(np.uint32), self.bscale.view(np.uint32)), np.argwhere(scale.view(np.uint32) != self.bscale.view(np.uint32))[:5].tolist()
        assert np.array_equal(got, self.codes), np.argwhere(got != self.codes)[:5].tolist()

    def rows(self, which, T):
        """Per request the stored values [T, Hkv, d] float64."""
        pool, scale = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        out = []
        for r, t in enumerate(T):
            if self.fp8:
                out.append(oracle.fp8_dequant_request(pool, scale, self.bt[r], int(t), self.P))
            else:
                out.append(oracle.bf16_to_f64(oracle.gather_request_kv(pool, self.bt[r], int(t), self.P)))
        return out


def check_attention(got, ref, mag, dots, label=""):
    """got: float64 from bf16 rows.  The kernel's probabilities are off by three things, each relative to the probability: the logit
    (a sum of d <= 128 products in 32 bits: 128 * 2^-24 of the sum of their magnitudes, `dots`, twice for the logit and the reference it is
    taken against), exp2 and its argument (a step of 2^-23 of a number of at most 2 * dots * log2 e, and 2^-22 of the result), and its
    rounding to bf16 for the second product (2^-8); the sums run in 32 bits (2^-12 together, for up to 2^12 terms).  They weigh |v|: `mag`.
    Then the output is rounded."""
    logit = 2 * 128 * 2.0 ** -24 * dots + 3 * 2.0 ** -23 * dots + 2.0 ** -22
    bound = (mag * (2.0 ** -8 + 2.0 ** -12 + logit[..., None])) * (1 + 2.0 ** -8) + BF16_HALF_STEP * np.abs(ref) + 1e-30
    assert np.isfinite(got).all(), f"{label}: not finite"
    worst = float((np.abs(got - ref) / bound).max(initial=0.0))
    assert worst <= 1.0, f"{label}: {worst:.2f} of the bound"
    return worst
