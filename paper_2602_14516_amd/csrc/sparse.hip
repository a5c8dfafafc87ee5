// HIP kernels for gfx950 of sparse attention over a paged KV cache: rotate and append, page bounds, page selection, attention over the
// selected pages (the steps of a block of 32 keys are those of the dense kernels, see kernels.hip).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "sparse.h"
#include "steps.h"

namespace ampd {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------------
// page bounds

// Chunks of 8 elements of a key are handled in pairs, D / 16 to a key: unit u of a page is slot u / (D / 16), pair u % (D / 16), and a lane
// whose units are 64 apart keeps its pair.
template <int D>
struct Units {
    static constexpr int PPT = D / 16;                // pairs per token
    static constexpr int COUNT(int P) { return P * PPT / 64; }
};

__device__ __forceinline__ void unpack8(const u32x4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void decode8(uint32_t lo, uint32_t hi, float (&f)[8]) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(lo, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(lo, true);
    const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), d = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
}

template <int CTRL>
__device__ __forceinline__ uint32_t add_dpp(uint32_t x) {
    return x + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
// the sum over the 16 lanes of a row, in all of them
__device__ __forceinline__ uint32_t row_sum(uint32_t x) {
    x = add_dpp<0xB1>(x);                             // quad_perm [1, 0, 3, 2]
    x = add_dpp<0x4E>(x);                             // quad_perm [2, 3, 0, 1]
    x = add_dpp<0x124>(x);                            // row_ror:4
    return add_dpp<0x128>(x);                         // row_ror:8
}

__device__ __forceinline__ uint32_t max16x2(uint32_t a, uint32_t b) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ uint32_t wave_umax(uint32_t x) {
    x = max_dpp<0xB1>(x);
    x = max_dpp<0x4E>(x);
    x = max_dpp<0x124>(x);
    x = max_dpp<0x128>(x);
    u32x2 r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(r[0], r[1]);
    r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max(r[0], r[1]);
}
__device__ __forceinline__ uint32_t wave_umin(uint32_t x) { return ~wave_umax(~x); }
__device__ __forceinline__ uint32_t wave_usum(uint32_t x) {
    x = row_sum(x);
    u32x2 r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = r[0] + r[1];
    r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return r[0] + r[1];
}

// the largest of non-negative numbers
__device__ __forceinline__ float wave_max(float x) { return __uint_as_float(wave_umax(__float_as_uint(x))); }

typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t smax16x2(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, a), __builtin_bit_cast(i16x2, b)));
}
__device__ __forceinline__ uint32_t smin16x2(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(i16x2, a), __builtin_bit_cast(i16x2, b)));
}
// Two bf16 values as whole numbers that order as they do, and back: the magnitude of negative ones is inverted.
__device__ __forceinline__ uint32_t ordered16x2(uint32_t x) {
    const i16x2 sign = __builtin_bit_cast(i16x2, x) >> 15;
    return x ^ (__builtin_bit_cast(uint32_t, sign) & 0x7fff7fffu);
}

// The lane's largest and smallest values so far of its 16 channels (chunk a: words 0..3, chunk b: 4..7, two channels each), over its own units.
// (Two to an instruction, and exchanged by swaps of lanes: in 32 bits with exchanges through LDS a reply of 701 tokens took 3.8 us instead of 3.1,
// one token rotated and appended 5.7 instead of 5.0.)
struct LaneBounds {
    uint32_t hi[8], lo[8];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            hi[i] = 0x80008000u;
            lo[i] = 0x7fff7fffu;
        }
    }
    __device__ __forceinline__ void take(int at, const u32x4& chunk) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = ordered16x2(chunk[i]);
            hi[at + i] = smax16x2(hi[at + i], x);
            lo[at + i] = smin16x2(lo[at + i], x);
        }
    }
    // 8-bit codes as their values
    __device__ __forceinline__ void take_codes(int at, uint32_t c0, uint32_t c1) { take(at, RawChunk<KV_FP8>::widen8(c0, c1, 1.0f)); }
};

// smallest e with amax <= 127 * 2^e  (127 = 1.984375 * 2^6), clamped to [-40, 96]
__device__ __forceinline__ int bounds_exponent(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int ex = (int)(u >> 23) - 127;
    int e = (u & 0x7fffffu) <= 0x7e0000u ? ex - 6 : ex - 5;
    if ((u >> 23) == 0) e = -40;                      // zero / subnormal
    return min(96, max(-40, e));
}

// Bounds of a page of one KV head from the wave's lanes; unit: what the lanes' values count in (a power of two: an 8-bit page's scale).
// The 64 / (D / 16) lanes that share a pair of chunks halve their words three times: a swap of rows of lanes leaves each lane both lanes' values
// of the half that it keeps.
template <int D>
__device__ __forceinline__ void store_bounds(LaneBounds& b, float unit, int ca, int cb, int lane, int8_t* codes, float* scale) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {                     // lanes 0..31 keep chunk a
        const u32x2 h = __builtin_amdgcn_permlane32_swap(b.hi[i], b.hi[4 + i], false, false), l = __builtin_amdgcn_permlane32_swap(b.lo[i], b.lo[4 + i], false, false);
        b.hi[i] = smax16x2(h[0], h[1]);
        b.lo[i] = smin16x2(l[0], l[1]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {                     // rows 0 and 2 of 16 lanes words 0 and 1
        const u32x2 h = __builtin_amdgcn_permlane16_swap(b.hi[i], b.hi[2 + i], false, false), l = __builtin_amdgcn_permlane16_swap(b.lo[i], b.lo[2 + i], false, false);
        b.hi[i] = smax16x2(h[0], h[1]);
        b.lo[i] = smin16x2(l[0], l[1]);
    }
    const bool upper = lane & 8;                      // lanes 0..7 of a row the first of the two
    auto other = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true); };     // row_ror:8
    uint32_t hw = smax16x2(upper ? b.hi[1] : b.hi[0], other(upper ? b.hi[0] : b.hi[1]));
    uint32_t lw = smin16x2(upper ? b.lo[1] : b.lo[0], other(upper ? b.lo[0] : b.lo[1]));
    if constexpr (D == 64) {                          // four pairs to a key: lanes 4 apart share one still
        hw = smax16x2(hw, (uint32_t)__shfl_xor((int)hw, 4, 64));
        lw = smin16x2(lw, (uint32_t)__shfl_xor((int)lw, 4, 64));
    }
    hw = ordered16x2(hw);
    lw = ordered16x2(lw);
    const int x = (lane & 32 ? cb : ca) * 8 + (lane & 16 ? 4 : 0) + (upper ? 2 : 0);     // the first of the lane's two channels
    const float hv[2] = {__uint_as_float(hw << 16) * unit, __uint_as_float(hw & 0xffff0000u) * unit};
    const float lv[2] = {__uint_as_float(lw << 16) * unit, __uint_as_float(lw & 0xffff0000u) * unit};
    const float amax = fmaxf(fmaxf(fabsf(hv[0]), fabsf(hv[1])), fmaxf(fabsf(lv[0]), fabsf(lv[1])));
    const int e = bounds_exponent(wave_max(amax));
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t h = 0, l = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        // (a value that underflows when it is scaled still counts)
        float u = ceilf(hv[i] * inv), d = floorf(lv[i] * inv);
        if (hv[i] > 0.0f) u = fmaxf(u, 1.0f);
        if (lv[i] < 0.0f) d = fminf(d, -1.0f);
        h |= ((uint32_t)(int)fminf(fmaxf(u, -127.0f), 127.0f) & 0xff) << (8 * i);
        l |= ((uint32_t)(int)fminf(fmaxf(d, -127.0f), 127.0f) & 0xff) << (8 * i);
    }
    if (D == 128 || !(lane & 4)) {
        *reinterpret_cast<uint16_t*>(codes + x) = (uint16_t)h;
        *reinterpret_cast<uint16_t*>(codes + D + x) = (uint16_t)l;
    }
    if (lane == 0) *scale = __uint_as_float((uint32_t)(e + 127) << 23);
}

// A wave per page and KV head.  Bound: memory, 165 MB in 31 us (35 without non-temporal loads), of which the launch's beginning and end are 4.
// (Two heads per wave gain 3 % of that, and cost a reply of 701 tokens 25 %.)
template <int D, int P, int KVT>
__global__ __launch_bounds__(WG) void page_bounds_kernel(const BoundsParams p) {
    constexpr int PPT = Units<D>::PPT, NU = Units<D>::COUNT(P);
    const int lane = threadIdx.x & 63, h = blockIdx.y * (WG / 64) + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const PageJob j = page_job(p.a);
    if (h >= p.a.Hkv || (uint32_t)j.page >= (uint64_t)p.num_pages) return;
    const int slots = j.t1 - (j.t0 & ~(P - 1)), pair = lane % PPT;
    const int64_t ph = (int64_t)j.page * p.a.Hkv + h;
    const char* pg = static_cast<const char*>(p.a.k_pool) + ph * (P * D * (KVT == KV_FP8 ? 1 : 2));
    float unit = 1.0f;
    if constexpr (KVT == KV_FP8) unit = p.a.k_scale[ph];
    LaneBounds b;
    b.clear();
    u32x4 x[NU], y[NU];
#pragma unroll
    for (int k = 0; k < NU; ++k) {
        const int s = min((lane + 64 * k) / PPT, slots - 1);              // (a slot behind the last token: the last token's once more)
        if constexpr (KVT == KV_BF16) {
            x[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(pg + s * (D * 2) + pair * 16));
            y[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(pg + s * (D * 2) + (pair + PPT) * 16));
        } else {
            x[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(pg + s * D + pair * 16));
        }
    }
#pragma unroll
    for (int k = 0; k < NU; ++k) {
        if constexpr (KVT == KV_BF16) {
            b.take(0, x[k]);
            b.take(4, y[k]);
        } else {
            b.take_codes(0, x[k].x, x[k].y);
            b.take_codes(4, x[k].z, x[k].w);
        }
    }
    const int ca = KVT == KV_BF16 ? pair : 2 * pair, cb = KVT == KV_BF16 ? pair + PPT : 2 * pair + 1;
    store_bounds<D>(b, unit, ca, cb, lane, p.codes + ph * (2 * D), p.bscale + ph);
}

// ---------------------------------------------------------------------------------------------
// rotate and append

// The chunks of a pair, so that the lanes of a key take neighbouring chunks with each load: two whose elements the rotation pairs (half
// apart) or, where it pairs neighbours or copies, any two.  ra, rb: whether they are rotated; a chunk of 8 elements is so as a whole.
struct ChunkPair {
    int a, b;
    bool ra, rb;
};
template <int D>
__device__ __forceinline__ ChunkPair chunk_pair(int pair, int rd, bool interleaved) {
    constexpr int PPT = Units<D>::PPT;
    const int half = rd >> 4;
    if (interleaved) return {pair, pair + PPT, pair < 2 * half, pair + PPT < 2 * half};
    if (pair < half) return {pair, pair + half, true, true};
    return {half + pair, PPT + pair, false, false};   // (the rest, 2 half .. 2 PPT, in two runs)
}

// Rotate a pair of chunks in type F; cs(i): cosine and sine of the i-th of the 8 angles of the pair (half apart: those of elements 0..7;
// interleaved: of the 4 pairs of chunk a, then of chunk b).
template <class F, class CS>
__device__ __forceinline__ void rotate(u32x4& va, u32x4& vb, const ChunkPair& cp, bool interleaved, CS&& cs) {
    float a[8], b[8];
    unpack8(va, a);
    unpack8(vb, b);
    bf16x8 ra, rb;
    auto turn = [&](int i, float x1, float x2, __bf16& y1, __bf16& y2) {
        F c, s;
        cs(i, c, s);
        float f1 = (float)((F)x1 * c - (F)x2 * s), f2 = (float)((F)x2 * c + (F)x1 * s);
        // two roundings, as defined: the compiler would make one of 64 -> 32 -> 16 bits (it differs where 32 bits end on a tie, 4 of a million)
        if constexpr (sizeof(F) == 8) asm("" : "+v"(f1), "+v"(f2));
        y1 = (__bf16)f1;
        y2 = (__bf16)f2;
    };
    if (interleaved) {                                // uniform
        if (cp.ra) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                __bf16 y1, y2;
                turn(i, a[2 * i], a[2 * i + 1], y1, y2);
                ra[2 * i] = y1;
                ra[2 * i + 1] = y2;
            }
            va = __builtin_bit_cast(u32x4, ra);
        }
        if (cp.rb) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                __bf16 y1, y2;
                turn(4 + i, b[2 * i], b[2 * i + 1], y1, y2);
                rb[2 * i] = y1;
                rb[2 * i + 1] = y2;
            }
            vb = __builtin_bit_cast(u32x4, rb);
        }
    } else if (cp.ra) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __bf16 y1, y2;
            turn(i, a[i], b[i], y1, y2);
            ra[i] = y1;
            rb[i] = y2;
        }
        va = __builtin_bit_cast(u32x4, ra);
        vb = __builtin_bit_cast(u32x4, rb);
    }
}

// Bound: memory (8 400 tokens of 32 + 2 x 8 heads of 128, 208 MB in 51 us, where a copy of as many bytes takes 42; the angles, the rotation in
// 64 bits and non-temporal loads or stores do not show in it), latency for few tokens (one: 5.0 us).
// One workgroup column per page that new tokens fall into; the column's waves share its jobs: K of a head, V of a head (the page's new tokens
// in registers, with the cached ones where the page's scale or bounds need them), and runs of 256 pairs of chunks of Q.
// The angles' cosines and sines are computed once per workgroup, in 64 bits, and kept as two 32-bit parts each: Q is rotated by the
// first, K by both, in 64 bits (K decides 8-bit codes, scales, bounds and through them page choices, which are whole numbers).
template <int D, int P, int KVT, bool BOUNDS>
__global__ __launch_bounds__(WG) void rope_append_kernel(const RopeParams p) {
    constexpr int PPT = Units<D>::PPT, NU = Units<D>::COUNT(P), ES = KVT == KV_FP8 ? 1 : 2;
    __shared__ f32x2 head[P * D / 2], tail[P * D / 2];                // (cos, sin) of token t, angle i at t * rd / 2 + i
    const AppendParams& a = p.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const PageJob j = page_job(a);
    const int n = j.t1 - j.t0, s0 = j.t0 & (P - 1), F = p.rd >> 1;
    for (int i = threadIdx.x; i < n * F; i += WG) {
        const int t = i / F;
        const int pos = p.positions ? p.positions[j.row + t] : j.t0 + t;
        double s, c;
        sincos((double)pos * (double)p.inv_freq[i - t * F], &s, &c);
        c *= (double)p.scale;
        s *= (double)p.scale;
        const f32x2 top = {(float)c, (float)s};
        head[i] = top;
        tail[i] = f32x2{(float)(c - (double)top.x), (float)(s - (double)top.y)};
    }
    __syncthreads();
    const int nkv = (uint32_t)j.page < (uint64_t)p.num_pages ? 2 * a.Hkv : 0, nq = p.q ? (n * p.Hq * PPT + 255) / 256 : 0;
    const ChunkPair cp = chunk_pair<D>(lane % PPT, p.rd, p.interleaved);
    // the i-th angle of the lane's pair, in table order
    const int f0 = p.interleaved ? 4 * cp.a : 8 * cp.a, f1 = p.interleaved ? 4 * cp.b - 4 : f0;   // angles 0..3 from f0, 4..7 from f1
    for (int job = blockIdx.y * (WG / 64) + wave; job < nkv + nq; job += gridDim.y * (WG / 64)) {
        if (job >= nkv) {
            const int units = n * p.Hq * PPT, u0 = (job - nkv) * 256 + lane;
            const float inv = __builtin_amdgcn_rcpf((float)p.Hq);
            u32x4 x[4], y[4];
            int tok[4], at[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int u = min(u0 + 64 * k, units - 1), th = u / PPT;
                tok[k] = (int)(((float)th + 0.5f) * inv);                     // th / Hq: th < 2^20, Hq < 2^14
                at[k] = th - tok[k] * p.Hq;
                const char* src = static_cast<const char*>(p.q) + (int64_t)(j.row + tok[k]) * p.q_stride + at[k] * (D * 2);
                x[k] = *reinterpret_cast<const u32x4*>(src + cp.a * 16);
                y[k] = *reinterpret_cast<const u32x4*>(src + cp.b * 16);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (cp.ra || cp.rb) {
                    const f32x2* t = head + tok[k] * F;
                    rotate<float>(x[k], y[k], cp, p.interleaved, [&](int i, float& c, float& s) {
                        const f32x2 v = t[(i < 4 ? f0 : f1) + i];
                        c = v.x;
                        s = v.y;
                    });
                }
                if (u0 + 64 * k < units) {
                    char* dst = static_cast<char*>(p.q_out) + ((int64_t)(j.row + tok[k]) * p.Hq + at[k]) * (D * 2);
                    *reinterpret_cast<u32x4*>(dst + cp.a * 16) = x[k];
                    *reinterpret_cast<u32x4*>(dst + cp.b * 16) = y[k];
                }
            }
            continue;
        }
        const bool is_v = job >= a.Hkv;
        const int h = is_v ? job - a.Hkv : job;
        const int64_t ph = (int64_t)j.page * a.Hkv + h;
        const char* src = static_cast<const char*>(is_v ? a.v_new : a.k_new) + (int64_t)j.row * (is_v ? p.v_stride : p.k_stride) + h * (D * 2);
        const int64_t stride = is_v ? p.v_stride : p.k_stride;
        char* pg = static_cast<char*>(is_v ? a.v_pool : a.k_pool) + ph * (P * D * ES);
        const bool cached = s0 > 0 && (KVT == KV_FP8 || (BOUNDS && !is_v));
        float* scl = KVT == KV_FP8 ? (is_v ? a.v_scale : a.k_scale) + ph : nullptr;
        float s_old = 1.0f;
        if (KVT == KV_FP8 && s0 > 0) s_old = *scl;
        float unit = 1.0f;
        LaneBounds lb;
        if (BOUNDS) lb.clear();
        // Units in runs: over a bf16 cache each run is done with before the next, so that a page of 64 tokens takes no more registers than one
        // of 32; 8-bit pages need all new tokens' magnitudes first.
        constexpr int RUN = KVT == KV_FP8 ? NU : NU < 4 ? NU : 4;
#pragma unroll 1
        for (int k0 = 0; k0 < NU; k0 += RUN) {
            u32x4 x[RUN], y[RUN];
            const int base = lane + 64 * k0;
#pragma unroll
            for (int k = 0; k < RUN; ++k) {
                const int s = (base + 64 * k) / PPT;
                x[k] = y[k] = u32x4{0, 0, 0, 0};
                if (s >= s0 && s < s0 + n) {
                    const char* r = src + (s - s0) * stride;
                    x[k] = *reinterpret_cast<const u32x4*>(r + cp.a * 16);
                    y[k] = *reinterpret_cast<const u32x4*>(r + cp.b * 16);
                } else if (cached && s < s0) {
                    if constexpr (KVT == KV_BF16) {
                        x[k] = *reinterpret_cast<const u32x4*>(pg + (s * D + cp.a * 8) * 2);
                        y[k] = *reinterpret_cast<const u32x4*>(pg + (s * D + cp.b * 8) * 2);
                    } else {
                        const u32x2 ca = *reinterpret_cast<const u32x2*>(pg + s * D + cp.a * 8), cb = *reinterpret_cast<const u32x2*>(pg + s * D + cp.b * 8);
                        x[k] = u32x4{ca.x, ca.y, cb.x, cb.y};
                    }
                }
            }
            if (!is_v && (cp.ra || cp.rb)) {
#pragma unroll
                for (int k = 0; k < RUN; ++k) {
                    const int s = (base + 64 * k) / PPT;
                    if (s >= s0 && s < s0 + n) {
                        const int t = (s - s0) * F;
                        rotate<double>(x[k], y[k], cp, p.interleaved, [&](int i, double& c, double& sn) {
                            const f32x2 v = head[t + (i < 4 ? f0 : f1) + i], w = tail[t + (i < 4 ? f0 : f1) + i];
                            c = (double)v.x + (double)w.x;
                            sn = (double)v.y + (double)w.y;
                        });
                    }
                    __builtin_amdgcn_sched_barrier(0);                    // (one unit at a time: registers)
                }
            }
            if constexpr (KVT == KV_FP8) {
                float amax = 0.0f;
#pragma unroll
                for (int k = 0; k < RUN; ++k) {
                    const int s = (base + 64 * k) / PPT;
                    if (s >= s0) amax = fmaxf(amax, fmaxf(chunk_amax(x[k]), chunk_amax(y[k])));
                }
                int e = exponent_for(wave_max(amax));
                const int e_old = (int)(__float_as_uint(s_old) >> 23) - 127;
                const bool raise = s0 > 0 && e > e_old;
                if (s0 > 0 && !raise) e = e_old;
                const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
                const float f = reencode_factor(e_old, e);                               // (used where the exponent rises)
#pragma unroll
                for (int k = 0; k < RUN; ++k) {
                    const int s = (base + 64 * k) / PPT;
                    const bool fresh = s >= s0;
                    if (fresh) {
                        const u32x2 ca = encode_chunk(x[k], inv), cb = encode_chunk(y[k], inv);
                        x[k] = u32x4{ca.x, ca.y, cb.x, cb.y};
                    } else if (raise) {
                        float g[8];
                        decode8(x[k].x, x[k].y, g);
                        x[k].x = encode4(g[0] * f, g[1] * f, g[2] * f, g[3] * f);
                        x[k].y = encode4(g[4] * f, g[5] * f, g[6] * f, g[7] * f);
                        decode8(x[k].z, x[k].w, g);
                        x[k].z = encode4(g[0] * f, g[1] * f, g[2] * f, g[3] * f);
                        x[k].w = encode4(g[4] * f, g[5] * f, g[6] * f, g[7] * f);
                    }
                    if (s < s0 + n && (fresh || raise)) {
                        *reinterpret_cast<u32x2*>(pg + s * D + cp.a * 8) = u32x2{x[k].x, x[k].y};
                        *reinterpret_cast<u32x2*>(pg + s * D + cp.b * 8) = u32x2{x[k].z, x[k].w};
                    }
                }
                unit = __uint_as_float((uint32_t)(e + 127) << 23);
                if (lane == 0) *scl = unit;
            } else {
#pragma unroll
                for (int k = 0; k < RUN; ++k) {
                    const int s = (base + 64 * k) / PPT;
                    if (s >= s0 && s < s0 + n) {
                        *reinterpret_cast<u32x4*>(pg + (s * D + cp.a * 8) * 2) = x[k];
                        *reinterpret_cast<u32x4*>(pg + (s * D + cp.b * 8) * 2) = y[k];
                    }
                }
            }
            if constexpr (BOUNDS) {
                if (!is_v) {
#pragma unroll
                    for (int k = 0; k < RUN; ++k) {
                        if ((base + 64 * k) / PPT >= s0 + n) continue;
                        if constexpr (KVT == KV_BF16) {
                            lb.take(0, x[k]);
                            lb.take(4, y[k]);
                        } else {
                            lb.take_codes(0, x[k].x, x[k].y);
                            lb.take_codes(4, x[k].z, x[k].w);
                        }
                    }
                }
            }
        }
        if constexpr (BOUNDS) {
            if (!is_v) store_bounds<D>(lb, unit, cp.a, cp.b, lane, p.codes + ph * (2 * D), p.bscale + ph);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// page selection

// The row of a launch that owns item idx: the last one that starts at or before it.  Every lane loads a row or two and the owner's is picked
// from the lanes.  The loads do not wait for n, so they make one trip to the arguments together with the scalar ones (what lies behind the n rows
// is not looked at).
template <int MAX, class Row, class F>
__device__ __forceinline__ Row row_of(const Row* rows, int n, int idx, F&& start) {
    static_assert(MAX > 64 && MAX <= 128 && sizeof(Row) % 4 == 0, "two rows per lane");
    constexpr int W = sizeof(Row) / 4;
    struct Words {
        int32_t w[W];
    };
    const int lane = threadIdx.x & 63;
    const Row a = rows[lane], b = rows[min(lane + 64, MAX - 1)];
    const int r = __popcll(__ballot(lane < n && start(a) <= idx)) + __popcll(__ballot(lane + 64 < n && start(b) <= idx)) - 1;
    const Words x = __builtin_bit_cast(Words, a), y = __builtin_bit_cast(Words, b);
    Words out;
#pragma unroll
    for (int i = 0; i < W; ++i) out.w[i] = __builtin_amdgcn_readlane(r < 64 ? x.w[i] : y.w[i], r & 63);
    return __builtin_bit_cast(Row, out);
}

// bytes b < 128 -> -b: 128 - b has bit 7 set where b is 0 alone; with bit 7 flipped it is -b modulo 256
__device__ __forceinline__ uint32_t negate_bytes(uint32_t x) { return (0x80808080u - x) ^ 0x80808080u; }

// 2^-f for the smallest f with amax <= 127 * 2^f, in two factors: f reaches -139 (one step above zero) and 122 (a group of zeros: any)
__device__ __forceinline__ void query_step(uint32_t amax_bits, float& m0, float& m1) {
    const float amax = __uint_as_float(amax_bits);    // = mantissa in [0.5, 1) * 2^x, numbers without a leading one included
    const int x = __builtin_amdgcn_frexp_expf(amax), f = __builtin_amdgcn_frexp_mantf(amax) <= 0.9921875f ? x - 7 : x - 6;
    const int fs = max(-126, min(127, -f));
    m0 = __uint_as_float((uint32_t)(fs + 127) << 23);
    m1 = __uint_as_float((uint32_t)(max(-126, min(127, -f - fs)) + 127) << 23);
}

// Whole numbers of a group's queries for one KV head, summed over its rows (tokens x heads), as two limbs of 7 bits in the operand layout of
// the 16x16x64 product: lane l holds bytes 16 (l / 16) .. of k-block kk; k = 0..d-1 the sums of the positive parts, d..2d-1 of the
// negative ones.  Every lane of a row of 16 ends up with the same.  At most 128 rows of at most 127 each: sums below 2^14.
// The lanes of a row of 16 take the group's rows in turn, the first 32 in flight at once.
template <int D>
__device__ __forceinline__ void quantise_queries(const char* q, int64_t token_bytes, int G, int rows, int lane, i32x4 (&limb)[2][D / 32]) {
    constexpr int NB = D / 64;                        // 64-channel blocks
    const int col = lane & 15;
    auto load = [&](int r, u32x4 (&x)[NB][2]) {       // (a lane without a row: the last one's once more, not counted)
        r = min(r, rows - 1);
        const int t = r / G;
        const char* src = q + t * token_bytes + (r - t * G) * (D * 2) + (lane >> 4) * 32;
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) {
            x[blk][0] = *reinterpret_cast<const u32x4*>(src + blk * 128);
            x[blk][1] = *reinterpret_cast<const u32x4*>(src + blk * 128 + 16);
        }
    };
    auto magnitude = [](const u32x4 (&v)[NB][2]) {
        uint32_t m = 0;                               // two 16-bit magnitudes
#pragma unroll
        for (int blk = 0; blk < NB; ++blk)
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int w = 0; w < 4; ++w) m = max16x2(m, v[blk][half][w] & 0x7fff7fffu);
        return m;
    };
    u32x4 x0[NB][2], x1[NB][2];
    load(col, x0);
    if (rows > 16) load(col + 16, x1);                // uniform
    uint32_t m = magnitude(x0);
    if (rows > 16) m = max16x2(m, magnitude(x1));
    for (int r = 32; r < rows; r += 16) {
        u32x4 y[NB][2];
        load(r + col, y);
        m = max16x2(m, magnitude(y));
    }
    float m0, m1;
    query_step(wave_umax(max(m >> 16, m & 0xffffu)) << 16, m0, m1);
    uint32_t sum[NB][16];                             // positive | negative << 16
#pragma unroll
    for (int blk = 0; blk < NB; ++blk)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[blk][i] = 0;
    auto add = [&](const u32x4 (&v)[NB][2], bool there) {
#pragma unroll
        for (int blk = 0; blk < NB; ++blk)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float y[8];
                unpack8(v[blk][half], y);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = (int)fminf(fmaxf(rintf(y[i] * m0 * m1), -127.0f), 127.0f);
                    const uint32_t one = c >= 0 ? (uint32_t)c : (uint32_t)(-c) << 16;
                    sum[blk][half * 8 + i] += there ? one : 0u;
                }
            }
    };
    add(x0, col < rows);
    if (rows > 16) add(x1, col + 16 < rows);
    for (int r = 32; r < rows; r += 16) {
        u32x4 y[NB][2];
        load(r + col, y);
        add(y, r + col < rows);
    }
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            // bytes of four channels: the low 7 bits and the rest, of the positive sums and, negated, of the negative ones
            uint32_t pl = 0, ph = 0, nl = 0, nh = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t s = row_sum(sum[blk][w * 4 + i]), lo = s & 0x007f007fu, hi = (s >> 7) & 0x007f007fu;
                pl |= (lo & 0xff) << (8 * i);
                nl |= (lo >> 16) << (8 * i);
                ph |= (hi & 0xff) << (8 * i);
                nh |= (hi >> 16) << (8 * i);
            }
            limb[0][blk][w] = (int)pl;
            limb[1][blk][w] = (int)ph;
            limb[0][NB + blk][w] = (int)negate_bytes(nl);
            limb[1][NB + blk][w] = (int)negate_bytes(nh);
        }
    }
}

// The same numbers for the dot products of single-token rows: lane l holds bytes 16 (l % LPP) .. of the 2d (LPP = 2d / 16 lanes to a page), so that a
// load of 64 lanes takes whole neighbouring bytes of 64 / LPP pages.  As the second operand of a matrix product every load would touch 16 pages
// for half a line each (96 rows of 2-16 k tokens: 38 us).
template <int D>
struct RowCodes {
    static constexpr int LPP = D / 8, PPI = 64 / LPP;
    u32x4 x[2];
    __device__ __forceinline__ static void load(const char* q, int64_t token_bytes, int G, int r, int lane, u32x4 (&x)[2]) {
        const int t = r / G;
        const char* src = q + t * token_bytes + (r - t * G) * (D * 2) + (lane % (D / 16)) * 32;
        x[0] = *reinterpret_cast<const u32x4*>(src);
        x[1] = *reinterpret_cast<const u32x4*>(src + 16);
    }
    __device__ __forceinline__ void start(const char* q, int64_t token_bytes, int G, int rows, int lane) {
        load(q, token_bytes, G, min(lane / LPP, rows - 1), lane, x);      // (a lane without a row: the last one's once more, not counted)
    }
    // limb[l]: 16 bytes of limb l
    __device__ __forceinline__ void finish(const char* q, int64_t token_bytes, int G, int rows, int lane, i32x4 (&limb)[2]) const {
        const bool neg = lane % LPP >= D / 16;
        auto magnitude = [](const u32x4 (&v)[2]) {
            uint32_t m = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) m = max16x2(m, v[w >> 2][w & 3] & 0x7fff7fffu);
            return m;
        };
        uint32_t m = magnitude(x);
        for (int r = lane / LPP + PPI; r < rows; r += PPI) {
            u32x4 y[2];
            load(q, token_bytes, G, r, lane, y);
            m = max16x2(m, magnitude(y));
        }
        float m0, m1;
        query_step(wave_umax(max(m >> 16, m & 0xffffu)) << 16, m0, m1);
        const float least = neg ? -127.0f : 0.0f, most = neg ? 0.0f : 127.0f;
        uint32_t sum[8];                              // two channels each
        auto add = [&](const u32x4 (&v)[2], bool first) {
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                const uint32_t u = v[w >> 2][w & 3];
                const float a = fminf(fmaxf(rintf(__uint_as_float(u << 16) * m0 * m1), least), most);
                const float b = fminf(fmaxf(rintf(__uint_as_float(u & 0xffff0000u) * m0 * m1), least), most);
                const uint32_t one = (uint32_t)fabsf(a) | (uint32_t)fabsf(b) << 16;
                sum[w] = first ? one : sum[w] + one;
            }
        };
        add(x, true);
        if (lane / LPP >= rows) {
#pragma unroll
            for (int w = 0; w < 8; ++w) sum[w] = 0;
        }
        for (int r = lane / LPP + PPI; r < rows; r += PPI) {
            u32x4 y[2];
            load(q, token_bytes, G, r, lane, y);
            add(y, false);
        }
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            if constexpr (LPP == 8) sum[w] = add_dpp<0x128>(sum[w]);      // row_ror:8
            u32x2 r = __builtin_amdgcn_permlane16_swap(sum[w], sum[w], false, false);
            const uint32_t t = r[0] + r[1];
            r = __builtin_amdgcn_permlane32_swap(t, t, false, false);
            sum[w] = r[0] + r[1];
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t a = sum[2 * w], b = sum[2 * w + 1];
            const uint32_t lo = __builtin_amdgcn_perm(b & 0x007f007fu, a & 0x007f007fu, 0x06040200u);
            const uint32_t hi = __builtin_amdgcn_perm((b >> 7) & 0x007f007fu, (a >> 7) & 0x007f007fu, 0x06040200u);
            limb[0][w] = (int)(neg ? negate_bytes(lo) : lo);
            limb[1][w] = (int)(neg ? negate_bytes(hi) : hi);
        }
    }
};

// A wave per group and KV head: the operand bytes, for the score launch's tiles of 16 groups.
template <int D>
__global__ __launch_bounds__(64) void query_codes_kernel(const SelectParams p) {
    const int lane = threadIdx.x, item = blockIdx.x, h = blockIdx.y, G = p.Hq / p.Hkv;
    const SelectRow r = row_of<SELECT_MAX_REQS>(p.rows, p.n, item, [](const SelectRow& x) { return x.item0; });
    const int tok0 = (item - r.item0) * p.g, m = min(p.g, r.L - tok0);
    const char* q = static_cast<const char*>(p.q) + ((int64_t)(r.row_off + tok0) * p.Hq + h * G) * (D * 2);
    i32x4 limb[2][D / 32];
    quantise_queries<D>(q, (int64_t)p.Hq * D * 2, G, m * G, lane, limb);
    if ((lane & 15) == 0) {
        int8_t* dst = p.qcodes + ((int64_t)item * p.Hkv + h) * (4 * D) + (lane >> 4) * 16;
#pragma unroll
        for (int l = 0; l < 2; ++l)
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk) *reinterpret_cast<i32x4*>(dst + l * (2 * D) + kk * 64) = limb[l][kk];
    }
}

// Scores as 32-bit numbers that order as the scores do; a page without a place in the pool (there: false) comes behind every score.
__device__ __forceinline__ uint32_t ordered(float x, bool there) {
    const uint32_t u = __float_as_uint(x);
    return there ? u & 0x80000000u ? ~u : u | 0x80000000u : 0u;
}

// A tile of 16 pages: their bounds of one KV head, as the second operand of the 16x16x64 whole-number product (lane l: bytes 16 (l / 16) .. of
// k-block kk of page l % 16; k = 0..2d-1: the largest keys' codes, then the smallest ones').
template <int D>
struct PageTile {
    i32x4 b[D / 32];
    float scale;
    bool there;
    __device__ __forceinline__ void load(const SelectParams& p, int id, int h, int lane) {
        there = (uint32_t)id < (uint64_t)p.num_pages;
        const int64_t ph = (int64_t)(there ? id : 0) * p.Hkv + h;
        const int8_t* src = p.codes + ph * (2 * D) + (lane >> 4) * 16;
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) b[kk] = *reinterpret_cast<const i32x4*>(src + kk * 64);
        scale = p.bscale[ph];
    }
    // the groups' queries (first operand, lane l: group l % 16) times the bounds, once per limb: lane l holds page l % 16 and groups 4 (l / 16) + i
    __device__ __forceinline__ void score(const i32x4 (&limb)[2][D / 32], uint32_t (&key)[4]) const {
        i32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) {
            lo = __builtin_amdgcn_mfma_i32_16x16x64_i8(limb[0][kk], b[kk], lo, 0, 0, 0);
            hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(limb[1][kk], b[kk], hi, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) key[i] = ordered((float)(hi[i] * 128 + lo[i]) * scale, there);
    }
};

// Where a wave of a score launch works: the waves of a workgroup are `heads` neighbouring KV heads of the same pages (a page's bounds of all
// heads lie next to each other), then neighbouring pages; a wave takes p.score_tiles tiles of 16 pages.
struct ScorePlace {
    SelectRow r;
    int h, ng, tile, pg0, end;                        // KV head; groups of the row; its tile of 16 groups; the wave's pages
    __device__ __forceinline__ bool find(const SelectParams& p, int heads, int wave) {
        r = row_of<SELECT_MAX_REQS>(p.rows, p.n, blockIdx.x, [](const SelectRow& x) { return x.tile0; });
        const int per_wave = p.score_tiles * 16, per_wg = per_wave * (SCORE_WAVES / heads);
        h = blockIdx.y * heads + wave % heads;
        ng = (r.L + p.g - 1) / p.g;
        const int tiles = (ng + 15) >> 4, at = blockIdx.x - r.tile0, block = at / tiles;
        tile = at - block * tiles;
        // pages that the tile's last group may choose by score
        const int last_group = min(ng, tile * 16 + 16) - 1;
        pg0 = block * per_wg + (wave / heads) * per_wave;
        end = min(pg0 + per_wave, ((r.C + last_group * p.g) >> p.logP) - p.last + 1);
        return h < p.Hkv && pg0 < end;
    }
    __device__ __forceinline__ int64_t stride(const SelectParams& p) const { return (((int64_t)r.C + r.L + p.P - 1) / p.P + 63) / 64 * 64; }
};

// Rows of one group each (decode steps).  A load of 64 lanes takes the bounds of PPI pages of one KV head, a lane 16 of a page's 2d bytes; four
// or eight whole-number dot products of 4 per limb and a sum over the page's lanes make its score.  The wave quantises the row's queries itself,
// while its first pages travel.
template <int D>
__global__ __launch_bounds__(64 * SCORE_WAVES) void row_scores_kernel(const SelectParams p, int heads) {
    constexpr int LPP = RowCodes<D>::LPP, PPI = RowCodes<D>::PPI, NL = 16 / PPI, TB = SCORE_BATCH;   // loads per tile; tiles in flight
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    ScorePlace w;
    if (!w.find(p, heads, wave)) return;
    const int G = p.Hq / p.Hkv, h = w.h, end = w.end;
    const int32_t* bt = p.block_table + (int64_t)w.r.req * p.max_pages;
    // lane's page of a tile: load i = lane % LPP (lanes from NL on: the last load's) brings page i * PPI + lane / LPP to the lane's LPP lanes
    const int mine = min(lane % LPP, NL - 1) * PPI + lane / LPP;
    auto page_id = [&](int first) {
        const int id = bt[min(first + mine, end - 1)];
        return (uint32_t)id < (uint64_t)p.num_pages ? id : -1;
    };
    int id[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) id[t] = page_id(w.pg0 + t * 16);
    RowCodes<D> qc;
    const char* q = static_cast<const char*>(p.q) + ((int64_t)w.r.row_off * p.Hq + h * G) * (D * 2);
    qc.start(q, (int64_t)p.Hq * D * 2, G, w.r.L * G, lane);
    i32x4 limb[2];
    uint32_t* keys = p.keys + (int64_t)w.r.key0 * 64 + h * w.stride(p);
    for (int at = w.pg0; at < end; at += TB * 16) {
        i32x4 b[TB][NL];
        float scale[TB];
        bool there[TB];
#pragma unroll
        for (int t = 0; t < TB; ++t) {
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int page = max(0, __shfl(id[t], (lane & ~(LPP - 1)) + i, 64));
                b[t][i] = *reinterpret_cast<const i32x4*>(p.codes + ((int64_t)page * p.Hkv + h) * (2 * D) + (lane % LPP) * 16);
            }
            scale[t] = p.bscale[(int64_t)max(0, id[t]) * p.Hkv + h];
            there[t] = id[t] >= 0;
        }
#pragma unroll
        for (int t = 0; t < TB; ++t) id[t] = page_id(at + (TB + t) * 16);
        if (at == w.pg0) {                            // uniform
            __builtin_amdgcn_sched_barrier(0);
            qc.finish(q, (int64_t)p.Hq * D * 2, G, w.r.L * G, lane, limb);
        }
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            int n = 0;
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                int lo = 0, hi = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    lo = __builtin_amdgcn_sdot4(limb[0][k], b[t][i][k], lo, false);
                    hi = __builtin_amdgcn_sdot4(limb[1][k], b[t][i][k], hi, false);
                }
                uint32_t s = (uint32_t)(hi * 128 + lo);
                s = add_dpp<0xB1>(s);
                s = add_dpp<0x4E>(s);
                // (the four lanes of a quad hold its sum: a mirrored half row is the other quad, a rotation by 8 the other half)
                s = add_dpp<0x141>(s);                // row_half_mirror
                if constexpr (LPP == 16) s = add_dpp<0x128>(s);           // row_ror:8
                n = i == lane % LPP ? (int)s : n;
            }
            const int page = at + t * 16 + mine;
            if (lane % LPP < NL && page < end) keys[page] = ordered((float)n * scale[t], there[t]);
        }
    }
}

// Scores of 16 groups x 16 pages at a time, SCORE_BATCH tiles in flight at once.  Bound: latency, and the trips of a tile's lines to the CUs.  (Codes,
// scores and choice of 4 groups in one workgroup, the keys in LDS, instead of three launches: 35 us instead of 23 for 64 groups over 2 050 pages,
// since every workgroup then takes all the pages' bounds.)
template <int D>
__global__ __launch_bounds__(64 * SCORE_WAVES) void page_scores_kernel(const SelectParams p, int heads) {
    constexpr int KK = D / 32, TB = SCORE_BATCH;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    ScorePlace w;
    if (!w.find(p, heads, wave)) return;
    const int h = w.h, end = w.end, col = lane & 15, c = lane >> 4;
    const int32_t* bt = p.block_table + (int64_t)w.r.req * p.max_pages;
    int id[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) id[t] = bt[min(w.pg0 + t * 16 + col, end - 1)];
    i32x4 limb[2][KK];
    {
        const int item = w.r.item0 + min(w.tile * 16 + col, w.ng - 1);    // (a group behind the last: the last one's, not stored)
        const int8_t* src = p.qcodes + ((int64_t)item * p.Hkv + h) * (4 * D) + c * 16;
#pragma unroll
        for (int l = 0; l < 2; ++l)
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) limb[l][kk] = *reinterpret_cast<const i32x4*>(src + l * (2 * D) + kk * 64);
    }
    const int64_t stride = w.stride(p);
    uint32_t* keys = p.keys + (int64_t)w.r.key0 * 64 + h * stride;
    for (int at = w.pg0; at < end; at += TB * 16) {
        PageTile<D> b[TB];
#pragma unroll
        for (int t = 0; t < TB; ++t) b[t].load(p, id[t], h, lane);
#pragma unroll
        for (int t = 0; t < TB; ++t) id[t] = bt[min(at + (TB + t) * 16 + col, end - 1)];
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            uint32_t key[4];
            b[t].score(limb, key);
            const int page = at + t * 16 + col;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int g = w.tile * 16 + c * 4 + i;
                if (page < end && g < w.ng) keys[(int64_t)g * p.Hkv * stride + page] = key[i];
            }
        }
    }
}

// What a group chooses from, for any KV head: pages [0, nfirst) and [cend, lp1] always, `need` of the n from cbeg = nfirst on.
struct Choice {
    int nfirst, cend, lp1, n, need;
    __device__ __forceinline__ Choice(const SelectParams& p, const SelectRow& r, int tok0) {
        const int m = min(p.g, r.L - tok0), lp0 = (r.C + tok0) >> p.logP;
        lp1 = (r.C + tok0 + m - 1) >> p.logP;
        nfirst = min(p.first, lp1 + 1);
        cend = max(nfirst, lp0 - p.last + 1);
        n = cend - nfirst;
        need = min(n, p.budget - nfirst - (lp1 + 1 - cend));
    }
    // the part of the list that needs no scores, by thread t of nt
    __device__ __forceinline__ void write_always(int32_t* out, int budget, int t, int nt) const {
        const int total = nfirst + need + lp1 + 1 - cend;
        for (int i = t; i < budget; i += nt) {
            if (i < nfirst) out[i] = i;
            else if (i >= nfirst + need) out[i] = i < total ? cend + i - nfirst - need : -1;
            else if (need == n) out[i] = i;
        }
    }
    __device__ __forceinline__ bool nothing_to_choose() const { return need == n || need == 0; }
};

__device__ __forceinline__ int lanes_below(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); }

// Sums over the lanes up to and with this one.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x, int lane) {
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true);     // row_shr:1, 2, 4, 8
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true);
    const uint32_t a = __builtin_amdgcn_readlane(x, 15), b = __builtin_amdgcn_readlane(x, 31), c = __builtin_amdgcn_readlane(x, 47);
    return x + (lane >= 16 ? a : 0u) + (lane >= 32 ? b : 0u) + (lane >= 48 ? c : 0u);
}

// Of n keys the `need` largest, the lowest index among equals, for one group and KV head, written as page indices in ascending order.
// The keys' range is cut into 512 bins that are counted in LDS; the bin in which the need-th largest lies is cut again until it is chosen
// whole or holds one value.  (Bins of the leading bits would hold nearly everything in one: scores of one row have few exponents.  Bisection
// instead, a count of all keys per step, took 13 to 20 steps and twice as long.)  KPL keys per lane stay in registers; KPL = 0: more keys than that,
// read again in every pass.  A wave holds a run of neighbouring keys, key i of it in lane i % 64.
template <int NW, int KPL>
__global__ __launch_bounds__(64 * NW) void choose_pages_kernel(const SelectParams p) {
    constexpr int BINS = 512, BPL = BINS / 64;
    __shared__ __attribute__((aligned(16))) uint32_t bins[BINS];
    __shared__ uint32_t range[2][NW], counts[2][NW];  // (two: with one value among all keys there is no barrier between them)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int item = blockIdx.x, h = blockIdx.y;
    const SelectRow r = row_of<SELECT_MAX_REQS>(p.rows, p.n, item, [](const SelectRow& x) { return x.item0; });
    const int grp = item - r.item0;
    const Choice ch(p, r, grp * p.g);
    int32_t* out = p.selected + ((int64_t)(r.out0 + grp) * p.Hkv + h) * p.budget;
    const int64_t stride = (((int64_t)r.C + r.L + p.P - 1) / p.P + 63) / 64 * 64;
    const int per = KPL ? KPL : (ch.n + 64 * NW - 1) / (64 * NW);         // keys per lane
    const int i0 = wave * (64 * per), n = min(64 * per, ch.n - i0);       // this wave's first key, and how many it has
    const uint32_t* src = p.keys + (int64_t)r.key0 * 64 + ((int64_t)grp * p.Hkv + h) * stride + ch.nfirst + i0;
    uint32_t reg[KPL ? KPL : 1];
    if constexpr (KPL > 0) {
        if (!ch.nothing_to_choose()) {
#pragma unroll
            for (int i = 0; i < KPL; ++i) reg[i] = i * 64 + lane < n ? src[i * 64 + lane] : 0u;
        }
    }
    ch.write_always(out, p.budget, threadIdx.x, 64 * NW);
    if (ch.nothing_to_choose()) return;               // uniform
    // f(key, place in the wave's run, whether there is one)
    auto each = [&](auto&& f) {
        if constexpr (KPL > 0) {
#pragma unroll
            for (int i = 0; i < KPL; ++i) f(reg[i], i * 64 + lane, i * 64 + lane < n);
        } else {
            for (int i = 0; i < per; ++i) {
                const bool there = i * 64 + lane < n;
                f(there ? src[i * 64 + lane] : 0u, i * 64 + lane, there);
            }
        }
    };
    uint32_t lo = 0xffffffffu, hi = 0;
    each([&](uint32_t k, int, bool there) {
        lo = min(lo, there ? k : 0xffffffffu);
        hi = max(hi, k);
    });
    lo = wave_umin(lo);
    hi = wave_umax(hi);
    if (lane == 0) {
        range[0][wave] = lo;
        range[1][wave] = hi;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        lo = min(lo, range[0][w]);
        hi = max(hi, range[1][w]);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    // keys above hi are chosen, `left` of those in [lo, hi], none below; whole: all in [lo, hi] are
    int left = ch.need;
    bool whole = false;
    for (int pass = 0; pass < 4 && lo < hi && !whole; ++pass) {           // (32 bits: 23, 14, 5 and 0 are left)
        const int shift = max(0, 32 - __clz((int)(hi - lo)) - 9);
        for (int i = threadIdx.x; i < BINS; i += 64 * NW) bins[i] = 0;
        __syncthreads();
        each([&](uint32_t k, int, bool there) {
            if (there && k >= lo && k <= hi) atomicAdd(&bins[(k - lo) >> shift], 1u);
        });
        __syncthreads();
        // every wave: lane l adds up bins BPL l .. from the top
        uint32_t b[BPL];
#pragma unroll
        for (int i = 0; i < BPL; i += 4) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(&bins[BINS - 4 - BPL * lane - i]);
            b[i] = v.w;
            b[i + 1] = v.z;
            b[i + 2] = v.y;
            b[i + 3] = v.x;
        }
        uint32_t sum = 0;
#pragma unroll
        for (int i = 0; i < BPL; ++i) sum += b[i];
        const uint32_t upto = wave_scan(sum, lane);
        uint32_t above = upto - sum;                  // keys in bins above this lane's
        const uint64_t reach = __ballot(upto >= (uint32_t)left);
        const int owner = __builtin_ctzll(reach);     // (the keys in [lo, hi] are `left` or more)
        uint32_t bin = BINS - 1 - BPL * lane, inside = b[0];
#pragma unroll
        for (int i = 1; i < BPL; ++i) {
            const bool on = above + inside < (uint32_t)left;
            above += on ? inside : 0u;
            bin -= on ? 1u : 0u;
            inside = on ? b[i] : inside;
        }
        bin = __builtin_amdgcn_readlane(bin, owner);
        left -= (int)__builtin_amdgcn_readlane(above, owner);
        whole = (int)__builtin_amdgcn_readlane(inside, owner) == left;
        lo += bin << shift;
        hi = lo + min(hi - lo, (1u << shift) - 1);    // (keys reach 2^32 - 1 where a page's scale is no number)
        __syncthreads();                              // before the bins are cleared again
    }
    if (whole) left = ch.n;
    int at = ch.nfirst;
    // what the waves before this one take
    uint32_t above = 0, equal = 0;
    each([&](uint32_t k, int, bool there) {
        above += there && k > hi ? 1u : 0u;
        equal += there && k >= lo && k <= hi ? 1u : 0u;
    });
    above = wave_usum(above);
    equal = wave_usum(equal);
    if (lane == 0) {
        counts[0][wave] = above;
        counts[1][wave] = equal;
    }
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
        const int take = min(left, (int)counts[1][w]);
        at += (int)counts[0][w] + take;
        left -= take;
    }
    each([&](uint32_t k, int i, bool there) {
        const bool equal = there && k >= lo && k <= hi;
        const uint64_t em = __ballot(equal);
        const bool take = (there && k > hi) || (equal && lanes_below(em) < left);
        const uint64_t m = __ballot(take);
        if (take) out[at + lanes_below(m)] = ch.nfirst + i0 + i;
        at += __popcll(m);
        left -= min(left, (int)__popcll(em));
    });
}

// ---------------------------------------------------------------------------------------------
// attention over listed pages

// K/V loader of one wave: blocks of 32 keys, two halves of 16 consecutive slots of a page each (global -> registers -> the wave's LDS region).
// A block's position in the list decides its page; the list entries of the wave's next 8 blocks come with one load, their page ids with
// another that is made a block later, so that neither is waited for.
// ONCE: every page is read by one group (rows of one group each): loads that leave no lines behind (96 rows of 128 pages: 144 -> 130 us).  Lists of
// neighbouring groups share pages, and their lines (64 groups of one row: 42 us, 48 so, when their probabilities went in one part).
template <int D, int KVT, bool ONCE>
struct ListLoader {
    using G_ = Geo<D>;
    using T = LanePlace<D, KVT, 1>;
    static constexpr int ES = T::ES;
    static constexpr int KPL = 1024 / (D * ES);       // keys per load
    static constexpr int LPH = 16 / KPL;              // loads per half block
    static constexpr int NL = 2 * LPH;
    static constexpr int IDS = 8;
    RawChunk<KVT> k[NL], v[NL];
    int entry, page;                                  // lane 2 n + h: list entry (-1: none) and page (-1: none) of half h of block n of eight
    int next;                                         // entries of the eight blocks that follow
    int first[2];                                     // of the block that was fetched last: position of each half's first key (NONE: no page)
    int at[2];                                        // ... of the block that is committed
    float scale[4], sc[4];
    static constexpr int NONE = 0x7fff0000;            // (positions end before 2^30; a block's keys, and differences of positions, stay in 32 bits)

    __device__ __forceinline__ void fetch_entries(const SparseParams& p, const int32_t* list, int key0, int step, int end, int j, int lane) {
        const int pos = key0 + (j + (lane >> 1) % IDS) * step + (lane & 1) * 16;
        next = -1;
        if (pos < end) next = list[pos >> p.logP];
    }
    __device__ __forceinline__ void fetch_pages(const SparseParams& p, const int32_t* bt, int last_page) {
        entry = next <= last_page ? next : -1;
        int id = -1;
        if (entry >= 0) id = bt[entry];
        page = (uint32_t)id < (uint64_t)p.num_pages ? id : -1;
    }
    // Block j of the wave (the j-th of its eight); false: neither half has a page, and nothing is fetched.
    __device__ __forceinline__ bool fetch(const SparseParams& p, int kvh, int pos, int j, int lane) {
        int64_t off[2];
        int id[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            id[h] = __builtin_amdgcn_readlane(page, 2 * (j % IDS) + h);
            const int slot = (pos + 16 * h) & (p.P - 1);
            first[h] = id[h] < 0 ? NONE : (__builtin_amdgcn_readlane(entry, 2 * (j % IDS) + h) << p.logP) + slot;
            off[h] = slot * (D * ES);
        }
        if (id[0] < 0 && id[1] < 0) return false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int use = id[h] < 0 ? id[1 - h] : id[h];        // (a half without a page: any slots of the other's, not used)
            const int64_t ph = (int64_t)use * p.Hkv + kvh;
            if constexpr (KVT == KV_FP8) {
                scale[h] = p.k_scale[ph];
                scale[2 + h] = p.v_scale[ph];
            }
            off[h] += (ph << p.logP) * (D * ES);
        }
        uint32_t lo = T::lane_off(lane);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const GlobalBytes ka = scalar_base(static_cast<const char*>(p.k_pool) + off[h]), va = scalar_base(static_cast<const char*>(p.v_pool) + off[h]);
            asm("" : "+v"(lo));
#pragma unroll
            for (int i = 0; i < LPH; ++i) {
                k[h * LPH + i].v = ONCE ? __builtin_nontemporal_load((GlobalChunk)(ka + i * 1024 + lo)) : *(GlobalChunk)(ka + i * 1024 + lo);
                v[h * LPH + i].v = ONCE ? __builtin_nontemporal_load((GlobalChunk)(va + i * 1024 + lo)) : *(GlobalChunk)(va + i * 1024 + lo);
            }
        }
        return true;
    }
    // To LDS; V rows that no row of the item sees become zeros, so that 0-weights never meet NaN garbage (K's logits are replaced).
    __device__ __forceinline__ void commit(uint32_t kl, uint32_t vl, int last_lim, int lane) {
#pragma unroll
        for (int l = 0; l < 4; ++l) sc[l] = KVT == KV_FP8 ? scale[l] : 1.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            at[h] = first[h];
            if (at[h] + 15 > last_lim) {              // uniform
#pragma unroll
                for (int i = 0; i < LPH; ++i)
                    if (at[h] + i * KPL + T::lane_key(lane) > last_lim) v[h * LPH + i].zero();
            }
        }
#pragma unroll
        for (int n = 0; n < NL; ++n) {
            T::put(k[n], sc[n / LPH], kl + T::slot_of(0, lane) + n * (T::GPP * G_::GS));
            T::put(v[n], sc[2 + n / LPH], vl + T::slot_of(0, lane) + n * (T::GPP * G_::GS));
        }
    }
};

// A lane's N probabilities 2^(S c - m) of a block as two bf16 parts each, the leading bits and the rest, together within 2^-15 of the probability.
// Returns their sum in fp32.  (Cutting the first part instead of rounding it: 41.2 us instead of 41.8 for 64 groups of 32 rows.)
template <int N, class Logit, class Prob>
__device__ __forceinline__ float exp_sum_parts(float c, float m_use, Logit&& S, Prob&& P) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = fast_exp2(__builtin_fmaf(S(i), c, -m_use));
        const uint32_t high = __float_as_uint(x) >> 16;
        sum += x;
        P(i, 0, __builtin_bit_cast(__bf16, (uint16_t)high));
        P(i, 1, (__bf16)(x - __uint_as_float(high << 16)));
    }
    return sum;
}

// What an item of sparse attention is about.
struct SparseItem {
    int kvh, G, rows;                                 // rows of this tile: row r is row r0 + r of the group, token / G
    int r0, tok0, C, row_off;
    int piece, tile, linear;
    int group;                                        // of the launch
    int req;
};
// Workgroups in launch order: KV head first (neighbouring workgroups run on different dies; a head's groups share lines on one die where the heads
// are as many), then piece, row tile, group.
__device__ __forceinline__ void sparse_place(const SparseParams& p, int b, SparseItem& it) {
    it.linear = b;
    it.kvh = b % p.Hkv;
    b /= p.Hkv;
    it.piece = b % p.splits;
    b /= p.splits;
    it.tile = b % p.tiles;
    it.group = b / p.tiles;
}
__device__ __forceinline__ bool sparse_item(const SparseParams& p, int ROWS, SparseItem& it) {
    const SparseRow r = row_of<SPARSE_MAX_REQS>(p.rows, p.n, it.group, [](const SparseRow& x) { return x.first; });
    it.req = r.req;
    it.G = p.Hq / p.Hkv;
    it.tok0 = (it.group - r.first) * p.g;
    it.C = r.C;
    it.row_off = r.row_off;
    it.r0 = it.tile * ROWS;
    it.rows = min(ROWS, min(p.g, r.L - it.tok0) * it.G - it.r0);
    return it.rows > 0;
}

template <int D, int NW, int ROWS>
constexpr int sparse_smem() {
    const int stage = NW * 2 * Geo<D>::B32, merge = NW * ROWS * (D + 4) * 4 + NW * ROWS * 8;
    return stage > merge ? stage : merge;
}

// An item: the rows of a group (tokens x heads of a KV head, ROWS at a time) over a piece of the group's list.  The waves take the piece's
// blocks of 32 keys in turn, each with a softmax state and an LDS region of its own, and the states are merged at the end.
// Logits, running maximum, sum and output are held in 32 bits; the matrix cores take the probabilities of the second product in 16 bits, so they
// go in two parts, one after the other over the same V operand (one part, rounded to bf16: 38 us instead of 41 for 64 groups of 32 rows, 129.4 instead of
// 130.0 for 96 rows, and outputs 0.0021 off their 64-bit values, relative, instead of 0.0017, which is the rounding of the output alone).
// Bound: memory where every list is another's (96 rows x 8 heads over 128 pages of 16, 809 MB in 130 us = 6.2 TB/s); LDS, through which K and V
// pass on their way into the operands' layout, and the products, where 32 rows share a list that is in L2 (64 groups by the trace: 45 us, on pages that
// never leave L2 42, without its products 32, without its loads 38, without what it writes to LDS 38; two waves a SIMD.  K loaded straight in
// the layout of a 32x32x16 or two 16x16x32 products, quarter or half lines at a time, took 52 and 50 where this took 42).  A group of more rows
// goes as tiles of 32 that stage its list again each (64 groups of 64 rows 80 us, 32 of 128 rows 78).
template <int D, int KVT, int ROWS, int NW, bool ONCE>
__global__ __launch_bounds__(64 * NW, 2) void sparse_rows_kernel(const SparseParams p) {
    using G_ = Geo<D>;
    constexpr bool R16 = ROWS == 16;
    __shared__ __attribute__((aligned(16))) char smem_raw[sparse_smem<D, NW, ROWS>()];
    const uint32_t smem = (uint32_t)(uintptr_t)LDS_PTR(char, smem_raw);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (the first list entries before the row they belong to is known)
    SparseItem it;
    sparse_place(p, blockIdx.x, it);
    const int begin = it.piece * p.chunk, end = min(p.budget << p.logP, begin + p.chunk);
    const int nblocks = (end - begin + 31) >> 5, step = 32 * NW, key0 = begin + wave * 32;
    const int nj = (nblocks - wave + NW - 1) / NW;
    const int32_t* list = p.selected + ((int64_t)it.group * p.Hkv + it.kvh) * p.budget;
    ListLoader<D, KVT, ONCE> ld;
    if (nj > 0) ld.fetch_entries(p, list, key0, step, end, 0, lane);
    if (!sparse_item(p, ROWS, it)) return;
    const int row = lane & (ROWS - 1);
    const bool valid = row < it.rows;
    const int gr = it.r0 + min(row, it.rows - 1), tok = it.tok0 + gr / it.G;
    const int lim = it.C + tok;                                           // last visible position
    const int first_lim = it.C + it.tok0 + it.r0 / it.G, last_lim = it.C + it.tok0 + (it.r0 + it.rows - 1) / it.G;
    const int last_page = last_lim >> p.logP;
    const int32_t* bt = p.block_table + (int64_t)it.req * p.max_pages;
    bf16x8 Q[R16 ? D / 32 : G_::NKK];
    {
        const int hq = it.kvh * it.G + gr % it.G, g = lane / ROWS;
        const char* src = static_cast<const char*>(p.q) + (((int64_t)(it.row_off + tok) * p.Hq + hq) * D + g * 8) * 2;
#pragma unroll
        for (int kk = 0; kk < (R16 ? D / 32 : G_::NKK); ++kk)
            Q[kk] = __builtin_bit_cast(bf16x8, valid ? *reinterpret_cast<const u32x4*>(src + kk * (R16 ? 64 : 32)) : u32x4{0, 0, 0, 0});
    }
    std::conditional_t<R16, WaveAcc16<D>, WaveAcc<D>> st;
    if constexpr (R16) {
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st.O[dt] = f32x4{0, 0, 0, 0};
    } else {
#pragma unroll
        for (int db = 0; db < G_::NDB; ++db) st.O[db] = f32x16{0};
    }
    st.m = NEG_INF;
    st.l = 0.0f;

    const uint32_t kl = smem + wave * (2 * G_::B32), vl = kl + G_::B32;
    bool have = false;
    if (nj > 0) {
        ld.fetch_pages(p, bt, last_page);
        have = ld.fetch(p, it.kvh, key0, 0, lane);
    }
    for (int j = 0; j < nj; ++j) {
        const bool now = have;                                            // uniform
        if (now) ld.commit(kl, vl, last_lim, lane);
        if (j + 1 < nj) {
            if ((j + 1) % ld.IDS == 0) ld.fetch_pages(p, bt, last_page);
            have = ld.fetch(p, it.kvh, key0 + (j + 1) * step, j + 1, lane);
            if ((j + 1) % ld.IDS == ld.IDS - 1) ld.fetch_entries(p, list, key0, step, end, j + 2, lane);
        }
        if (!now) continue;
        const bool masked = max(ld.at[0], ld.at[1]) + 15 > first_lim;
        const int sub = R16 ? 4 * key_group16(lane >> 4) : 4 * (lane >> 5);
        const int rel0 = lim - ld.at[0] - sub, rel1 = lim - ld.at[1] - sub;
        if constexpr (R16) {
            f32x4 S[2];
            qk16<D>(kl, Q, S, lane);
            if (masked) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    S[0][i] = i <= rel0 ? S[0][i] : NEG_INF;
                    S[1][i] = i <= rel1 ? S[1][i] : NEG_INF;
                }
            }
            float mx = fmaxf(fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3])), fmaxf(fmaxf(S[1][0], S[1][1]), fmaxf(S[1][2], S[1][3])));
            mx = max_xor32(max_xor16(mx)) * p.c_log2;
            if (__any(mx > st.m + RESCALE_SLACK)) raise_reference16<D>(st, mx);
            bf16x8 P[2];
            st.l += exp_sum_parts<8>(p.c_log2, st.m == NEG_INF ? 0.0f : st.m, [&](int i) { return S[i >> 2][i & 3]; }, [&](int i, int part, __bf16 v) { P[part][i] = v; });
            pv16_parts<D, 2>(vl, P, st, lane);
        } else {
            // a wave that has begun a block's products goes first: 64 groups of 32 rows over 128 pages 42.8 -> 41.9 us (LDS is what it waits for)
            __builtin_amdgcn_s_setprio(1);
            f32x16 S;
            bf16x8 P[2][2];
            qk32<D>(kl, Q, S, lane);
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int koff = ((i >> 2) & 1) * 8 + (i & 3);
                    S[i] = koff <= (i < 8 ? rel0 : rel1) ? S[i] : NEG_INF;
                }
            }
            const float mx = rowmax32(S) * p.c_log2;
            if (__any(mx > st.m + RESCALE_SLACK)) raise_reference<D>(st, mx);
            st.l += exp_sum_parts<16>(p.c_log2, st.m == NEG_INF ? 0.0f : st.m, [&](int i) { return S[i]; }, [&](int i, int part, __bf16 v) { P[part][i >> 3][i & 7] = v; });
            pv32_parts<D, 2>(vl, P, st, lane);
            __builtin_amdgcn_s_setprio(0);
        }
    }
    // merge the waves' states: LDS holds O as [state][row][D + 4] fp32 and (m, l) as [state][row][2]
    __syncthreads();                                      // every wave is done with its K/V region
    constexpr int OSTR = D + 4;
    const uint32_t mlbase = smem + NW * ROWS * OSTR * 4;
    {
        const int g = lane / ROWS, slot = wave * ROWS + row;
        const uint32_t orow = smem + slot * OSTR * 4;
        const float ltot = R16 ? sum_xor32(sum_xor16(st.l)) : sum_xor32(st.l);
        if constexpr (R16) {
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) *LDS_PTR(f32x4, orow + (dt * 16 + g * 4) * 4) = st.O[dt];
        } else {
#pragma unroll
            for (int db = 0; db < G_::NDB; ++db)
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) {
                    f32x4 o = {st.O[db][i4 * 4], st.O[db][i4 * 4 + 1], st.O[db][i4 * 4 + 2], st.O[db][i4 * 4 + 3]};
                    *LDS_PTR(f32x4, orow + (db * 32 + i4 * 8 + g * 4) * 4) = o;
                }
        }
        if (g == 0) {
            *LDS_PTR(float, mlbase + slot * 8) = st.m;
            *LDS_PTR(float, mlbase + slot * 8 + 4) = ltot;
        }
    }
    __syncthreads();
    // thread -> (row r, DPT consecutive d): 16 threads per row
    constexpr int DPT = D / 16;
    const int dc = (tid & 15) * DPT;
    for (int r = tid >> 4; r < it.rows; r += 4 * NW) {
        float mw[NW], lw[NW], mall = NEG_INF;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            mw[w] = *LDS_PTR(float, mlbase + (w * ROWS + r) * 8);
            lw[w] = *LDS_PTR(float, mlbase + (w * ROWS + r) * 8 + 4);
            mall = fmaxf(mall, mw[w]);
        }
        const float muse = mall == NEG_INF ? 0.0f : mall;
        float lsum = 0.0f, acc[DPT];
#pragma unroll
        for (int x = 0; x < DPT; ++x) acc[x] = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float wgt = fast_exp2(mw[w] - muse);
            lsum += lw[w] * wgt;
            const uint32_t src = smem + ((w * ROWS + r) * OSTR + dc) * 4;
#pragma unroll
            for (int x = 0; x < DPT; x += 4) {
                const f32x4 o = *LDS_PTR(f32x4, src + x * 4);
                acc[x] += o[0] * wgt;
                acc[x + 1] += o[1] * wgt;
                acc[x + 2] += o[2] * wgt;
                acc[x + 3] += o[3] * wgt;
            }
        }
        if (p.splits == 1) {
            const float inv = lsum > 0.0f ? 1.0f / lsum : 0.0f;           // a row that sees no key: zeros
            const int t = (it.r0 + r) / it.G, hq = it.kvh * it.G + (it.r0 + r) - t * it.G;
            char* dst = static_cast<char*>(p.out) + (((int64_t)(it.row_off + it.tok0 + t) * p.Hq + hq) * D + dc) * 2;
#pragma unroll
            for (int x = 0; x < DPT; x += 4) {
                bf16x4 o = {(__bf16)(acc[x] * inv), (__bf16)(acc[x + 1] * inv), (__bf16)(acc[x + 2] * inv), (__bf16)(acc[x + 3] * inv)};
                *reinterpret_cast<u32x2*>(dst + x * 2) = __builtin_bit_cast(u32x2, o);
            }
        } else {
            float* po = p.partial + (int64_t)it.linear * (ROWS * (D + 2)) + r * D + dc;
#pragma unroll
            for (int x = 0; x < DPT; x += 4) *reinterpret_cast<f32x4*>(po + x) = f32x4{acc[x], acc[x + 1], acc[x + 2], acc[x + 3]};
            if ((tid & 15) == 0) {
                float* ml = p.partial + (int64_t)it.linear * (ROWS * (D + 2)) + ROWS * D + r * 2;
                ml[0] = mall;
                ml[1] = lsum;
            }
        }
    }
}

// Merge the pieces of a list: one workgroup per (group, row tile, KV head) and pass of WG / (D / 4) rows.  Up to UN pieces are on their way before
// the row they belong to is known (rows that a tile does not have are read too, and dropped).
template <int D, int ROWS>
__global__ __launch_bounds__(WG) void sparse_join_kernel(const SparseParams p) {
    constexpr int QPR = D / 4, RPP = WG / QPR, UN = 16;
    SparseItem it;
    const int b = blockIdx.x, kvh = b % p.Hkv;
    sparse_place(p, (b / p.Hkv) * p.splits * p.Hkv + kvh, it);
    const int r = blockIdx.y * RPP + threadIdx.x / QPR, dq = (threadIdx.x % QPR) * 4;
    const int64_t stride = (int64_t)p.Hkv * (ROWS * (D + 2));             // from piece to piece
    const float* base = p.partial + (int64_t)it.linear * (ROWS * (D + 2));
    float m = NEG_INF, l = 0.0f;
    f32x4 acc = {0, 0, 0, 0};
    float mv[UN], lv[UN];
    f32x4 ov[UN];
    auto fetch = [&](int s0) {
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const float* part = base + min(s0 + i, p.splits - 1) * stride;
            mv[i] = part[ROWS * D + r * 2];
            lv[i] = part[ROWS * D + r * 2 + 1];
            ov[i] = *reinterpret_cast<const f32x4*>(part + r * D + dq);
        }
    };
    fetch(0);
    const bool there = sparse_item(p, ROWS, it) && r < it.rows;
    for (int s0 = 0; s0 < p.splits; s0 += UN) {
        if (s0 > 0) fetch(s0);
        float mg = m;
#pragma unroll
        for (int i = 0; i < UN; ++i) mg = fmaxf(mg, mv[i]);
        const float muse = mg == NEG_INF ? 0.0f : mg, back = fast_exp2(m - muse);
        l *= back;
        acc *= back;
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            if (s0 + i < p.splits) {
                const float w = fast_exp2(mv[i] - muse);
                l += lv[i] * w;
                acc += ov[i] * w;
            }
        }
        m = mg;
    }
    if (!there) return;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    const int t = (it.r0 + r) / it.G, hq = it.kvh * it.G + (it.r0 + r) - t * it.G;
    char* dst = static_cast<char*>(p.out) + (((int64_t)(it.row_off + it.tok0 + t) * p.Hq + hq) * D + dq) * 2;
    bf16x4 o = {(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv), (__bf16)(acc[3] * inv)};
    *reinterpret_cast<u32x2*>(dst) = __builtin_bit_cast(u32x2, o);
}

// ---------------------------------------------------------------------------------------------
// launchers

constexpr int64_t MAX_PAGES = 1 << 22;                // pages per launch (a grid holds fewer than 2^32 threads)

template <int D, int P, int KVT>
static void rope_t(const RopeParams& p, unsigned nx, unsigned ny, hipStream_t st) {
    if (p.codes)
        hipLaunchKernelGGL((rope_append_kernel<D, P, KVT, true>), dim3(nx, ny), dim3(WG), 0, st, p);
    else
        hipLaunchKernelGGL((rope_append_kernel<D, P, KVT, false>), dim3(nx, ny), dim3(WG), 0, st, p);
}
template <int D, int KVT>
static void rope_p(const RopeParams& p, unsigned nx, unsigned ny, hipStream_t st) {
    if (p.a.P == 16) rope_t<D, 16, KVT>(p, nx, ny, st);
    else if (p.a.P == 32) rope_t<D, 32, KVT>(p, nx, ny, st);
    else rope_t<D, 64, KVT>(p, nx, ny, st);
}

// max_new: the most new tokens of a page
hipError_t launch_rope(RopeParams& p, int kvt, int64_t pages, int max_new, hipStream_t st) {
    const int64_t jobs = 2 * p.a.Hkv + (p.q ? ((int64_t)max_new * p.Hq * (p.a.D / 16) + 255) / 256 : 0);
    // a wave per job while that fills the chip; in long launches fewer waves share a page's jobs, and its angles, evenly
    const int64_t least = std::min((jobs + 3) / 4, std::max<int64_t>(1, 2048 / pages)), each = std::max<int64_t>(1, jobs / (4 * least));
    const int64_t ny = (jobs + 4 * each - 1) / (4 * each);
    for (int64_t at = 0; at < pages; at += MAX_PAGES) {
        p.a.pg0 = (int32_t)at;
        const unsigned nx = (unsigned)std::min(MAX_PAGES, pages - at);
        if (p.a.D == 128) {
            if (kvt == KV_BF16) rope_p<128, KV_BF16>(p, nx, (unsigned)ny, st);
            else rope_p<128, KV_FP8>(p, nx, (unsigned)ny, st);
        } else {
            if (kvt == KV_BF16) rope_p<64, KV_BF16>(p, nx, (unsigned)ny, st);
            else rope_p<64, KV_FP8>(p, nx, (unsigned)ny, st);
        }
    }
    return hipGetLastError();
}

template <int D, int P, int KVT>
static void bounds_t(const BoundsParams& p, unsigned nx, hipStream_t st) {
    hipLaunchKernelGGL((page_bounds_kernel<D, P, KVT>), dim3(nx, (p.a.Hkv + 3) / 4), dim3(WG), 0, st, p);
}
template <int D, int KVT>
static void bounds_p(const BoundsParams& p, unsigned nx, hipStream_t st) {
    if (p.a.P == 16) bounds_t<D, 16, KVT>(p, nx, st);
    else if (p.a.P == 32) bounds_t<D, 32, KVT>(p, nx, st);
    else bounds_t<D, 64, KVT>(p, nx, st);
}

hipError_t launch_bounds(BoundsParams& p, int kvt, int64_t pages, hipStream_t st) {
    for (int64_t at = 0; at < pages; at += MAX_PAGES) {
        p.a.pg0 = (int32_t)at;
        const unsigned nx = (unsigned)std::min(MAX_PAGES, pages - at);
        if (p.a.D == 128) {
            if (kvt == KV_BF16) bounds_p<128, KV_BF16>(p, nx, st);
            else bounds_p<128, KV_FP8>(p, nx, st);
        } else {
            if (kvt == KV_BF16) bounds_p<64, KV_BF16>(p, nx, st);
            else bounds_p<64, KV_FP8>(p, nx, st);
        }
    }
    return hipGetLastError();
}

template <int D>
static void select_t(const SelectParams& p, int groups, int score_blocks, bool codes, int64_t max_keys, hipStream_t st) {
    if (score_blocks > 0) {
        const int heads = score_heads(p.Hkv);
        const dim3 grid(score_blocks, (p.Hkv + heads - 1) / heads);
        if (!codes) {
            hipLaunchKernelGGL((row_scores_kernel<D>), grid, dim3(64 * SCORE_WAVES), 0, st, p, heads);
        } else {
            hipLaunchKernelGGL((query_codes_kernel<D>), dim3(groups, p.Hkv), dim3(64), 0, st, p);
            hipLaunchKernelGGL((page_scores_kernel<D>), grid, dim3(64 * SCORE_WAVES), 0, st, p, heads);
        }
    }
    const dim3 grid(groups, p.Hkv);
    // As few waves as hold the keys in a few registers each: they meet at barriers.  (768 choices of 128 to 1 024 pages: a wave alone with 16 keys a lane
    // 7.6 us, 4 waves with 4 6.7; 512 of 2 050: 8 waves with 8 8.4, 12 with 3 8.8, 4 with 9 7.1.)
    if (max_keys <= 4 * 64 * 4) hipLaunchKernelGGL((choose_pages_kernel<4, 4>), grid, dim3(256), 0, st, p);
    else if (max_keys <= 4 * 64 * 10) hipLaunchKernelGGL((choose_pages_kernel<4, 10>), grid, dim3(256), 0, st, p);
    else if (max_keys <= 8 * 64 * 8) hipLaunchKernelGGL((choose_pages_kernel<8, 8>), grid, dim3(512), 0, st, p);
    else if (max_keys <= 16 * 64 * 16) hipLaunchKernelGGL((choose_pages_kernel<16, 16>), grid, dim3(1024), 0, st, p);
    else hipLaunchKernelGGL((choose_pages_kernel<16, 0>), grid, dim3(1024), 0, st, p);
}

// groups: of this launch; score_blocks: workgroup columns of the score launch (0: every group takes all its pages); codes: some row has more
// than one group; max_keys: the most pages a group chooses from
hipError_t launch_select(const SelectParams& p, int D, int groups, int score_blocks, bool codes, int64_t max_keys, hipStream_t st) {
    if (D == 128) select_t<128>(p, groups, score_blocks, codes, max_keys, st);
    else select_t<64>(p, groups, score_blocks, codes, max_keys, st);
    return hipGetLastError();
}

template <int D, int KVT, int ROWS, bool ONCE>
static void sparse_t(const SparseParams& p, int groups, int waves, hipStream_t st) {
    const int64_t items = (int64_t)groups * p.tiles * p.Hkv;
    const dim3 grid((unsigned)(items * p.splits));
    if (waves == 8) hipLaunchKernelGGL((sparse_rows_kernel<D, KVT, ROWS, 8, ONCE>), grid, dim3(512), 0, st, p);
    else hipLaunchKernelGGL((sparse_rows_kernel<D, KVT, ROWS, 4, ONCE>), grid, dim3(256), 0, st, p);
    if (p.splits > 1) hipLaunchKernelGGL((sparse_join_kernel<D, ROWS>), dim3((unsigned)items, ROWS * D / 4 / WG), dim3(WG), 0, st, p);
}
template <int D, int KVT>
static void sparse_k(const SparseParams& p, int groups, int waves, hipStream_t st) {
    const int rows = p.g * (p.Hq / p.Hkv);
    bool once = rows <= sparse_tile(rows);
    for (int i = 0; i < p.n; ++i) once &= p.rows[i].L <= p.g;
    if (sparse_tile(rows) == 16) {
        if (once) sparse_t<D, KVT, 16, true>(p, groups, waves, st);
        else sparse_t<D, KVT, 16, false>(p, groups, waves, st);
    } else {
        if (once) sparse_t<D, KVT, 32, true>(p, groups, waves, st);
        else sparse_t<D, KVT, 32, false>(p, groups, waves, st);
    }
}

hipError_t launch_sparse(const SparseParams& p, int D, int kvt, int groups, int waves, hipStream_t st) {
    if (D == 128) {
        if (kvt == KV_BF16) sparse_k<128, KV_BF16>(p, groups, waves, st);
        else sparse_k<128, KV_FP8>(p, groups, waves, st);
    } else {
        if (kvt == KV_BF16) sparse_k<64, KV_BF16>(p, groups, waves, st);
        else sparse_k<64, KV_FP8>(p, groups, waves, st);
    }
    return hipGetLastError();
}

}  // namespace ampd
