// What the attention and cache kernels for gfx950 are built from: vector types, the LDS layout of a K/V tile, the steps of one block
// of 32 keys (products on the matrix cores and the softmax between them), the lane's place in a K/V load, and the encoding of 8-bit
// pages.  kernels.hip begins with the formulation these steps follow.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernels.h"

namespace ampd {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

#define LDS_PTR(T, p) ((__attribute__((address_space(3))) T*)(uintptr_t)(p))
typedef const __attribute__((address_space(1))) char* GlobalBytes;
typedef const __attribute__((address_space(1))) u32x4* GlobalChunk;

constexpr int WG = 256;                 // append / combine kernels
constexpr int AWG = 64 * ATTN_WAVES;    // attention kernel: 8 waves, one workgroup per CU
constexpr int KT = 128;                 // keys per LDS stage of a wide item (one barrier per stage)
constexpr int NSTAGE = 2;               // LDS ring of K/V stages for wide items
constexpr float NEG_INF = -__builtin_inff();

template <int D>
struct Geo {
    static constexpr int CPK = D / 8;                  // 16-byte (8-element) chunks per key row
    static constexpr int KPW = 64 / CPK;               // keys per group (one wave-wide load)
    static constexpr int GS = 1024 + 16;               // LDS bytes per group
    static constexpr int B32 = (32 / KPW) * GS;        // bytes of a 32-key block (K or V)
    static constexpr int KTILE = (KT / 32) * B32;      // bytes of KT keys (K or V)
    static constexpr int WIDE_STAGE = 2 * KTILE;       // KT keys of K, then KT keys of V
    static constexpr int MERGE = ATTN_WAVES * 32 * (D + 4) * 4 + ATTN_WAVES * 32 * 2 * 4;   // narrow items: waves x (O, m, l)
    static constexpr int NARROW = ATTN_WAVES * 2 * B32;                // one private 32-key K+V block per wave
    static constexpr int SMEM0 = NSTAGE * WIDE_STAGE > MERGE ? NSTAGE * WIDE_STAGE : MERGE;
    static constexpr int SMEM = SMEM0 > NARROW ? SMEM0 : NARROW;
    static constexpr int NDB = D / 32;                 // 32-row blocks of O^T
    static constexpr int NKK = D / 16;                 // MFMA k-steps of the first product
};

// ---------------------------------------------------------------------------------------------
// small helpers

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Exchange with lane^32 folded into the reduction: v_permlane32_swap(x, x) returns
// r0 = {x[0..31], x[0..31]} and r1 = {x[32..63], x[32..63]} (by destination lane halves), so
// op(r0, r1) is op(x[l], x[l^32]) in every lane.
__device__ __forceinline__ float max_xor32(float x) {
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_xor32(float x) {
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A wave-uniform global address in scalar registers.
__device__ __forceinline__ GlobalBytes scalar_base(const char* p) {
    const uint64_t a = (uint64_t)p;
    return (GlobalBytes)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a));
}

// 8 stored elements -> 8 bf16 (as a 16-byte vector) for LDS.
template <int KVT>
struct RawChunk;
template <>
struct RawChunk<KV_BF16> {
    u32x4 v;
    static constexpr int ES = 2;                      // bytes per stored element
    __device__ __forceinline__ void zero() { v = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ void load(const char* base, uint32_t lane_off) {
        v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(base + lane_off));   // streamed: see BlockLoader
    }
    __device__ __forceinline__ u32x4 widen(float) const { return v; }
};
template <>
struct RawChunk<KV_FP8> {
    u32x4 v;                                          // 16 codes: two neighbouring chunks of one key row
    static constexpr int ES = 1;
    __device__ __forceinline__ void zero() { v = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ void load(const char* base, uint32_t lane_off) {
        v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(base + lane_off));
    }
    // decode(code) * scale is exact in bf16: 4 significant bits times a power of two.  The page scales are
    // powers of two (the append kernel writes no others), so the hardware's scaled conversion, which applies
    // the exponent of `scale` only, is that product: one instruction per two elements.
    __device__ __forceinline__ static u32x4 widen8(uint32_t lo, uint32_t hi, float scale) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
        const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
        const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
        return u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
                     __builtin_bit_cast(uint32_t, d)};
    }
    __device__ __forceinline__ u32x4 widen_first(float scale) const { return widen8(v.x, v.y, scale); }
    __device__ __forceinline__ u32x4 widen_second(float scale) const { return widen8(v.z, v.w, scale); }
};

// Per-lane state of one wave: 32 query rows (lane % 32), O^T as D/32 accumulator blocks.
// m is a *reference* maximum in the log2 domain (scale * log2(e) folded in), not the exact
// running maximum: it is raised (and O, l rescaled) only when probabilities against it would grow too large:
// narrow items raise it when a block maximum exceeds it by more than RESCALE_SLACK (probabilities stay below
// 2^RESCALE_SLACK); wide items when a lane's 16 probabilities of a block sum to more than PSUM_LIMIT.
// (m, l, O) remain a consistent triple, which is all the final normalisation and the split-KV
// merge need.
template <int D>
struct WaveAcc {
    f32x16 O[Geo<D>::NDB];
    float m;
    float l;      // this lane's share of the running sum (lanes l and l^32 hold halves)
};
constexpr float RESCALE_SLACK = 8.0f;
constexpr float PSUM_LIMIT = 4096.0f;

// ---------------------------------------------------------------------------------------------
// the steps of one 32-key block

// S^T = K Q^T for the 32 keys whose LDS tile starts at kl.
template <int D>
__device__ __forceinline__ void qk32(uint32_t kl, const bf16x8 (&Q)[Geo<D>::NKK], f32x16& S, int lane) {
    using G_ = Geo<D>;
    const int r = lane & 31, g = lane >> 5;
    // chunk 2*kk + g of key r
    const uint32_t ka = kl + (r / G_::KPW) * G_::GS + (r % G_::KPW) * 64 + g * 16;
    S = f32x16{0};
#pragma unroll
    for (int kk = 0; kk < G_::NKK; ++kk) {
        const u32x4 raw = *LDS_PTR(const u32x4, ka + (kk >> 1) * (G_::KPW * 64) + (kk & 1) * 32);
        S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, raw), Q[kk], S, 0, 0, 0);
    }
}

// rel: per lane, (last visible key of this lane's query) - (first key of the block) - 4*(lane/32)
__device__ __forceinline__ void mask32(f32x16& S, int rel) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int koff = (i >> 2) * 8 + (i & 3);
        S[i] = koff <= rel ? S[i] : NEG_INF;
    }
}

__device__ __forceinline__ float rowmax32(const f32x16& S) {
    float mx = S[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, S[i]);
    return max_xor32(mx);
}

// Raise the reference maximum to cover mx (log2 domain) and rescale O and l.
template <int D>
__device__ __forceinline__ void raise_reference(WaveAcc<D>& st, float mx) {
    const float m_new = fmaxf(st.m, mx);
    const float alpha = fast_exp2(st.m - (m_new == NEG_INF ? 0.0f : m_new));
    st.l *= alpha;
#pragma unroll
    for (int db = 0; db < Geo<D>::NDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.O[db][i] *= alpha;
    st.m = m_new;
}

// p = 2^(S*c - m); returns psum + this lane's sum over the ROUNDED probabilities, two per instruction (dot product of a bf16 pair with
// (1, 1) accumulated in fp32), which is also what the second product adds up; P = bf16(p) as the two B operands.  The rule of prefill rows:
// tiles, and blocks that take a tile's place (see ItemCtx::rounded).
__device__ __forceinline__ float exp32_dot(const f32x16& S, float c, float m_use, bf16x8 (&P)[2], float psum) {
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const bf16x2 pr = {(__bf16)fast_exp2(__builtin_fmaf(S[i], c, -m_use)), (__bf16)fast_exp2(__builtin_fmaf(S[i + 1], c, -m_use))};
        psum = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, psum, false);
        P[i >> 3][i & 7] = pr[0];
        P[i >> 3][(i + 1) & 7] = pr[1];
    }
    return psum;
}

// The same for a lane of a narrow item with its N logits in S: the sum is taken over the rounded probabilities where `rounded`
// (uniform) says so, over the fp32 ones otherwise.  Both sums are taken: a branch would keep the reads of V from moving up past it.
template <int N, class Logit, class Prob>
__device__ __forceinline__ float exp_sum(float c, float m_use, bool rounded, Logit&& S, Prob&& P) {
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
    float sum = 0.0f, rounded_sum = 0.0f;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float p0 = fast_exp2(__builtin_fmaf(S(i), c, -m_use)), p1 = fast_exp2(__builtin_fmaf(S(i + 1), c, -m_use));
        const bf16x2 pr = {(__bf16)p0, (__bf16)p1};
        sum += p0;
        sum += p1;
        rounded_sum = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, rounded_sum, false);
        P(i, pr[0]);
        P(i + 1, pr[1]);
    }
    return rounded ? rounded_sum : sum;
}

// O^T += V^T P^T for the 32 keys whose LDS tile starts at vl; P: a row's probabilities, in one part or as the sum of several.
// k-slot s of MFMA cc is key 16*cc + 8*(s/4) + 4*(lane/32) + s%4 of the block.
template <int D, int PARTS>
__device__ __forceinline__ void pv32_parts(uint32_t vl, const bf16x8 (&P)[PARTS][2], WaveAcc<D>& st, int lane) {
    using G_ = Geo<D>;
    const int g = lane >> 5, hi = (lane >> 4) & 1, i16 = lane & 15;
    // the 16 lanes of a transpose read address 4 keys (4*g + i16/4 ..) x 16 consecutive d
    const int key = 4 * g + (i16 >> 2);
    // inside the 64-byte quad of d block db: bytes hi*32 + (i16&3)*8
    const uint32_t va = vl + (key / G_::KPW) * G_::GS + (key % G_::KPW) * 64 + hi * 32 + (i16 & 3) * 8;
    constexpr int K8 = (8 / G_::KPW) * G_::GS + (8 % G_::KPW) * 64;      // +8 keys
    constexpr int K16 = (16 / G_::KPW) * G_::GS;                        // +16 keys
#pragma unroll
    for (int cc = 0; cc < 2; ++cc) {
#pragma unroll
        for (int db = 0; db < G_::NDB; ++db) {
            const uint32_t a0 = va + cc * K16 + db * (G_::KPW * 64);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, a0));
            const s16x4 hi4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, a0 + K8));
            const s16x8 av = {lo[0], lo[1], lo[2], lo[3], hi4[0], hi4[1], hi4[2], hi4[3]};
#pragma unroll
            for (int part = 0; part < PARTS; ++part)
                st.O[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, av), P[part][cc], st.O[db], 0, 0, 0);
        }
    }
}
template <int D>
__device__ __forceinline__ void pv32(uint32_t vl, const bf16x8 (&P)[2], WaveAcc<D>& st, int lane) {
    pv32_parts<D, 1>(vl, reinterpret_cast<const bf16x8(&)[1][2]>(P), st, lane);
}

// One 32-key block, straight: used by narrow items (bandwidth-bound, no pipelining needed).
template <int D>
__device__ __forceinline__ void block32(uint32_t kl, uint32_t vl, const bf16x8 (&Q)[Geo<D>::NKK], WaveAcc<D>& st,
                                        float c, int rel, bool masked, bool rounded, int lane) {
    f32x16 S;
    bf16x8 P[2];
    qk32<D>(kl, Q, S, lane);
    if (masked) mask32(S, rel);                          // wave-uniform
    const float mx = rowmax32(S) * c;
    if (__any(mx > st.m + RESCALE_SLACK)) raise_reference<D>(st, mx);
    st.l += exp_sum<16>(c, st.m == NEG_INF ? 0.0f : st.m, rounded, [&](int i) { return S[i]; }, [&](int i, __bf16 v) { P[i >> 3][i & 7] = v; });
    pv32<D>(vl, P, st, lane);
}

// ---------------------------------------------------------------------------------------------
// The same steps for a wave of at most 16 query rows (a decode row's grouped heads), with v_mfma_f32_16x16x32_bf16:
// half the matrix and softmax work of the 32-row steps per key.  A lane owns query column lane % 16; with g = lane / 16
// it holds S^T for keys 4 k + i and 16 + 4 k + i (i < 4; k = key_group16(g)) of the block, which are also its eight k-slots
// of the second product, so P^T is again built in registers; O^T tile dt holds d = 16 dt + 4 g + i.

__device__ __forceinline__ float max_xor16(float x) {      // as max_xor32, for lane ^ 16
    const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_xor16(float x) {
    const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Which group of 4 keys (of the 16 keys of a tile) the lanes 16 g .. 16 g + 15 hold: 0, 2, 1, 3.  With this order the 32 lanes
// that one pass of a transpose read serves (g = 0, 1 or g = 2, 3) touch 256 contiguous bytes of the padded key groups
// (keys 0-3 and 8-11, or 4-7 and 12-15: LDS groups 16 bytes apart modulo 256) for d = 128; measured, the bank-conflict
// cycles of a decode launch are half of those with the order 0, 1, 2, 3.
__device__ __forceinline__ int key_group16(int g) { return ((g & 1) << 1) | ((g >> 1) & 1); }

template <int D>
struct WaveAcc16 {
    f32x4 O[D / 16];
    float m;
    float l;      // this lane's share of the running sum (the four lanes of a column hold quarters)
};

template <int D>
__device__ __forceinline__ void qk16(uint32_t kl, const bf16x8 (&Q)[D / 32], f32x4 (&S)[2], int lane) {
    using G_ = Geo<D>;
    // matrix row rho = lane % 16 carries key 4 * key_group16(rho / 4) + rho % 4 of the tile, so that lane group g ends up
    // with the keys of group key_group16(g)
    const int r = key_group16((lane & 15) >> 2) * 4 + (lane & 3), g = lane >> 4;
    // chunk 4*kk + g of key 16*t + r
    const uint32_t ka = kl + (r / G_::KPW) * G_::GS + (r % G_::KPW) * 64 + g * 16;
    constexpr int K16 = (16 / G_::KPW) * G_::GS;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        S[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) {
            const u32x4 raw = *LDS_PTR(const u32x4, ka + t * K16 + kk * (G_::KPW * 64));
            S[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, raw), Q[kk], S[t], 0, 0, 0);
        }
    }
}

// rel: per lane, (last visible key of this lane's query) - (first key of the block) - 4*key_group16(lane/16)
__device__ __forceinline__ void mask16(f32x4 (&S)[2], int rel) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) S[t][i] = 16 * t + i <= rel ? S[t][i] : NEG_INF;
}

template <int D>
__device__ __forceinline__ void raise_reference16(WaveAcc16<D>& st, float mx) {
    const float m_new = fmaxf(st.m, mx);
    const float alpha = fast_exp2(st.m - (m_new == NEG_INF ? 0.0f : m_new));
    st.l *= alpha;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) st.O[dt] *= alpha;
    st.m = m_new;
}

template <int D, int PARTS>
__device__ __forceinline__ void pv16_parts(uint32_t vl, const bf16x8 (&P)[PARTS], WaveAcc16<D>& st, int lane) {
    using G_ = Geo<D>;
    const int g = lane >> 4, i16 = lane & 15;
    // the 16 lanes of a transpose read address 4 keys x 16 consecutive d and receive 4 keys of one d each
    const int key = 4 * key_group16(g) + (i16 >> 2);
    const uint32_t va = vl + (key / G_::KPW) * G_::GS + (key % G_::KPW) * 64 + (i16 & 3) * 8;
    constexpr int K16 = (16 / G_::KPW) * G_::GS;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
        const uint32_t a0 = va + (dt >> 1) * (G_::KPW * 64) + (dt & 1) * 32;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, a0));
        const s16x4 hi4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, a0 + K16));
        const s16x8 av = {lo[0], lo[1], lo[2], lo[3], hi4[0], hi4[1], hi4[2], hi4[3]};
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
            st.O[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av), P[part], st.O[dt], 0, 0, 0);
    }
}
template <int D>
__device__ __forceinline__ void pv16(uint32_t vl, const bf16x8& P, WaveAcc16<D>& st, int lane) {
    pv16_parts<D, 1>(vl, reinterpret_cast<const bf16x8(&)[1]>(P), st, lane);
}

// S^T and its softmax; P = the operand of the second product
template <int D>
__device__ __forceinline__ bf16x8 softmax16(uint32_t kl, const bf16x8 (&Q)[D / 32], WaveAcc16<D>& st, float c, int rel, bool masked, bool rounded, int lane) {
    f32x4 S[2];
    qk16<D>(kl, Q, S, lane);
    if (masked) mask16(S, rel);                          // wave-uniform
    float mx = fmaxf(fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3])), fmaxf(fmaxf(S[1][0], S[1][1]), fmaxf(S[1][2], S[1][3])));
    mx = max_xor32(max_xor16(mx)) * c;
    if (__any(mx > st.m + RESCALE_SLACK)) raise_reference16<D>(st, mx);
    bf16x8 P;
    st.l += exp_sum<8>(c, st.m == NEG_INF ? 0.0f : st.m, rounded, [&](int i) { return S[i >> 2][i & 3]; }, [&](int i, __bf16 v) { P[i] = v; });
    return P;
}

// ---------------------------------------------------------------------------------------------
// f(integral_constant<int, I>) for I = I0 .. N-1, unrolled at compile time (a runtime loop, even one marked for
// unrolling, leaves the fragment arrays below indexed at run time, i.e. in scratch memory)
template <int I, int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

// One wave-wide direct global -> LDS load: lane i moves the 16 bytes at gbase + voff_i to LDS
// byte lds + 16 i (gbase and lds wave-uniform; the LDS base travels in M0).  Written as inline
// assembly so that the compiler does not track it: its own LDS reads of the *other* pipeline
// stage would otherwise wait for these loads.  dma_wait() must precede the barrier that
// publishes the data.  Compiler-issued vmcnt waits stay correct: vector-memory loads retire in
// order, so extra loads in flight only make them stricter.  M0 is named as clobbered so that the compiler never
// assumes a value of its own survives the statement (it is a reserved register, which the compiler reports with a
// warning that is silenced here: nothing has to be preserved, M0 is rewritten before every use).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16(const char* gbase, uint32_t voff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(gbase)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void dma_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Where the lane's part of a K/V load comes from and where it belongs in LDS, for NW waves that move consecutive groups of keys: lane i
// of a wave fetches the chunk that belongs in LDS slot i of its group.
template <int D, int KVT, int NW>
struct LanePlace {
    using G_ = Geo<D>;
    static constexpr int KPW = G_::KPW;
    // 8-bit cache: a wave moves two consecutive groups per pass, 16 codes per lane (lanes 0-31 the first group, 32-63 the
    // second; a lane fills two neighbouring LDS slots): half as many loads and address computations per byte as with
    // one 8-byte chunk per lane.  Two groups are 8 or 16 keys from a multiple of that, so they share a page too.
    static constexpr int GPP = KVT == KV_FP8 ? 2 : 1; // groups per wave and pass
    static constexpr int KPP = GPP * KPW;             // keys per wave and pass
    static constexpr int ES = RawChunk<KVT>::ES;

    // The lane's first LDS slot inside its group, and which of the pass's groups that is.  Slot l = (quad, key, chunk in
    // quad); with two groups per pass a lane owns slots l and l + 1 (l even: neighbouring chunks of one key row).
    __device__ __forceinline__ static int lane_slot(int t) { return GPP == 1 ? (t & 63) : 2 * (t & 31); }
    __device__ __forceinline__ static int lane_group(int t) { return GPP == 1 ? 0 : (t & 63) >> 5; }
    __device__ __forceinline__ static int lane_key(int t) { return lane_group(t) * KPW + (lane_slot(t) >> 2) % KPW; }   // within the pass
    __device__ __forceinline__ static uint32_t lane_off(int t) {
        const int l = lane_slot(t);
        return (uint32_t)((lane_key(t) * D + ((l / (4 * KPW)) * 4 + (l & 3)) * 8) * ES);
    }

    __device__ __forceinline__ static uint32_t slot_of(int ps, int t) {
        return ((ps * NW + (t >> 6)) * GPP + lane_group(t)) * G_::GS + lane_slot(t) * 16;
    }
    __device__ __forceinline__ static void put(const RawChunk<KVT>& c, float scale, uint32_t at) {
        if constexpr (KVT == KV_FP8) {
            *LDS_PTR(u32x4, at) = c.widen_first(scale);
            *LDS_PTR(u32x4, at + 16) = c.widen_second(scale);
        } else {
            *LDS_PTR(u32x4, at) = c.widen(scale);
        }
    }
};

// ---------------------------------------------------------------------------------------------
// 8-bit pages

__device__ __forceinline__ int exponent_for(float amax) {
    // smallest e with amax <= 448 * 2^e  (448 = 1.75 * 2^8), clamped to [-40, 119]
    const uint32_t u = __float_as_uint(amax);
    const int ex = (int)(u >> 23) - 127;
    const uint32_t man = u & 0x7fffffu;
    int e = (man <= 0x600000u) ? ex - 8 : ex - 7;
    if ((u >> 23) == 0) e = -40;                              // zero / subnormal
    return min(119, max(-40, e));
}

__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
}

// The three passes over one (page, KV head) of K or V that an append into an 8-bit cache takes, by nthr threads (this one: t).
// src: packed row of the first new token of this page and head (consecutive tokens row_bytes apart); n: new tokens of the page.
__device__ __forceinline__ u32x4 new_chunk(const char* src, int64_t row_bytes, int u, int cph) {
    return *reinterpret_cast<const u32x4*>(src + (u / cph) * row_bytes + (u % cph) * 16);
}
__device__ __forceinline__ float chunk_amax(const u32x4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float amax = 0.0f;
#pragma unroll
    for (int x = 0; x < 4; ++x) amax = fmaxf(amax, fmaxf(fabsf(__uint_as_float(w[x] << 16)), fabsf(__uint_as_float(w[x] & 0xffff0000u))));
    return amax;
}
__device__ __forceinline__ u32x2 encode_chunk(const u32x4& v, float inv) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float f[8];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        f[2 * x] = __uint_as_float(w[x] << 16) * inv;
        f[2 * x + 1] = __uint_as_float(w[x] & 0xffff0000u) * inv;
    }
    if (inv <= 0x1p-119f) {                           // the exponent is clamped: finite numbers saturate (the conversion makes them NaN from 464 on)
#pragma unroll
        for (int x = 0; x < 8; ++x) f[x] = fabsf(f[x]) > 448.0f && fabsf(f[x]) < 512.0f ? copysignf(448.0f, f[x]) : f[x];
    }
    return u32x2{encode4(f[0], f[1], f[2], f[3]), encode4(f[4], f[5], f[6], f[7])};
}
// this thread's largest magnitude
__device__ __forceinline__ float page_amax(const char* src, int64_t row_bytes, int n, int cph, int t, int nthr) {
    float amax = 0.0f;
    for (int u = t; u < n * cph; u += nthr) amax = fmaxf(amax, chunk_amax(new_chunk(src, row_bytes, u, cph)));
    return amax;
}
// 2^(e_old - e) for the codes of a page whose exponent rises to e; the exponents are up to 159 apart, and below 2^-126 every code becomes a
// zero of its sign (448 * 2^-127 is far below half the smallest code).
__device__ __forceinline__ float reencode_factor(int e_old, int e) { return __uint_as_float((uint32_t)max(0, e_old - e + 127) << 23); }
// the page's first n_old slots held codes of exponent e_old: re-encode them for e > e_old
__device__ __forceinline__ void page_reencode(uint8_t* pg, int n_old, int D, int e_old, int e, int t, int nthr) {
    const float f = reencode_factor(e_old, e);
    for (int u = t; u < n_old * (D / 4); u += nthr) {
        uint32_t* q4 = reinterpret_cast<uint32_t*>(pg) + u;
        const uint32_t w = *q4;
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
        const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        *q4 = encode4(lo.x * f, lo.y * f, hi.x * f, hi.y * f);
    }
}
// encode the new tokens into the slots from dst on: x * 2^-e
__device__ __forceinline__ void page_encode(uint8_t* dst, const char* src, int64_t row_bytes, int n, int D, int e, int t, int nthr) {
    const int cph = D / 8;
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    for (int u = t; u < n * cph; u += nthr)
        *reinterpret_cast<u32x2*>(dst + (u / cph) * D + (u % cph) * 8) = encode_chunk(new_chunk(src, row_bytes, u, cph), inv);
}

// ---------------------------------------------------------------------------------------------
// launches of one workgroup column per page that new tokens fall into

struct PageJob {
    int page;                  // physical page
    int C, t0, t1;             // cached tokens of the row; positions [t0, t1) of it are this page's new tokens
    int row;                   // packed row of token t0
};
// Every lane loads a row or two, and the row of this workgroup's page is then picked from the lanes: one trip to the arguments.
__device__ __forceinline__ PageJob page_job(const AppendParams& p) {
    const int idx = p.pg0 + (int)blockIdx.x - p.up_blocks, lane = threadIdx.x & 63;
    static_assert(APPEND_MAX_REQS == 128, "two rows per lane");
    const AppendRow lo = p.rows[lane];
    AppendRow hi = {0, 0, 0, 0};
    if (p.n > 64) hi = p.rows[lane + 64];
    // the last row whose pages start at or before idx (rows without new tokens share their successor's start)
    const int r = __popcll(__ballot(lane < p.n && lo.pg_off <= idx)) + __popcll(__ballot(lane + 64 < p.n && hi.pg_off <= idx)) - 1;
    const AppendRow s = r < 64 ? lo : hi;
    const int C = __builtin_amdgcn_readlane(s.C, r & 63), L = __builtin_amdgcn_readlane(s.L, r & 63);
    const int lp = (C >> p.logP) + idx - __builtin_amdgcn_readlane(s.pg_off, r & 63);
    PageJob j;
    j.C = C;
    j.t0 = max(C, lp << p.logP);
    j.t1 = min(C + L, (lp + 1) << p.logP);
    j.row = __builtin_amdgcn_readlane(s.row_off, r & 63) + j.t0 - C;
    j.page = p.block_table[(int64_t)(p.req0 + r) * p.max_pages + lp];
    return j;
}

}  // namespace ampd
