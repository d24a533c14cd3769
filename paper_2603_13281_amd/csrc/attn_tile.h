// What the attention kernels on the matrix cores share (bf16 storage, head_dim 128, blocks of 16): loads of a 32-token group, its scores,
// softmax and sum of values for up to three or four tiles of 16 queries, and the image in which a workgroup's waves meet.
//
// MFMA 16x16x32 bf16 operand layout (lane l, q = l / 16):
//   A[row l%16][k 8q..8q+7], B[k 8q..8q+7][col l%16], C[row 4q+i][col l%16] (i = 0..3).
// Token <-> tile-row mapping inside a 32-token group (two KV blocks), chosen so that the 8
// P values a lane owns after the two S^T tiles are 8 consecutive tokens of one block:
//   S^T tile t, row 4q'+i'  <->  block q'/2, token-in-block 8(q'%2) + 4t + i'
//   PV contraction index k = 8q + 4t + i  <->  block q/2, token-in-block 8(q%2) + 4t + i.
#pragma once
#include "device_util.h"

#include <type_traits>

namespace icarus {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

namespace {

constexpr int kD = 128;       // head_dim
constexpr int kBk = 16;       // tokens per block
constexpr int kGrp = 32;      // tokens per wave iteration (two blocks)
constexpr int kKS = kD / 32;  // k-steps of the QK^T contraction
constexpr int kDT = kD / 16;  // d tiles of the PV product
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.f;  // log2 units a score may exceed the softmax reference before it is moved

struct KVFrag {
    bf16x8 k[2][kKS];  // k[t][ks]: A operand of S^T tile t, k-step ks
    bf16x8 v[kDT];     // v[dt]:    A operand of O^T tile dt
};

__device__ __forceinline__ bf16x8 zero8() {
    bf16x8 z;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = (__bf16)0.f;
    return z;
}

// Issue the 16 loads of one 32-token group.  blk0/blk1: physical block ids (wave-uniform).
__device__ __forceinline__ void load_group(KVFrag &f, const bf16_t *__restrict__ pool, int blk0, int blk1, int c, int Hkv,
                                           int lane) {
    const int m = lane & 15, q = lane >> 4;
    const size_t head_stride = (size_t)2 * kBk * kD;
    // K rows: lane m reads block m/8, token-in-block 8((m/4)%2) + 4t + m%4, d = 32ks + 8q
    const bf16_t *kb = pool + ((size_t)((m >> 3) ? blk1 : blk0) * Hkv + c) * head_stride;
    const int tok0 = 8 * ((m >> 2) & 1) + (m & 3);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int ks = 0; ks < kKS; ++ks)
            f.k[t][ks] = *(const bf16x8 *)(kb + (size_t)(tok0 + 4 * t) * kD + 32 * ks + 8 * q);
    // V^T rows: lane reads block q/2, d = 16dt + m, tokens 8(q%2) .. +7
    const bf16_t *vb = pool + ((size_t)((q >> 1) ? blk1 : blk0) * Hkv + c) * head_stride + (size_t)kBk * kD;
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) f.v[dt] = *(const bf16x8 *)(vb + (size_t)(16 * dt + m) * kBk + 8 * (q & 1));
}

// The O^T accumulators live in the accumulation registers, where the matrix cores update them in place.  The
// rare rescale (a moved softmax reference) multiplies copies in ordinary registers; left to itself the
// compiler then keeps the accumulators of the common path in ordinary registers too and moves all of them
// across for every group.  An empty statement that demands its operand in an accumulation register, placed
// where the two paths meet, keeps the copies inside the rare branch.
#define ICARUS_IN_ACC(x) asm volatile("" : "+a"(x))

// Where the decode walks keep the wave's Q fragments: in registers when the wave has two or three query tiles (a
// wave issues in order and is alone on its SIMD, so a fragment read in front of the MFMAs that need it stalls it for
// the read's whole latency, up to twelve times per group); with one tile they stay in LDS, which keeps that
// instantiation at two workgroups per CU.
template <int NT>
constexpr bool kQInRegs = NT > 1;

// Per-wave running state for NT query tiles.
template <int NT>
struct State {
    f32x4 o[kDT][NT];  // O^T accumulators: [d 16dt + 4q + i][query 16qt + l%16]
    float m[NT];       // running max (log2 domain), uniform over the 4 lanes sharing a query
    float l[NT];       // running sum, per-lane partial (reduced over q at the end)
};

// One 32-token group: S^T, online softmax, PV, one 16-query tile at a time so that only one
// tile's scores are live.  Uses the first N tiles of st.  Q fragments of those tiles (B operands): qr, in
// registers, or qlds, in LDS as [qt][ks][lane] (see kQInRegs).
// tail == false: all 32 tokens are valid for every query.
// tail == true:  `left` tokens of the chunk remain from this group's first token on (for the row
//   with the longest context); query tile qt of this lane may attend only to the first
//   left - stag[qt] of them (stag: how many positions the lane's query row ends before the last
//   row -- 0 at decode, the causal stagger of a prefill chunk).
template <int NT, int N, bool tail>
__device__ __forceinline__ void compute_group(State<NT> &st, KVFrag &f, const bf16x8 (&qr)[NT][kKS], const bf16x8 *__restrict__ qlds, int left,
                                              const int (&stag)[NT], float scale_log2, int lane) {
    const int q = lane >> 4;
    // token index inside the group of S^T element (tile t, register i) on this lane: tbase + 4t + i
    const int tbase = 16 * (q >> 1) + 8 * (q & 1);
    if (tail) {
        // stale cache bytes past the end may hold anything: zero those V columns (scores are masked below)
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (tbase + e >= left) f.v[dt][e] = (__bf16)0.f;
    }
#pragma unroll
    for (int qt = 0; qt < N; ++qt) {
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) ICARUS_IN_ACC(st.o[dt][qt]);
        f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < kKS; ++ks) {
            const bf16x8 qv = kQInRegs<NT> ? qr[qt][ks] : qlds[(qt * kKS + ks) * 64 + lane];
            s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.k[0][ks], qv, s0, 0, 0, 0);
            s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.k[1][ks], qv, s1, 0, 0, 0);
        }
        // raw scores; the softmax scale (> 0) is applied to their maximum and inside the exponent's fused
        // multiply-add, not to each score
        float sv[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sv[i] = s0[i];
            sv[4 + i] = s1[i];
        }
        if (tail) {
            const int lim = left - stag[qt];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (tbase + e >= lim) sv[e] = -INFINITY;
        }
        float mx = sv[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, sv[e]);
        mx *= scale_log2;
        // st.m is a reference exponent, not necessarily the exact running max: it moves (and the
        // accumulators are rescaled) only when some score exceeds it by more than kSlack, so
        // p = 2^(s - m) stays below 2^kSlack and the common case needs no cross-lane exchange.
        if (__any(mx > st.m[qt] + kSlack)) {
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float m_old = st.m[qt];
            const float m_new = fmaxf(m_old, mx);
            st.m[qt] = m_new;
            // in a tail group a query may have no valid token yet (m_new still -inf): nothing to rescale
            float alpha = (tail && m_new == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f(m_old - m_new);
            st.l[qt] *= alpha;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) {
                st.o[dt][qt][0] *= alpha; st.o[dt][qt][1] *= alpha; st.o[dt][qt][2] *= alpha; st.o[dt][qt][3] *= alpha;
                ICARUS_IN_ACC(st.o[dt][qt]);
            }
        }
        const float m_ref = st.m[qt];
        float rs = 0.f;
        bf16x8 pb;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[e], scale_log2, -m_ref));
            if (tail && m_ref == -INFINITY) p = 0.f;
            rs += p;
            pb[e] = (__bf16)p;
        }
        st.l[qt] += rs;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) st.o[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v[dt], pb, st.o[dt][qt], 0, 0, 0);
    }
}

// A wave's walk over its share of the chunk: groups first, first + stride, ... with N query tiles, two register buffers, loads
// issued one group ahead; f0 holds group `first` (or is on its way) when the walk begins.  The first n_clean groups are valid for
// every query; the last ones of the wave, a partial last group among them, are multiplied with masks.  What the loop loads it also
// multiplies: loads that only repeat the last block would hold up the loads of the next piece.  (The loop's own loads are
// unconditional: with a load under a condition the compiler no longer knows how many younger loads are in flight when a buffer
// is consumed and waits for all of them, the prefetch included.)
template <int NT, int N, typename Frag, typename Load, typename Compute>
__device__ __forceinline__ void wave_walk(State<NT> &st, Frag &f0, int n_tok, int first, int stride, Load load, Compute compute) {
    const int n_grp = (n_tok + kGrp - 1) / kGrp;
    Frag f1;
    int grp = first;
#pragma nounroll
    for (; grp + 2 * stride < n_grp; grp += 2 * stride) {
        load(f1, grp + stride);
        compute(std::false_type(), f0, kGrp);
        load(f0, grp + 2 * stride);
        compute(std::false_type(), f1, kGrp);
    }
    if (grp + stride < n_grp) {
        load(f1, grp + stride);
        compute(std::false_type(), f0, kGrp);
        f0 = f1;
        grp += stride;
    }
    if (grp < n_grp) compute(std::true_type(), f0, n_tok - grp * kGrp);
}

// ---- FP8 (E4M3) cache: 1-byte codes, value = code * scale (one scale for K, one for V) ----------------
// The codes are exact in bf16, so they go through the same bf16 MFMAs after a register conversion; the
// scales are folded into the softmax scale (K) and the final normalisation (V).  Loads stay 16 bytes
// per lane for K: a lane's 16 codes are 16 consecutive d of one token, i.e. the lane's operand
// elements of TWO k-steps, so the contraction index is laid out differently from the bf16 path
//   k-step 2s + h, lane quarter q  <->  d = 64 s + 16 q + 8 h .. + 7
// and the Q fragments are staged in the same order (a dot product does not care).  V^T rows hold 16
// tokens in 16 bytes; a lane needs the 8 of its quarter: 8-byte loads, 16 rows x 16 bytes of a block
// fully used by each wave-wide load.
struct KVRaw8 {
    uint4 k[2][2];  // k[t][s]: tile t, d slab s (64 codes per row, 16 per lane)
    uint2 v[kDT];   // v[dt]: 8 tokens of row d = 16 dt + l%16
};

__device__ __forceinline__ void load_group8(KVRaw8 &f, const uint8_t *__restrict__ pool, int blk0, int blk1, int c, int Hkv,
                                            int lane) {
    const int m = lane & 15, q = lane >> 4;
    const size_t head_stride = (size_t)2 * kBk * kD;  // bytes
    const uint8_t *kb = pool + ((size_t)((m >> 3) ? blk1 : blk0) * Hkv + c) * head_stride;
    const int tok0 = 8 * ((m >> 2) & 1) + (m & 3);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int sl = 0; sl < 2; ++sl) f.k[t][sl] = *(const uint4 *)(kb + (size_t)(tok0 + 4 * t) * kD + 64 * sl + 16 * q);
    const uint8_t *vb = pool + ((size_t)((q >> 1) ? blk1 : blk0) * Hkv + c) * head_stride + (size_t)kBk * kD;
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) f.v[dt] = *(const uint2 *)(vb + (size_t)(16 * dt + m) * kBk + 8 * (q & 1));
}

// 8 FP8 codes (two dwords) -> 8 bf16, exactly.
__device__ __forceinline__ bf16x8 cvt8(uint32_t lo, uint32_t hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    uint4 r;
    r.x = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
    r.y = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
    r.z = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
    r.w = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
    return __builtin_bit_cast(bf16x8, r);
}

// compute_group for raw FP8 fragments: the scores of all N tiles first (K codes are converted one
// k-step at a time and die at once), then the softmax of every tile, then PV with V^T codes converted
// one d tile at a time.  scale_log2 includes the K scale; the V scale is applied when the piece ends.
template <int NT, int N, bool tail>
__device__ __forceinline__ void compute_group8(State<NT> &st, const KVRaw8 &f, const bf16x8 (&qr)[NT][kKS], const bf16x8 *__restrict__ qlds, int left,
                                               const int (&stag)[NT], float scale_log2, int lane) {
    const int q = lane >> 4;
    const int tbase = 16 * (q >> 1) + 8 * (q & 1);
    f32x4 s0[N], s1[N];
#pragma unroll
    for (int qt = 0; qt < N; ++qt) {
        s0[qt] = f32x4{0.f, 0.f, 0.f, 0.f}; s1[qt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) ICARUS_IN_ACC(st.o[dt][qt]);
    }
#pragma unroll
    for (int ks = 0; ks < kKS; ++ks) {
        const uint4 r0 = f.k[0][ks >> 1], r1 = f.k[1][ks >> 1];
        const bf16x8 a0 = (ks & 1) ? cvt8(r0.z, r0.w) : cvt8(r0.x, r0.y);
        const bf16x8 a1 = (ks & 1) ? cvt8(r1.z, r1.w) : cvt8(r1.x, r1.y);
#pragma unroll
        for (int qt = 0; qt < N; ++qt) {
            const bf16x8 qv = kQInRegs<NT> ? qr[qt][ks] : qlds[(qt * kKS + ks) * 64 + lane];
            s0[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, qv, s0[qt], 0, 0, 0);
            s1[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, qv, s1[qt], 0, 0, 0);
        }
    }
    bf16x8 pb[N];
#pragma unroll
    for (int qt = 0; qt < N; ++qt) {
        float sv[8];  // raw scores, see compute_group
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sv[i] = s0[qt][i];
            sv[4 + i] = s1[qt][i];
        }
        if (tail) {
            const int lim = left - stag[qt];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (tbase + e >= lim) sv[e] = -INFINITY;  // also replaces whatever stale codes produced
        }
        float mx = sv[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, sv[e]);
        mx *= scale_log2;
        if (__any(mx > st.m[qt] + kSlack)) {  // see compute_group: lazy softmax reference
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float m_old = st.m[qt];
            const float m_new = fmaxf(m_old, mx);
            st.m[qt] = m_new;
            float alpha = (tail && m_new == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f(m_old - m_new);
            st.l[qt] *= alpha;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) {
                st.o[dt][qt][0] *= alpha; st.o[dt][qt][1] *= alpha; st.o[dt][qt][2] *= alpha; st.o[dt][qt][3] *= alpha;
                ICARUS_IN_ACC(st.o[dt][qt]);
            }
        }
        const float m_ref = st.m[qt];
        float rs = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[e], scale_log2, -m_ref));
            if (tail && m_ref == -INFINITY) p = 0.f;
            rs += p;
            pb[qt][e] = (__bf16)p;
        }
        st.l[qt] += rs;
    }
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) {
        bf16x8 av = cvt8(f.v[dt].x, f.v[dt].y);
        if (tail) {  // stale codes past the end may decode to anything, NaN included
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (tbase + e >= left) av[e] = (__bf16)0.f;
        }
#pragma unroll
        for (int qt = 0; qt < N; ++qt) st.o[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, pb[qt], st.o[dt][qt], 0, 0, 0);
    }
}

// The four waves' states of a piece, each over its own groups, put together: every wave leaves its state in LDS (image_store) and, after a
// barrier, each takes a quarter of the head dimension (image_finish): d tiles 2w, 2w + 1 of all queries.
template <int NT>
struct Image {
    static constexpr int kO = kDT * NT * 64, kBytes = kO * 16 + NT * 64 * 8;  // f32x4 [dt][qt][lane], float2 (max, sum) [qt][lane]
};
template <int NT>
__device__ __forceinline__ void image_store(const State<NT> &st, char *__restrict__ img, int lane) {
    f32x4 *o = (f32x4 *)img;
    float2 *ml = (float2 *)(img + Image<NT>::kO * 16);
#pragma unroll
    for (int qt = 0; qt < NT; ++qt) {
        ml[qt * 64 + lane] = make_float2(st.m[qt], st.l[qt]);
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) o[(dt * NT + qt) * 64 + lane] = st.o[dt][qt];
    }
}

}  // namespace
}  // namespace icarus
