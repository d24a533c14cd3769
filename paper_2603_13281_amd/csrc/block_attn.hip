// Attention of single-token rows over the blocks that were selected for their sequence and kv-head.
#include "attn_tile.h"
#include "block_ops.h"

#include <algorithm>

namespace icarus {
namespace {

#define DISPATCH_T(bf16, ...)                                        \
    do {                                                             \
        if (bf16) { typedef bf16_t T; __VA_ARGS__; }                 \
        else { typedef float T; __VA_ARGS__; }                       \
    } while (0)
#define DISPATCH_TK(bf16, kv8, ...)                                   \
    do {                                                              \
        if (kv8) { typedef fp8_t KT; DISPATCH_T(bf16, __VA_ARGS__); } \
        else if (bf16) { typedef bf16_t T; typedef bf16_t KT; __VA_ARGS__; } \
        else { typedef float T; typedef float KT; __VA_ARGS__; }      \
    } while (0)

// Any shape: a workgroup to a query head of a row; a thread to a position for the scores, to a channel for the sum of the values.
// Running maximum and sum in float32, rounds of kChunk positions.
constexpr int kChunk = 512;
template <typename T, typename KT>
__global__ void __launch_bounds__(256) k_block_attn_generic(BlockAttnArgs a, int Hq, int Hkv, int D, int Bk, float scale, float k_scale, float v_scale) {
    __shared__ float qs[256], sc[kChunk], red[16];
    __shared__ int64_t where[kChunk];  // element of a position's key block, with its place in the block in the low bits; -1: masked
    const int s = blockIdx.y, h = blockIdx.x, c = h / (Hq / Hkv);
    const int row0 = min(max(a.row_start[s], 0), a.R), row1 = min(max(a.row_start[s + 1], row0), a.R);
    const int len = max(a.kv_lens[s], 0), n_sel = min(max(a.counts[s], 0), a.max_selected);
    const int32_t *list = a.blocks + ((size_t)s * Hkv + c) * a.max_selected;
    const int32_t *bt = a.bt + (size_t)s * a.max_blocks;
    const KT *pool = (const KT *)a.pool + (size_t)c * 2 * Bk * D;
    const size_t blk_stride = (size_t)Hkv * 2 * Bk * D;
    for (int row = row0; row < row1; ++row) {
        const T *q = (const T *)a.q + ((size_t)row * Hq + h) * D;
        __syncthreads();
        for (int i = threadIdx.x; i < D; i += 256) qs[i] = Elem<T>::ld(q + i);
        float m = -INFINITY, l = 0.f, acc = 0.f;
        const int64_t n = (int64_t)n_sel * Bk;
        for (int64_t t0 = 0; t0 < n; t0 += kChunk) {
            const int cnt = (int)min((int64_t)kChunk, n - t0);
            __syncthreads();
            float most = -INFINITY;
            for (int t = threadIdx.x; t < cnt; t += 256) {
                const int b = list[(t0 + t) / Bk], off = (int)((t0 + t) % Bk);
                int id = -1;
                if (b >= 0 && b < a.max_blocks && (int64_t)b * Bk + off < len) id = bt[b];
                float dot = -INFINITY;
                where[t] = -1;
                if (id >= 0 && id < a.num_blocks) {
                    const KT *k = pool + (size_t)id * blk_stride + (size_t)off * D;
                    dot = 0.f;
                    for (int i = 0; i < D; ++i) dot += qs[i] * KVElem<KT>::ld(k + i, k_scale);
                    dot *= scale;
                    where[t] = (int64_t)((size_t)id * blk_stride + (size_t)Bk * D + off);
                }
                sc[t] = dot;
                most = fmaxf(most, dot);
            }
            const float m_new = fmaxf(m, block_max(most, red));
            if (m_new == -INFINITY) continue;  // nothing yet
            float sum = 0.f;
            for (int t = threadIdx.x; t < cnt; t += 256) {
                const float p = __expf(sc[t] - m_new);
                sc[t] = p;
                sum += p;
            }
            sum = block_sum(sum, red);
            const float alpha = m == -INFINITY ? 0.f : __expf(m - m_new);
            l = l * alpha + sum;
            acc *= alpha;
            m = m_new;
            if (threadIdx.x < D)
                for (int t = 0; t < cnt; ++t)
                    if (where[t] >= 0) acc += sc[t] * KVElem<KT>::ld(pool + where[t] + (size_t)threadIdx.x * Bk, v_scale);
        }
        if (threadIdx.x < D) Elem<T>::st((T *)a.out + ((size_t)row * Hq + h) * D + threadIdx.x, l > 0.f ? acc / l : 0.f);
    }
}

// ---- matrix cores: bf16 storage, head_dim 128, blocks of 16 -------------------------------------------------------------
// A workgroup (4 waves) takes one sequence, kv-head and range of its list, with up to NT tiles of 16 stacked queries (rows x g heads); its waves
// take groups of two blocks in turn, in the operand layout of attn_tile.h.  Blocks are independent reads of 8 KB (FP8: 4 KB) wherever they lie.
//
// Short lists are the rule (a sequence's whole walk is some hundred KB), so what a workgroup waits for at its start and end counts, and two or more
// workgroups share a CU to fill each other's waits: accumulators in ordinary registers, one buffer of keys and one of values, each refilled as soon as the
// products that read it are issued.  Keys of the next group are on their way during the softmax and the values' products, values during the scores.
//
// In front of the walk the workgroup turns its range of the list into block ids in LDS: full blocks first, then blocks that end behind the sequence's
// last token, entries that name nothing dropped.  Then the loop over full blocks needs no masks and loads without conditions.
constexpr int kMaxEntries = 1024;  // of the list to a round of a workgroup (its ids and fills sit in LDS)

struct SplitOut {
    float *o;        // [splits][R][Hq][D]
    float2 *ml;      // [splits][R][Hq]: maximum in log2 units, sum
    int splits;      // 1: the output itself is written
};

// Kept as whole words: as vectors of bfloat16 that some path masks by elements the compiler took them apart, a register to an element.
template <bool KV8> struct Keys { uint4 r[2][kKS]; };       // [t][ks]: A operand of S^T tile t, k-step ks
template <> struct Keys<true> { uint4 r[2][2]; };           // 16 codes of a token: two k-steps, see KVRaw8
template <bool KV8> struct Values { uint4 r[kDT]; };        // [dt]: A operand of O^T tile dt
template <> struct Values<true> { uint2 r[kDT]; };

template <bool KV8>
__device__ __forceinline__ void load_keys(Keys<KV8> &k, const void *pool, int b0, int b1, int c, int Hkv, int lane) {
    const int m = lane & 15, q = lane >> 4;
    const size_t at = ((size_t)((m >> 3) ? b1 : b0) * Hkv + c) * 2 * kBk * kD + (size_t)(8 * ((m >> 2) & 1) + (m & 3)) * kD;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if constexpr (KV8) {
#pragma unroll
            for (int sl = 0; sl < 2; ++sl) k.r[t][sl] = *(const uint4 *)((const uint8_t *)pool + at + 4 * t * kD + 64 * sl + 16 * q);
        } else {
#pragma unroll
            for (int ks = 0; ks < kKS; ++ks) k.r[t][ks] = *(const uint4 *)((const bf16_t *)pool + at + 4 * t * kD + 32 * ks + 8 * q);
        }
    }
}
template <bool KV8>
__device__ __forceinline__ void load_values(Values<KV8> &v, const void *pool, int b0, int b1, int c, int Hkv, int lane) {
    const int m = lane & 15, q = lane >> 4;
    const size_t at = ((size_t)((q >> 1) ? b1 : b0) * Hkv + c) * 2 * kBk * kD + kBk * kD + (size_t)m * kBk + 8 * (q & 1);
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) {
        if constexpr (KV8) v.r[dt] = *(const uint2 *)((const uint8_t *)pool + at + 16 * dt * kBk);
        else v.r[dt] = *(const uint4 *)((const bf16_t *)pool + at + 16 * dt * kBk);
    }
}

template <int NT>
struct Running {
    f32x4 o[kDT][NT];  // O^T: [d 16 dt + 4 q + i][query 16 qt + l % 16]
    float m[NT], l[NT];  // reference exponent (log2), sum of this lane's tokens
};

// S^T of N tiles.
template <int NT, int N, bool KV8>
__device__ __forceinline__ void scores_of(f32x4 (&sc)[NT][2], const Keys<KV8> &k, const bf16x8 (&qr)[NT][kKS]) {
#pragma unroll
    for (int qt = 0; qt < N; ++qt) sc[qt][0] = sc[qt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < kKS; ++ks)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            bf16x8 kv;
            if constexpr (KV8) {
                const uint4 r = k.r[t][ks >> 1];
                kv = (ks & 1) ? cvt8(r.z, r.w) : cvt8(r.x, r.y);
            } else {
                kv = __builtin_bit_cast(bf16x8, k.r[t][ks]);
            }
#pragma unroll
            for (int qt = 0; qt < N; ++qt) sc[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv, qr[qt][ks], sc[qt][t], 0, 0, 0);
        }
}

// Scores -> weights (bfloat16, the matrix cores' operand: half a step of 2^-8 each, while the sum l takes them unrounded); there: tokens of this lane's block
// that exist.  The reference moves, and the accumulators with it, only where a score passes it by kSlack (see compute_group).
template <int NT, int N, bool masked>
__device__ __forceinline__ void weights_of(uint4 (&p)[NT], Running<NT> &st, const f32x4 (&sc)[NT][2], int there, float scale_log2, int lane) {
    const int t0 = 8 * ((lane >> 4) & 1);
#pragma unroll
    for (int qt = 0; qt < N; ++qt) {
        float sv[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) sv[i] = masked && t0 + i >= there ? -INFINITY : sc[qt][i >> 2][i & 3];
        float mx = sv[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) mx = fmaxf(mx, sv[i]);
        mx *= scale_log2;
        if (__any(mx > st.m[qt] + kSlack)) {
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float m_old = st.m[qt], m_new = fmaxf(m_old, mx);
            st.m[qt] = m_new;
            const float f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_old - m_new);
            st.l[qt] *= f;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) st.o[dt][qt] *= f;
        }
        const float m_ref = masked && st.m[qt] == -INFINITY ? 0.f : st.m[qt];  // nothing yet: every weight 0
#pragma unroll
        for (int i = 0; i < 8; ++i) sv[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[i], scale_log2, -m_ref));
        p[qt] = make_uint4(pack_bf16(sv[0], sv[1]), pack_bf16(sv[2], sv[3]), pack_bf16(sv[4], sv[5]), pack_bf16(sv[6], sv[7]));
        st.l[qt] += ((sv[0] + sv[1]) + (sv[2] + sv[3])) + ((sv[4] + sv[5]) + (sv[6] + sv[7]));
    }
}

template <int NT, int N, bool KV8, bool masked>
__device__ __forceinline__ void add_values(Running<NT> &st, const Values<KV8> &v, const uint4 (&p)[NT], int there, int lane) {
    uint32_t keep[4];  // places behind the last token may hold anything
    if (masked) {
        const int t0 = 8 * ((lane >> 4) & 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) keep[i] = (t0 + 2 * i < there ? 0xffffu : 0u) | (t0 + 2 * i + 1 < there ? 0xffff0000u : 0u);
    }
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) {
        uint4 a;
        if constexpr (KV8) a = __builtin_bit_cast(uint4, cvt8(v.r[dt].x, v.r[dt].y));
        else a = v.r[dt];
        if (masked) a = make_uint4(a.x & keep[0], a.y & keep[1], a.z & keep[2], a.w & keep[3]);
#pragma unroll
        for (int qt = 0; qt < N; ++qt)
            st.o[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, p[qt]), st.o[dt][qt], 0, 0, 0);
    }
}

template <int NT, bool KV8>
__global__ void __launch_bounds__(256, 2) k_block_attn(BlockAttnArgs a, SplitOut part, int Hq, int Hkv, int tile_groups, float scale_log2, float v_scale) {
    __shared__ f32x4 image[4][kDT][64];  // one query tile of the four waves' accumulators, and its reference and sum
    __shared__ float2 image_ml[4][64];
    __shared__ int ids[kMaxEntries], wave_n[2][4];
    __shared__ uint8_t fill[kMaxEntries];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15, q = lane >> 4, g = Hq / Hkv;
    // workgroups of the same blocks (tile groups) follow each other on one XCD, whose L2 then serves all but the first
    const int lo = blockIdx.x & 7, rest = blockIdx.x >> 3, pair = rest / tile_groups * 8 + lo, tg0 = rest % tile_groups;
    if (pair >= a.S * Hkv) return;
    const int s = pair / Hkv, c = pair % Hkv, split = blockIdx.y;
    const int row0 = min(max(a.row_start[s], 0), a.R), G = (min(max(a.row_start[s + 1], row0), a.R) - row0) * g;
    const int len = max(a.kv_lens[s], 0), n_sel = min(max(a.counts[s], 0), a.max_selected);
    const int per = ((n_sel + part.splits - 1) / part.splits + 1) & ~1;  // whole groups to a split
    const int e_begin = min(n_sel, split * per), e_end = min(n_sel, e_begin + per);
    const int32_t *list = a.blocks + (size_t)pair * a.max_selected, *bt = a.bt + (size_t)s * a.max_blocks;

    for (int j0 = tg0 * NT * 16; j0 < G; j0 += tile_groups * NT * 16) {
        const int tiles = min(NT, (G - j0 + 15) / 16);
        // query 16 qt + m of this workgroup -> row row0 + j / g, head c * g + j % g; order of d in a k-step: see KVRaw8
        bf16x8 qr[NT][kKS];
#pragma unroll
        for (int qt = 0; qt < NT; ++qt) {
            const int j = min(j0 + 16 * qt + m, G - 1);  // behind the last query: the last again, its results are not kept
            const bf16_t *qp = (const bf16_t *)a.q + ((size_t)(row0 + j / g) * Hq + c * g + j % g) * kD;
#pragma unroll
            for (int ks = 0; ks < kKS; ++ks)
                qr[qt][ks] = *(const bf16x8 *)(qp + (KV8 ? 64 * (ks >> 1) + 16 * q + 8 * (ks & 1) : 32 * ks + 8 * q));
        }
        Running<NT> st;
#pragma unroll
        for (int qt = 0; qt < NT; ++qt) {
            st.m[qt] = -INFINITY;
            st.l[qt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) st.o[dt][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        for (int e0 = e_begin; e0 < e_end; e0 += kMaxEntries) {
            const int e1 = min(e_end, e0 + kMaxEntries);
            int n_full = 0, n_part = 0;
            for (int i0 = e0; i0 < e1; i0 += 256) {
                const int i = i0 + threadIdx.x;
                int id = -1, n = 0;
                if (i < e1) {
                    const int b = list[i];
                    if (b >= 0 && b < a.max_blocks) {
                        n = (int)min((int64_t)kBk, (int64_t)len - (int64_t)b * kBk);
                        if (n > 0) id = bt[b];
                    }
                }
                const bool there = id >= 0 && id < a.num_blocks, full = there && n == kBk, some = there && n < kBk;
                const unsigned long long mf = __ballot(full), mp = __ballot(some), below = (1ull << lane) - 1;
                __syncthreads();  // wave_n of the chunk before and ids of the round before have been read
                if (lane == 0) {
                    wave_n[0][w] = __popcll(mf);
                    wave_n[1][w] = __popcll(mp);
                }
                __syncthreads();
                int at = n_full + __popcll(mf & below), ap = n_part + __popcll(mp & below);
                for (int k = 0; k < 4; ++k) {
                    if (k < w) { at += wave_n[0][k]; ap += wave_n[1][k]; }
                    n_full += __builtin_amdgcn_readfirstlane(wave_n[0][k]);
                    n_part += __builtin_amdgcn_readfirstlane(wave_n[1][k]);
                }
                if (full) ids[at] = id;
                if (some) {  // from the back
                    ids[kMaxEntries - 1 - ap] = id;
                    fill[kMaxEntries - 1 - ap] = (uint8_t)n;
                }
            }
            __syncthreads();
            const int n_blk = n_full + n_part, n_grp = (n_blk + 1) / 2;
            // block i of the round: full ones in order, the others behind them
            auto at_of = [&](int i) { return i < n_full ? i : kMaxEntries - 1 - (i - n_full); };
            auto id_of = [&](int i) { return __builtin_amdgcn_readfirstlane(ids[at_of(min(i, n_blk - 1))]); };
            auto there_of = [&](int grp) {  // tokens of this lane's block of a group
                const int i = 2 * grp + (q >> 1);
                return i < n_full ? kBk : i < n_blk ? (int)fill[at_of(i)] : 0;
            };
            auto walk = [&](auto n_tiles) {
                constexpr int N = decltype(n_tiles)::value;
                Keys<KV8> k;
                Values<KV8> v;
                f32x4 sc[NT][2];
                uint4 p[NT];
                int b0 = id_of(2 * w), b1 = id_of(2 * w + 1), grp = w;
                load_keys<KV8>(k, a.pool, b0, b1, c, Hkv, lane);
                load_values<KV8>(v, a.pool, b0, b1, c, Hkv, lane);
                b0 = id_of(2 * (grp + 4)), b1 = id_of(2 * (grp + 4) + 1);
                // The barriers keep each load where it is written: hoisted above the products that read the same buffer, it would need a second one.
#pragma nounroll
                for (const int stop = min(n_grp - 4, n_full >> 1); grp < stop; grp += 4) {
                    const int n0 = id_of(2 * (grp + 8)), n1 = id_of(2 * (grp + 8) + 1);
                    scores_of<NT, N, KV8>(sc, k, qr);
                    __builtin_amdgcn_sched_barrier(0);
                    load_keys<KV8>(k, a.pool, b0, b1, c, Hkv, lane);
                    __builtin_amdgcn_sched_barrier(0);
                    weights_of<NT, N, false>(p, st, sc, kBk, scale_log2, lane);
                    add_values<NT, N, KV8, false>(st, v, p, kBk, lane);
                    __builtin_amdgcn_sched_barrier(0);
                    load_values<KV8>(v, a.pool, b0, b1, c, Hkv, lane);
                    __builtin_amdgcn_sched_barrier(0);
                    b0 = n0;
                    b1 = n1;
                }
                // the wave's last group, and any before it with a block that ends early
                for (;;) {
                    const int there = there_of(grp);
                    scores_of<NT, N, KV8>(sc, k, qr);
                    weights_of<NT, N, true>(p, st, sc, there, scale_log2, lane);
                    add_values<NT, N, KV8, true>(st, v, p, there, lane);
                    grp += 4;
                    if (grp >= n_grp) break;
                    b0 = id_of(2 * grp), b1 = id_of(2 * grp + 1);
                    load_keys<KV8>(k, a.pool, b0, b1, c, Hkv, lane);
                    load_values<KV8>(v, a.pool, b0, b1, c, Hkv, lane);
                }
            };
            if (w < n_grp) {
                if (tiles == 1) walk(std::integral_constant<int, 1>());
                if constexpr (NT >= 2) if (tiles == 2) walk(std::integral_constant<int, 2>());
                if constexpr (NT >= 3) if (tiles == 3) walk(std::integral_constant<int, 3>());
            }
        }
        // The four waves' states put together, a query tile at a time: each wave takes d tiles 2 w, 2 w + 1.
#pragma unroll
        for (int qt = 0; qt < NT; ++qt) {
            if (qt >= tiles) break;
            __syncthreads();
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) image[w][dt][lane] = st.o[dt][qt];
            image_ml[w][lane] = make_float2(st.m[qt], st.l[qt]);
            __syncthreads();
            float2 ml[4];
            float mx = -INFINITY, l = 0.f;
            f32x4 o[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                ml[k] = image_ml[k][lane];
                mx = fmaxf(mx, ml[k].x);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float f = ml[k].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[k].x - mx);  // a wave without tokens
                l += f * ml[k].y;
#pragma unroll
                for (int h = 0; h < 2; ++h) o[h] += f * image[k][2 * w + h][lane];
            }
            l += __shfl_xor(l, 16, 64);
            l += __shfl_xor(l, 32, 64);
            const int j = j0 + 16 * qt + m;
            if (j >= G) continue;
            const size_t at = (size_t)(row0 + j / g) * Hq + c * g + j % g;
            if (part.splits == 1) {
                const float inv = l > 0.f ? v_scale / l : 0.f;
                bf16_t *op = (bf16_t *)a.out + at * kD + 32 * w + 4 * q;
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *(uint2 *)(op + 16 * h) = make_uint2(pack_bf16(o[h][0] * inv, o[h][1] * inv), pack_bf16(o[h][2] * inv, o[h][3] * inv));
            } else {
                const size_t ps = (size_t)split * a.R * Hq + at;
#pragma unroll
                for (int h = 0; h < 2; ++h) *(f32x4 *)(part.o + ps * kD + 32 * w + 16 * h + 4 * q) = o[h] * v_scale;
                if (w == 0 && q == 0) part.ml[ps] = make_float2(mx, l);
            }
        }
    }
}

// The splits of a row's head joined, in their order: a wave to a head, two channels to a lane.
__global__ void __launch_bounds__(256) k_block_attn_join(BlockAttnArgs a, SplitOut part, int Hq) {
    const int s = blockIdx.x, h = blockIdx.z * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (h >= Hq) return;
    const int row0 = min(max(a.row_start[s], 0), a.R), row1 = min(max(a.row_start[s + 1], row0), a.R);
    for (int row = row0 + blockIdx.y; row < row1; row += gridDim.y) {
        const size_t at = (size_t)row * Hq + h, step = (size_t)a.R * Hq;
        const float2 mine = lane < part.splits ? part.ml[at + lane * step] : make_float2(-INFINITY, 0.f);
        const float mx = wave_max(mine.x), f = mine.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mine.x - mx);
        const float l = wave_sum(f * mine.y);
        float x = 0.f, y = 0.f;
        for (int k = 0; k < part.splits; ++k) {
            const float2 o = *(const float2 *)(part.o + (at + k * step) * kD + 2 * lane);
            const float fk = __shfl(f, k, 64);
            x += fk * o.x;
            y += fk * o.y;
        }
        const float inv = l > 0.f ? 1.f / l : 0.f;
        ((uint32_t *)a.out)[at * (kD / 2) + lane] = pack_bf16(x * inv, y * inv);
    }
}

constexpr int kMaxSplits = 32;  // k_block_attn_join has a lane to a split
int splits_for(int64_t pairs, int max_selected, int64_t wgs) {
    const int64_t want = (wgs + pairs - 1) / pairs, most = (max_selected + 7) / 8;  // 8 blocks: a group to a wave
    return (int)std::max<int64_t>(1, std::min<int64_t>({want, most, kMaxSplits}));
}

template <int NT, bool KV8>
hipError_t launch_mfma(const Dims &dm, const BlockAttnArgs &a, SplitOut part, int tile_groups, hipStream_t st) {
    const float scale_log2 = kLog2e / sqrtf((float)kD) * (KV8 ? dm.k_scale : 1.f);
    const int64_t pairs = (int64_t)a.S * dm.Hkv;
    hipLaunchKernelGGL((k_block_attn<NT, KV8>), dim3((unsigned)((pairs + 7) / 8 * 8 * tile_groups), part.splits), dim3(256), 0, st, a, part, dm.Hq, dm.Hkv,
                       tile_groups, scale_log2, KV8 ? dm.v_scale : 1.f);
    return hipGetLastError();
}

}  // namespace

bool block_attn_mfma_supported(const Dims &dm) { return dm.bf16 && dm.D == kD && dm.Bk == kBk; }

size_t block_attn_workspace(const Dims &dm, int S, int R, int max_selected) {
    if (!block_attn_mfma_supported(dm) || S == 0) return 256;
    const int splits = splits_for((int64_t)S * dm.Hkv, max_selected, 512);
    return splits > 1 ? (size_t)splits * R * dm.Hq * (kD + 2) * 4 + 512 : 256;
}

hipError_t launch_block_attn(const Dims &dm, const BlockAttnArgs &a, void *workspace, hipStream_t st) {
    const int g = dm.Hq / dm.Hkv;
    const int64_t pairs = (int64_t)a.S * dm.Hkv;
    const int rows = a.seq_rows ? a.seq_rows : (a.R + a.S - 1) / a.S;  // of a sequence, about
    const int tiles = (rows * g + 15) / 16, nt = tiles == 1 ? 1 : 2;
    const int tile_groups = std::min((tiles + nt - 1) / nt, 64);
    SplitOut part;
    part.splits = splits_for(pairs, a.max_selected, std::max<int64_t>(1, 512 / tile_groups));
    part.o = (float *)workspace;
    part.ml = (float2 *)(part.o + (size_t)part.splits * a.R * dm.Hq * kD);
    hipError_t e;
    if (nt == 1) e = dm.kv8 ? launch_mfma<1, true>(dm, a, part, tile_groups, st) : launch_mfma<1, false>(dm, a, part, tile_groups, st);
    else e = dm.kv8 ? launch_mfma<2, true>(dm, a, part, tile_groups, st) : launch_mfma<2, false>(dm, a, part, tile_groups, st);
    if (e != hipSuccess || part.splits == 1) return e;
    hipLaunchKernelGGL(k_block_attn_join, dim3(a.S, std::min(std::max(rows, 1), 64), (dm.Hq + 3) / 4), dim3(256), 0, st, a, part, dm.Hq);
    return hipGetLastError();
}

hipError_t launch_block_attn_generic(const Dims &dm, const BlockAttnArgs &a, hipStream_t st) {
    const float scale = 1.f / sqrtf((float)dm.D);
    DISPATCH_TK(dm.bf16, dm.kv8, hipLaunchKernelGGL((k_block_attn_generic<T, KT>), dim3(dm.Hq, a.S), dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.D, dm.Bk, scale,
                                                    dm.k_scale, dm.v_scale));
    return hipGetLastError();
}

}  // namespace icarus
