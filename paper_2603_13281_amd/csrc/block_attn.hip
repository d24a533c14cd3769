// Attention of single-token rows over the blocks that were selected for their sequence and kv-head.
#include "attn_tile.h"
#include "block_ops.h"
#include "block_util.h"

#include <algorithm>
#include <atomic>

namespace icarus {
namespace {

// Any shape: a workgroup to a query head of a row; a thread to a position for the scores, to a channel for the sum of the values.
// Running maximum and sum in float32, rounds of kChunk positions.  Right for every block and head size, and slow: see k_block_attn_f32.
constexpr int kChunk = 512;
template <typename T, typename KT>
__global__ void __launch_bounds__(256) k_block_attn_generic(BlockAttnArgs a, int Hq, int Hkv, int D, int Bk, float scale, float k_scale, float v_scale) {
    __shared__ float qs[256], sc[kChunk], red[16];
    __shared__ int64_t where[kChunk];  // a position's element of channel 0 of the values, -1: masked
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
            const float m_ref = m_new == -INFINITY ? 0.f : m_new;  // nothing yet, or nothing but NaN, which the maximum passes over
            float sum = 0.f;
            for (int t = threadIdx.x; t < cnt; t += 256) {
                const float p = __expf(sc[t] - m_ref);
                sc[t] = p;
                sum += p;
            }
            sum = block_sum(sum, red);
            if (m_new == -INFINITY && sum == 0.f) continue;
            const float alpha = m == -INFINITY ? 0.f : __expf(m - m_new);
            l = l * alpha + sum;
            acc *= alpha;
            m = m_new;
            if (threadIdx.x < D)
                for (int t = 0; t < cnt; ++t)
                    if (where[t] >= 0) acc += sc[t] * KVElem<KT>::ld(pool + where[t] + (size_t)threadIdx.x * Bk, v_scale);
        }
        if (threadIdx.x < D) Elem<T>::st((T *)a.out + ((size_t)row * Hq + h) * D + threadIdx.x, l == 0.f ? 0.f : acc / l);  // a NaN stays one
    }
}

// ---- matrix cores: bf16 storage, head_dim 128, blocks of 16 -------------------------------------------------------------
// An item is a sequence, kv-head, range of its list and up to NT tiles of 16 stacked queries (rows x g heads).  One workgroup (4 waves) to a CU takes
// items in turn; its waves take groups of two blocks in turn, two groups in registers, one of them on its way (attn_tile.h has the arithmetic).  The blocks are
// independent reads of 8 KB (FP8: 4 KB) wherever they lie, bound by HBM.
//
// Items are short -- a list of 64 blocks is 8 groups to a wave -- and what an item waits for before its first key is a chain of reads: its list entry, the block id of the
// entry, the block.  So while item i is walked, the ids of item i + 1 and its queries, and the list entries of item i + 2 are on their way, and the first blocks of item i + 1
// are requested before the waves' states of item i are put together.
// 64 sequences, 1-8 agents, 64 blocks (268 MB): 57.9 us, 4.7 TB/s, of which about 10 us are the first item's start and the last one's end.  Two workgroups to a CU, a buffer of
// keys and one of values each: 75 us; one with two buffers, each item from nothing: 70-75 us.  More than three tiles: the queries are dealt to
// workgroups three tiles at a time (16 sequences over an FP8 cache, 72 queries, 256 blocks 39 us; five tiles to a workgroup and half the list 51 us).
//
// The ids of an item stand in LDS, full blocks first, then blocks that end behind the sequence's last token, entries that name nothing dropped: the loop over full
// blocks needs no masks and loads without conditions.
constexpr int kItemBlocks = 256;  // list entries of an item, at most: a thread to an entry

struct SplitOut {
    float *o;    // [splits][R][Hq][D]
    float2 *ml;  // [splits][R][Hq]: maximum in log2 units, sum
    int splits;  // 1: the output itself is written
    int per;     // list entries of a split, even on the 128 kernel
    int tiles, tile_groups, n_items;  // tiles of an item, items to the rows of the call's largest sequence
};

// Which part of the call an item is: workgroups of one XCD that run at the same time take the tile groups of the same blocks, which its L2 then reads once.
struct Item {
    int s, c, split, tg;
    __device__ __forceinline__ Item(int i, const SplitOut &p, int S, int Hkv) {
        const int lo = i & 7, rest = i >> 3, pairs8 = (S * Hkv + 7) >> 3;
        tg = rest % p.tile_groups;
        const int hi = rest / p.tile_groups % pairs8;
        split = rest / p.tile_groups / pairs8;
        const int pair = hi * 8 + lo;
        s = pair / Hkv;
        c = pair - s * Hkv;
    }
};

// One group of two blocks for N query tiles: scores of all of them, one look whether any softmax reference has to move (rare: see compute_group), and then straight-line code in
// which the weights of one tile and the products of the tile before can be under way together -- with a branch to a tile, as compute_group has it, a wave
// that is alone on its SIMD waits out every step of every tile.  there: tokens of this lane's block (masked only).
//
// Weights and the values' product.  Weights of one bfloat16 (half a step, 2^-8, each) add as much error, squared, as the output's own rounding: 0.0023 of the output
// where that alone is 0.0017.  bfloat16 values: a weight is cut to 8 bits and the rest goes through a second product (2^-15; 64 sequences 57.4 -> 57.9 us, 1 sequence 8.2 -> 8.35).
// The rest is made greater than 0 (by 2^-20 of the weight) wherever the weight is, so that an infinite value stays what it is.  FP8
// values, whose codes are float16 numbers too: weights in float16 (2^-11, at the same speed; a second product 39 -> 48 us), kLift powers of two up, to at most 2^14, so
// that only weights below 2^-20 of the reference lose bits to float16's least exponent.
constexpr float kLift = 6.f;
template <int NT, int N, bool KV8, bool masked, typename Frag>
__device__ __forceinline__ void group_of(State<NT> &st, const Frag &f, const bf16x8 (&qr)[NT][kKS], const bf16x8 *__restrict__ qlds, int there, float scale_log2, int lane) {
    const int t0 = 8 * ((lane >> 4) & 1);
    f32x4 sc[N][2];
    uint4 v[kDT];
#pragma unroll
    for (int qt = 0; qt < N; ++qt) sc[qt][0] = sc[qt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < kKS; ++ks) {
        bf16x8 k[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if constexpr (KV8) {
                const uint4 r = f.k[t][ks >> 1];
                k[t] = (ks & 1) ? cvt8(r.z, r.w) : cvt8(r.x, r.y);
            } else {
                k[t] = f.k[t][ks];
            }
        }
#pragma unroll
        for (int qt = 0; qt < N; ++qt) {
            const bf16x8 qv = kQInRegs<NT> ? qr[qt][ks] : qlds[(qt * kKS + ks) * 64 + lane];
#pragma unroll
            for (int t = 0; t < 2; ++t) sc[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[t], qv, sc[qt][t], 0, 0, 0);
        }
    }
    uint32_t keep[4];  // places behind the last token may hold anything
    if (masked) {
#pragma unroll
        for (int i = 0; i < 4; ++i) keep[i] = (t0 + 2 * i < there ? 0xffffu : 0u) | (t0 + 2 * i + 1 < there ? 0xffff0000u : 0u);
    }
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) {
        if constexpr (KV8) v[dt] = cvt8_f16(f.v[dt].x, f.v[dt].y);
        else v[dt] = __builtin_bit_cast(uint4, f.v[dt]);
        if (masked) v[dt] = make_uint4(v[dt].x & keep[0], v[dt].y & keep[1], v[dt].z & keep[2], v[dt].w & keep[3]);
    }
    float mx[N];
    bool move = false;
#pragma unroll
    for (int qt = 0; qt < N; ++qt) {
        if (masked)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (t0 + i >= there) sc[qt][i >> 2][i & 3] = -INFINITY;
        const f32x4 a = sc[qt][0], b = sc[qt][1];
        mx[qt] = fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3]))) * scale_log2;
        move |= mx[qt] > st.m[qt] + kSlack;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) ICARUS_IN_ACC(st.o[dt][qt]);
    }
    if (__any(move)) {
#pragma unroll
        for (int qt = 0; qt < N; ++qt) {
            float m_new = fmaxf(mx[qt], __shfl_xor(mx[qt], 16, 64));
            m_new = fmaxf(st.m[qt], fmaxf(m_new, __shfl_xor(m_new, 32, 64)));
            if (!__any(mx[qt] > st.m[qt] + kSlack)) m_new = st.m[qt];  // a tile's results must not depend on the tiles beside it
            const float c = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m[qt] - m_new);
            st.m[qt] = m_new;
            st.l[qt] *= c;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) {
                st.o[dt][qt][0] *= c; st.o[dt][qt][1] *= c; st.o[dt][qt][2] *= c; st.o[dt][qt][3] *= c;
                ICARUS_IN_ACC(st.o[dt][qt]);
            }
        }
    }
#pragma unroll
    for (int qt = 0; qt < N; ++qt) {
        const float m_ref = (st.m[qt] == -INFINITY ? 0.f : st.m[qt]) - (KV8 ? kLift : 0.f);  // nothing yet: every weight 0
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[qt][i >> 2][i & 3], scale_log2, -m_ref));
        st.l[qt] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));  // as they are
        if constexpr (KV8) {
            const f16x8 p = __builtin_bit_cast(f16x8, make_uint4(pack_f16(e[0], e[1]), pack_f16(e[2], e[3]), pack_f16(e[4], e[5]), pack_f16(e[6], e[7])));
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) st.o[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v[dt]), p, st.o[dt][qt], 0, 0, 0);
        } else {
            uint32_t p[4], rest[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t x = __float_as_uint(e[2 * i]) & 0xffff0000u, y = __float_as_uint(e[2 * i + 1]) & 0xffff0000u;
                p[i] = x >> 16 | y;
                rest[i] = pack_bf16(__builtin_fmaf(e[2 * i], 1.f + 0x1p-20f, -__uint_as_float(x)), __builtin_fmaf(e[2 * i + 1], 1.f + 0x1p-20f, -__uint_as_float(y)));
            }
            const bf16x8 hi = __builtin_bit_cast(bf16x8, make_uint4(p[0], p[1], p[2], p[3])), lo = __builtin_bit_cast(bf16x8, make_uint4(rest[0], rest[1], rest[2], rest[3]));
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) st.o[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[dt]), hi, st.o[dt][qt], 0, 0, 0);
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) st.o[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[dt]), lo, st.o[dt][qt], 0, 0, 0);
        }
    }
}

template <int NT, bool KV8>
__global__ void __launch_bounds__(256) k_block_attn(BlockAttnArgs a, SplitOut part, int Hq, int Hkv, float scale_log2, float v_scale) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    // LDS: the waves' states | two buffers of Q fragments [qt][ks][lane]
    constexpr int kQBytes = NT * kKS * 1024, kQAt = 4 * Image<NT>::kBytes;
    __shared__ int ids[2][kItemBlocks], wave_n[2][4];
    __shared__ uint8_t fill[2][kItemBlocks];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15, q = lane >> 4, g = Hq / Hkv, n_wgs = gridDim.x;
    typedef typename std::conditional<KV8, KVRaw8, KVFrag>::type Frag;

    // The item of round r; the places of a round move on by an XCD's step, so that tile groups that most sequences do not have fall to all workgroups.
    auto item_of = [&](int r) {
        const int i = r * n_wgs + (blockIdx.x + 8 * r) % n_wgs;
        return i < part.n_items ? i : -1;
    };
    struct Meta { int s, c, split, row0, G, j0, len, n_sel; };  // G: stacked queries, from j0 on this item's; n_sel: entries of the list
    auto meta_of = [&](int i) {
        Meta x{};
        if (i < 0) return x;
        const Item it(i, part, a.S, Hkv);
        if (it.s >= a.S) return x;
        x.s = it.s;
        x.c = it.c;
        x.split = it.split;
        x.row0 = min(max(a.row_start[it.s], 0), a.R);
        x.G = (min(max(a.row_start[it.s + 1], x.row0), a.R) - x.row0) * g;
        x.j0 = it.tg * part.tiles * 16;
        x.len = max(a.kv_lens[it.s], 0);
        x.n_sel = min(max(a.counts[it.s], 0), a.max_selected);
        return x;
    };
    auto entry_of = [&](int i) {  // this thread's list entry
        if (i < 0) return -1;
        const Item it(i, part, a.S, Hkv);
        const int e = it.split * part.per + threadIdx.x;
        if (it.s >= a.S || (int)threadIdx.x >= part.per || e >= a.max_selected) return -1;
        return a.blocks[((size_t)it.s * Hkv + it.c) * a.max_selected + e];
    };
    auto id_of_entry = [&](const Meta &x, int entry, int &n) {  // its block, and the block's tokens
        n = 0;
        if (x.j0 >= x.G || x.split * part.per + (int)threadIdx.x >= x.n_sel || entry < 0 || entry >= a.max_blocks) return -1;
        n = (int)min((int64_t)kBk, (int64_t)x.len - (int64_t)entry * kBk);
        return n > 0 ? a.bt[(size_t)x.s * a.max_blocks + entry] : -1;
    };
    auto load_q = [&](const Meta &x, bf16x8 (&qv)[NT]) {  // wave w brings k-step w of every tile; order of d: see KVRaw8
#pragma unroll
        for (int qt = 0; qt < NT; ++qt) {
            const int j = max(min(x.j0 + 16 * qt + m, x.G - 1), 0);  // behind the last query: the last again, its results are not kept
            const int row = min(x.row0 + j / g, a.R - 1);
            qv[qt] = *(const bf16x8 *)((const bf16_t *)a.q + ((size_t)row * Hq + x.c * g + j % g) * kD +
                                       (KV8 ? 64 * (w >> 1) + 16 * q + 8 * (w & 1) : 32 * w + 8 * q));
        }
    };
    int n_full = 0, n_blk = 0;
    // first half: every wave counts its blocks; second half, after a barrier: the ids find their places
    auto count = [&](int id, int n) {
        const bool there = id >= 0 && id < a.num_blocks;
        const unsigned long long mf = __ballot(there && n == kBk), mp = __ballot(there && n < kBk);
        if (lane == 0) {
            wave_n[0][w] = __popcll(mf);
            wave_n[1][w] = __popcll(mp);
        }
    };
    auto place = [&](int id, int n, int buf) {
        const bool there = id >= 0 && id < a.num_blocks, full = there && n == kBk, some = there && n < kBk;
        const unsigned long long mf = __ballot(full), mp = __ballot(some), below = (1ull << lane) - 1;
        int at = __popcll(mf & below), ap = __popcll(mp & below), nf = 0, np = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int f = wave_n[0][k], p = wave_n[1][k];
            if (k < w) { at += f; ap += p; }
            nf += f;
            np += p;
        }
        n_full = __builtin_amdgcn_readfirstlane(nf);
        n_blk = __builtin_amdgcn_readfirstlane(nf + np);
        if (full) ids[buf][at] = id;
        if (some) {
            ids[buf][nf + ap] = id;
            fill[buf][nf + ap] = (uint8_t)n;
        }
        if (threadIdx.x == 0 && n_blk == 0) ids[buf][0] = 0;  // something to load
    };
    auto load = [&](Frag &f, const Meta &x, int buf, int grp) {
        const int most = max(n_blk - 1, 0);
        const int b0 = __builtin_amdgcn_readfirstlane(ids[buf][min(2 * grp, most)]), b1 = __builtin_amdgcn_readfirstlane(ids[buf][min(2 * grp + 1, most)]);
        if constexpr (KV8) load_group8(f, (const uint8_t *)a.pool, b0, b1, x.c, Hkv, lane);
        else load_group(f, (const bf16_t *)a.pool, b0, b1, x.c, Hkv, lane);
    };
    auto q_to_lds = [&](const bf16x8 (&qv)[NT], int buf) {
#pragma unroll
        for (int qt = 0; qt < NT; ++qt) ((bf16x8 *)(smem + kQAt + buf * kQBytes))[(qt * kKS + w) * 64 + lane] = qv[qt];
    };

    int r = 0, i1 = item_of(0);
    Frag f0;
    Meta x = meta_of(i1), nx;
    int entry, id, n;
    {
        const int e0 = entry_of(i1);
        entry = entry_of(item_of(1));
        bf16x8 qv[NT];
        id = id_of_entry(x, e0, n);
        load_q(x, qv);
        count(id, n);
        q_to_lds(qv, 0);
        __syncthreads();
        place(id, n, 0);
        __syncthreads();
        load(f0, x, 0, w);
    }
    for (int buf = 0;; buf ^= 1) {
        const bf16x8 *qlds = (const bf16x8 *)(smem + kQAt + buf * kQBytes);
        bf16x8 qr[NT][kKS], qv[NT];
        if constexpr (kQInRegs<NT>) {
#pragma unroll
            for (int qt = 0; qt < NT; ++qt)
#pragma unroll
                for (int ks = 0; ks < kKS; ++ks) qr[qt][ks] = qlds[(qt * kKS + ks) * 64 + lane];
        }
        // a sequence with more rows than the launch was sized for: the same blocks again for its next tiles
        const int far = part.tile_groups * part.tiles * 16;
        const bool again = x.j0 + far < x.G;
        const int i2 = again ? i1 : item_of(r + 1);
        if (again) {
            nx = x;
            nx.j0 += far;
            id = id_of_entry(nx, entry_of(i1), n);
            load_q(nx, qv);
        } else if (i2 >= 0) {
            nx = meta_of(i2);
            id = id_of_entry(nx, entry, n);
            load_q(nx, qv);
            entry = entry_of(item_of(r + 2));
        }
        State<NT> st;
#pragma unroll
        for (int qt = 0; qt < NT; ++qt) {
            st.m[qt] = -INFINITY;
            st.l[qt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) st.o[dt][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int n_grp = (n_blk + 1) / 2, stop = min(n_grp - 4, n_full >> 1), tiles = min(part.tiles, (x.G - x.j0 + 15) / 16);
        auto walk = [&](auto n_tiles) {
            constexpr int N = decltype(n_tiles)::value;
            auto compute = [&](auto masked, const Frag &f, int there) {
                group_of<NT, N, KV8, decltype(masked)::value>(st, f, qr, qlds, there, scale_log2, lane);
            };
            Frag f1;
            int grp = w;
#pragma nounroll
            for (; grp + 4 < stop; grp += 8) {
                load(f1, x, buf, grp + 4);
                compute(std::false_type(), f0, kBk);
                load(f0, x, buf, grp + 8);
                compute(std::false_type(), f1, kBk);
            }
            if (grp < stop) {
                load(f1, x, buf, grp + 4);
                compute(std::false_type(), f0, kBk);
                f0 = f1;
                grp += 4;
            }
            // the wave's last group, and any before it with a block that ends early
#pragma nounroll
            for (;;) {
                const int b = 2 * grp + (q >> 1);  // this lane's block
                compute(std::true_type(), f0, b < n_full ? kBk : b < n_blk ? (int)fill[buf][b] : 0);
                grp += 4;
                if (grp >= n_grp) break;
                load(f0, x, buf, grp);
            }
        };
        if (w < n_grp && tiles > 0) {
            if (tiles == 1) walk(std::integral_constant<int, 1>());
            if constexpr (NT >= 2) if (tiles == 2) walk(std::integral_constant<int, 2>());
            if constexpr (NT >= 3) if (tiles == 3) walk(std::integral_constant<int, 3>());
        }
        // The waves' states are put together: each wave leaves its own in LDS and takes d tiles 2 w, 2 w + 1 of all queries.
        auto leave = [&] {
            f32x4 *o = (f32x4 *)(smem + w * Image<NT>::kBytes);
            float2 *ml = (float2 *)(o + Image<NT>::kO);
#pragma unroll
            for (int qt = 0; qt < NT; ++qt) {
                ml[qt * 64 + lane] = make_float2(st.m[qt], st.l[qt]);
#pragma unroll
                for (int dt = 0; dt < kDT; ++dt) o[(dt * NT + qt) * 64 + lane] = st.o[dt][qt];
            }
        };
        auto take = [&] {
#pragma unroll
            for (int qt = 0; qt < NT; ++qt) {
                const int j = x.j0 + 16 * qt + m;
                if (qt >= tiles) continue;
                float2 ml[4];
                float mx = -INFINITY, l = 0.f;
                f32x4 o[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    ml[k] = ((const float2 *)(smem + k * Image<NT>::kBytes + Image<NT>::kO * 16))[qt * 64 + lane];
                    mx = fmaxf(mx, ml[k].x);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float f = ml[k].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[k].x - mx);  // a wave without tokens
                    l += f * ml[k].y;
#pragma unroll
                    for (int h = 0; h < 2; ++h) o[h] += f * ((const f32x4 *)(smem + k * Image<NT>::kBytes))[((2 * w + h) * NT + qt) * 64 + lane];
                }
                l += __shfl_xor(l, 16, 64);
                l += __shfl_xor(l, 32, 64);
                if (j >= x.G) continue;
                const size_t at = (size_t)(x.row0 + j / g) * Hq + x.c * g + j % g;
                if (part.splits == 1) {
                    const float inv = l > 0.f ? v_scale / l : 0.f;
                    bf16_t *op = (bf16_t *)a.out + at * kD + 32 * w + 4 * q;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        *(uint2 *)(op + 16 * h) = make_uint2(pack_bf16(o[h][0] * inv, o[h][1] * inv), pack_bf16(o[h][2] * inv, o[h][3] * inv));
                } else {
                    const size_t ps = (size_t)x.split * a.R * Hq + at;
#pragma unroll
                    for (int h = 0; h < 2; ++h) *(f32x4 *)(part.o + ps * kD + 32 * w + 16 * h + 4 * q) = o[h] * v_scale;
                    if (w == 0 && q == 0) part.ml[ps] = make_float2(mx, l);
                }
            }
        };
        __syncthreads();  // every wave has taken its part of the item before: a wave without a group of this one is here at once
        if (i2 >= 0) count(id, n);
        leave();
        if (i2 >= 0) q_to_lds(qv, buf ^ 1);
        __syncthreads();
        if (i2 >= 0) place(id, n, buf ^ 1);
        __syncthreads();
        if (i2 >= 0) load(f0, nx, buf ^ 1, w);
        take();
        if (i2 < 0) break;
        x = nx;
        i1 = i2;
        r += !again;
    }
}

bool on_matrix_cores(const Dims &dm) { return dm.bf16 && dm.D == kD && dm.Bk == kBk; }

// ---- block and head sizes that are multiples of 16: matrix cores in float32 ------------------------------------------------------
// For float32, head sizes other than 128 and blocks of more than 16 tokens.  A workgroup takes a sequence, kv-head, range of the list and a tile of 16 stacked queries; a wave takes
// sixteen tokens of a block in turn (with the next ones on their way: no faster).  Products of 16 x 16 x 4 with the transposed operands: scores are keys [token][channel] times
// queries [channel][query], which leaves lane t + 16 p query t's scores of tokens 4 p .. 4 p + 3, and these are at once the right operand of the values'
// product [channel][token] x [token][query], whose left operand is a row piece of the transposed block.  So nothing passes through LDS until the waves join, and
// a query's reference, sum and sums of values lie in its own four lanes.  float32, 4 heads of 64, 25 sequences x 9 rows x up to 190 blocks (147 MB): 29 us, 5.1 TB/s;
// the same on the vector units with the queries in LDS took 76 us, bound by LDS.  Rows beyond 16 / g read the blocks again, from the caches: float32, 8 heads of 128 for
// 32 queries, 32 x up to 9 rows x 64 blocks (268 MB) 85 us; two tiles of queries to a workgroup halve the reads and took 121 us, for want of waves.  bfloat16 keys and
// values become float32 here: 8 heads of 64 (134 MB) 63 us, bound by the products, a sixteenth of the rate of 16-bit ones; blocks of 64 tokens, 64 sequences of 4 rows
// x 32 heads over 1024 tokens of 8 heads of 128 (268 MB) 77 us, in blocks of 16 (k_block_attn) 45, a thread to a position (below 16 tokens or with odd sizes) 13.9 ms.
template <typename T, typename KT, int DT, bool EXACT>  // tiles of 16 channels: at most DT, or DT exactly
__global__ void __launch_bounds__(256) k_block_attn_f32(BlockAttnArgs a, SplitOut part, int Hq, int Hkv, int D_, int Bk, float scale_log2, float v_scale) {
    typedef typename Quad<KT>::raw Raw;
    __shared__ f32x4 image[2][DT][64];
    __shared__ int2 ids[kItemBlocks];  // of the list's entries: block of the pool, and its tokens
    __shared__ float image_m[4][16], image_l[4][16];
    const int D = EXACT ? 16 * DT : D_, d16 = D / 16;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, p4 = 4 * (lane >> 4), g = Hq / Hkv;
    const int pair = blockIdx.x, s = pair / Hkv, c = pair - s * Hkv, split = blockIdx.y;
    const int row0 = min(max(a.row_start[s], 0), a.R), G = (min(max(a.row_start[s + 1], row0), a.R) - row0) * g;
    const int len = max(a.kv_lens[s], 0), n_sel = min(max(a.counts[s], 0), a.max_selected);
    const int e0 = split * part.per, entries = max(0, min(part.per, n_sel - e0));
    const int parts = Bk / 16, units = entries * parts, step = 4 / parts, step_parts = 4 % parts;  // sixteen tokens of a block are a unit
    if ((int)threadIdx.x < entries) {
        int2 x = make_int2(0, 0);
        const int b = a.blocks[(size_t)pair * a.max_selected + e0 + threadIdx.x];
        if (b >= 0 && b < a.max_blocks && (int64_t)b * Bk < len) {
            const int id = a.bt[(size_t)s * a.max_blocks + b];
            if (id >= 0 && id < a.num_blocks) x = make_int2(id, min(Bk, len - b * Bk));
        }
        ids[threadIdx.x] = x;
    }
    __syncthreads();
    for (int j0 = 16 * blockIdx.z; j0 < G; j0 += 16 * gridDim.z) {
        const int j = min(j0 + t, G - 1);
        const size_t at = (size_t)(row0 + j / g) * Hq + c * g + j % g;
        float q[DT][4];
#pragma unroll
        for (int x = 0; x < DT; ++x)
            if (EXACT || x < d16) Quad<T>::get(*(const typename Quad<T>::raw *)((const T *)a.q + at * D + 16 * x + p4), q[x]);
        f32x4 o[DT];
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int x = 0; x < DT; ++x) o[x] = f32x4{0.f, 0.f, 0.f, 0.f};
        const auto add = [&](int id, int first, int n) {  // n of the block's tokens, from `first` on
            const KT *blk = (const KT *)a.pool + ((size_t)id * Hkv + c) * 2 * Bk * D;
            const KT *kr = blk + (first + min(t, n - 1)) * D + p4, *vr = blk + (D + t) * Bk + first + p4;  // behind the last token: the last again
            Raw k[DT], v[DT];
#pragma unroll
            for (int x = 0; x < DT; ++x)
                if (EXACT || x < d16) k[x] = *(const Raw *)(kr + 16 * x);
#pragma unroll
            for (int x = 0; x < DT; ++x)
                if (EXACT || x < d16) v[x] = *(const Raw *)(vr + (size_t)16 * Bk * x);
            f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < DT; ++x) {
                if (!EXACT && x >= d16) continue;
                float kf[4];
                Quad<KT>::get(k[x], kf);
#pragma unroll
                for (int u = 0; u < 4; ++u) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[u], q[x][u], sc, 0, 0, 0);
            }
            float most = -INFINITY, p[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                sc[u] = p4 + u < n ? sc[u] * scale_log2 : -INFINITY;
                most = fmaxf(most, sc[u]);
            }
            if (__any(most > m + kSlack)) {  // see compute_group: the reference moves rarely
                most = fmaxf(most, __shfl_xor(most, 16, 64));
                most = fmaxf(most, __shfl_xor(most, 32, 64));
                const float m_new = fmaxf(m, most), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
                m = m_new;
                l *= f;
#pragma unroll
                for (int x = 0; x < DT; ++x) o[x] *= f;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                p[u] = sc[u] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sc[u] - m);
                l += p[u];
            }
#pragma unroll
            for (int x = 0; x < DT; ++x) {
                if (!EXACT && x >= d16) continue;
                float vf[4];
                Quad<KT>::get(v[x], vf);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (n < 16) vf[u] = p4 + u < n ? vf[u] : 0.f;  // places behind the last token may hold anything
                    o[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[u], p[u], o[x], 0, 0, 0);
                }
            }
        };
        int e = w / parts, part_of = w % parts;
        for (int u = w; u < units; u += 4) {
            const int id = __builtin_amdgcn_readfirstlane(ids[e].x), n = __builtin_amdgcn_readfirstlane(ids[e].y) - 16 * part_of;
            if (n > 0) add(id, 16 * part_of, min(16, n));
            e += step;
            part_of += step_parts;
            if (part_of >= parts) part_of -= parts, ++e;
        }
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (lane < 16) {
            image_m[w][t] = m;
            image_l[w][t] = l;
        }
        __syncthreads();
        const float mx = fmaxf(fmaxf(image_m[0][t], image_m[1][t]), fmaxf(image_m[2][t], image_m[3][t]));
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += (image_m[k][t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(image_m[k][t] - mx)) * image_l[k][t];
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx);
#pragma unroll
        for (int x = 0; x < DT; ++x) o[x] *= f;
        const auto give = [&](int at) {
#pragma unroll
            for (int x = 0; x < DT; ++x)
                if (EXACT || x < d16) image[at][x][lane] = o[x];
        };
        const auto take = [&](int at) {
#pragma unroll
            for (int x = 0; x < DT; ++x)
                if (EXACT || x < d16) o[x] += image[at][x][lane];
        };
        if (w >= 2) give(w - 2);
        __syncthreads();
        if (w < 2) take(w);
        if (w == 1) give(1);  // its own place
        __syncthreads();
        if (w != 0) continue;
        take(1);
        if (j0 + t >= G) continue;
        if (part.splits == 1) {
            const float inv = sum == 0.f ? 0.f : v_scale / sum;
#pragma unroll
            for (int x = 0; x < DT; ++x) {
                if (!EXACT && x >= d16) continue;
                T *out = (T *)a.out + at * D + 16 * x + p4;
                if constexpr (sizeof(T) == 2) *(uint2 *)out = make_uint2(pack_bf16(o[x][0] * inv, o[x][1] * inv), pack_bf16(o[x][2] * inv, o[x][3] * inv));
                else *(f32x4 *)out = o[x] * inv;
            }
        } else {
            const size_t ps = (size_t)split * a.R * Hq + at;
#pragma unroll
            for (int x = 0; x < DT; ++x)
                if (EXACT || x < d16) *(f32x4 *)(part.o + ps * D + 16 * x + p4) = o[x] * v_scale;
            if (p4 == 0) part.ml[ps] = make_float2(mx, sum);
        }
    }
}

// The splits of a row's head joined, in their order: a wave to a head, two channels at a time to a lane.  Bound by its chain of two reads: 4 us for one sequence
// of 9 rows x 32 heads x 16 splits as for 16 of them.
template <typename T>
__global__ void __launch_bounds__(256) k_block_attn_join(BlockAttnArgs a, SplitOut part, int Hq, int D) {
    const int s = blockIdx.x, h = blockIdx.z * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (h >= Hq) return;
    const int row0 = min(max(a.row_start[s], 0), a.R), row1 = min(max(a.row_start[s + 1], row0), a.R);
    for (int row = row0 + blockIdx.y; row < row1; row += gridDim.y) {
        const size_t at = (size_t)row * Hq + h, step = (size_t)a.R * Hq;
        for (int d0 = 0; d0 < D; d0 += 128) {
            const int d = min(d0 + 2 * lane, D - 2);
            float mx = -INFINITY, l = 0.f, x = 0.f, y = 0.f;
            for (int k0 = 0; k0 < part.splits; k0 += 64) {
                const int cnt = min(64, part.splits - k0);
                const float2 mine = lane < cnt ? part.ml[at + (k0 + lane) * step] : make_float2(-INFINITY, 0.f);
                const float m_new = fmaxf(mx, wave_max(mine.x));
                const float f = mine.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mine.x - m_new), old = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx - m_new);
                l = l * old + wave_sum(f * mine.y);
                x *= old;
                y *= old;
                for (int k = 0; k < cnt; k += 8) {  // eight loads in flight; behind the last split: the last again, left out
                    float2 o[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = *(const float2 *)(part.o + (at + (k0 + min(k + e, cnt - 1)) * step) * D + d);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float fk = __shfl(f, (k + e) & 63, 64);  // 0 behind the last
                        const uint32_t there = (uint32_t)(k + e - cnt >> 31);  // bits, not a condition: that would hold up the loads
                        x += fk * __uint_as_float(__float_as_uint(o[e].x) & there);
                        y += fk * __uint_as_float(__float_as_uint(o[e].y) & there);
                    }
                }
                mx = m_new;
            }
            const float inv = l > 0.f ? 1.f / l : 0.f;
            if (d0 + 2 * lane < D) {
                if constexpr (sizeof(T) == 2) *(uint32_t *)((T *)a.out + at * D + d) = pack_bf16(x * inv, y * inv);
                else *(float2 *)((T *)a.out + at * D + d) = make_float2(x * inv, y * inv);
            }
        }
    }
}

// Tiles of 16 queries of `rows` rows, and in how many groups an item each takes them.
struct TileGroups { int64_t tiles; int groups; };
constexpr int kWgs = 256, kItemCost = 12, kMaxSplits = 32, kMaxTileGroups = 64;
TileGroups tile_groups_for(const Dims &dm, int64_t pairs, int64_t rows) {
    const bool mfma = on_matrix_cores(dm);
    const int64_t tiles = std::max<int64_t>(1, (rows * (dm.Hq / dm.Hkv) + 15) / 16);
    int groups = (int)std::min<int64_t>(mfma ? (tiles + 2) / 3 : tiles, kMaxTileGroups);
    // few lists: tiles apart while their items and 8 splits fit on the chip at once (1 sequence, 8 kv-heads, 3 tiles, 128 blocks: 11.5 -> 8.5 us; 2 of 2 tiles, 64 blocks: 9.2 -> 8.3)
    while (mfma && groups < std::min<int64_t>(tiles, 3) && pairs * (groups + 1) * 8 <= kWgs) ++groups;
    return {tiles, groups};
}

// Splits of the lists: the number whose rounds of workgroups cost least.  Unit: what 16 tokens take a workgroup that is alone, 0.15 us on the 128 kernel
// and 0.25 on the float32 one; an item costs kItemCost besides, a join 4 us and 1 us for each 2000 rows' heads (64 sequences, 340 rows of 32 heads: 9.6).  Next to others HBM is shared: 256 blocks of 192 lists take the 128 kernel 76 us in one
// part (twice the unit; in four parts, three rounds, 88), of 96 lists 47 (two parts 42), of 8 lists 39 (eight parts 11); 32 blocks of 96 lists the float32 one 15 us (four
// parts 12).  The chip holds 1 workgroup to a CU of the 128 kernel and 3 of the float32 one (counted on 4: 33 for 29 us on its 25 sequences above, on 8 35).
// A sum's order goes by the splits, so they go by the arrays' sizes alone: the rows are taken to be spread evenly over the sequences, whatever seq_rows says.
int splits_for(const Dims &dm, int S, int R, int max_selected) {
    const bool mfma = on_matrix_cores(dm);
    const int64_t lists = (int64_t)S * dm.Hkv, pairs = lists * tile_groups_for(dm, lists, ((int64_t)R + S - 1) / S).groups;
    const int least = (max_selected + kItemBlocks - 1) / kItemBlocks, parts = mfma ? 1 : dm.Bk / 16;
    const int limit = (int)std::min<int64_t>({kMaxSplits, max_selected, ((int64_t)max_selected * parts + 7) / 8});  // 8 times 16 tokens: a group of two or two units to a wave
    const int64_t wgs = mfma ? kWgs : 3 * kWgs;
    const auto round = [&](int64_t running, int64_t blocks) { return 128 * kItemCost + blocks * (128 + (mfma ? std::max<int64_t>(running - 64, 0) : running * 5 / 8)); };
    const int64_t join = 128 * (mfma ? 24 : 16) + 128 * (int64_t)R * dm.Hq / (mfma ? 300 : 500);
    int best = 0;
    int64_t cost = 0;
    for (int n = std::max(1, least); n <= std::max(least, limit) || !best; ++n) {
        const int64_t items = pairs * n, blocks = (int64_t)((max_selected + n - 1) / n) * parts;
        const int64_t t = items / wgs * round(wgs, blocks) + (items % wgs ? round(items % wgs, blocks) : 0) + (n > 1 ? join : 0);
        if (!best || t < cost) {
            best = n;
            cost = t;
        }
    }
    return best;
}

template <int NT, bool KV8>
hipError_t launch_mfma(const Dims &dm, const BlockAttnArgs &a, const SplitOut &part, hipStream_t st) {
    const size_t lds = 4 * Image<NT>::kBytes + 2 * NT * kKS * 1024;
    if (lds > 64 * 1024) {  // each device has its own copy of the kernel
        static std::atomic<uint64_t> set{0};
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        const uint64_t bit = 1ull << (dev & 63);
        if (dev > 63 || !(set.load() & bit)) {
            e = hipFuncSetAttribute((const void *)k_block_attn<NT, KV8>, hipFuncAttributeMaxDynamicSharedMemorySize, 150 * 1024);
            if (e != hipSuccess) return e;
            if (dev <= 63) set.fetch_or(bit);
        }
    }
    const float scale_log2 = kLog2e / sqrtf((float)kD) * (KV8 ? dm.k_scale : 1.f);
    hipLaunchKernelGGL((k_block_attn<NT, KV8>), dim3(std::min(part.n_items, kWgs)), dim3(256), lds, st, a, part, dm.Hq, dm.Hkv, scale_log2, KV8 ? dm.v_scale : 1.f);
    return hipGetLastError();
}

}  // namespace

bool block_attn_fast(const Dims &dm) { return dm.Bk % 16 == 0 && dm.D % 16 == 0; }

size_t block_attn_workspace(const Dims &dm, int S, int R, int max_selected) {
    if (!block_attn_fast(dm) || S == 0) return 256;
    const int splits = splits_for(dm, S, R, max_selected);
    return splits > 1 ? (size_t)splits * R * dm.Hq * (dm.D + 2) * 4 + 512 : 256;
}

template <typename T, typename KT>
static hipError_t launch_f32(const Dims &dm, const BlockAttnArgs &a, const SplitOut &part, hipStream_t st) {
    const dim3 grid(a.S * dm.Hkv, part.splits, part.tile_groups);
    const float scale_log2 = kLog2e / sqrtf((float)dm.D) * (sizeof(KT) == 1 ? dm.k_scale : 1.f), v_scale = sizeof(KT) == 1 ? dm.v_scale : 1.f;
#define BLOCK_ATTN_F32(DT, EXACT) hipLaunchKernelGGL((k_block_attn_f32<T, KT, DT, EXACT>), grid, dim3(256), 0, st, a, part, dm.Hq, dm.Hkv, dm.D, dm.Bk, scale_log2, v_scale)
    if (dm.D == 64) BLOCK_ATTN_F32(4, true);
    else if (dm.D == 128) BLOCK_ATTN_F32(8, true);
    else if (dm.D < 128) BLOCK_ATTN_F32(8, false);
    else BLOCK_ATTN_F32(16, false);
#undef BLOCK_ATTN_F32
    return hipGetLastError();
}

hipError_t launch_block_attn(const Dims &dm, const BlockAttnArgs &a, void *workspace, hipStream_t st) {
    const int64_t pairs = (int64_t)a.S * dm.Hkv;
    const int rows = std::min(a.R, a.seq_rows ? a.seq_rows : 2 * ((a.R + a.S - 1) / a.S));  // of a sequence, about: the kernels go on where there are more
    const bool mfma = on_matrix_cores(dm);
    const TileGroups of = tile_groups_for(dm, pairs, rows);
    SplitOut part;
    part.tile_groups = of.groups;
    part.tiles = (int)std::min<int64_t>((of.tiles + of.groups - 1) / of.groups, 3);
    part.splits = splits_for(dm, a.S, a.R, a.max_selected);
    part.per = (a.max_selected + part.splits - 1) / part.splits;
    if (mfma) part.per = std::max(2, (part.per + 1) & ~1);
    part.o = (float *)workspace;
    part.ml = (float2 *)(part.o + (size_t)part.splits * a.R * dm.Hq * dm.D);
    part.n_items = (int)((pairs + 7) / 8 * 8 * part.splits * part.tile_groups);
    hipError_t e = hipSuccess;
    if (!mfma) DISPATCH_TK(dm.bf16, dm.kv8, e = (launch_f32<T, KT>(dm, a, part, st)));
    else if (part.tiles == 1) e = dm.kv8 ? launch_mfma<1, true>(dm, a, part, st) : launch_mfma<1, false>(dm, a, part, st);
    else if (part.tiles == 2) e = dm.kv8 ? launch_mfma<2, true>(dm, a, part, st) : launch_mfma<2, false>(dm, a, part, st);
    else e = dm.kv8 ? launch_mfma<3, true>(dm, a, part, st) : launch_mfma<3, false>(dm, a, part, st);
    if (e != hipSuccess || part.splits == 1) return e;
    DISPATCH_T(dm.bf16, hipLaunchKernelGGL(k_block_attn_join<T>, dim3(a.S, std::min(std::max(rows, 1), 64), (dm.Hq + 3) / 4), dim3(256), 0, st, a, part, dm.Hq, dm.D));
    return hipGetLastError();
}

hipError_t launch_block_attn_generic(const Dims &dm, const BlockAttnArgs &a, hipStream_t st) {
    const float scale = 1.f / sqrtf((float)dm.D);
    DISPATCH_TK(dm.bf16, dm.kv8, hipLaunchKernelGGL((k_block_attn_generic<T, KT>), dim3(dm.Hq, a.S), dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.D, dm.Bk, scale,
                                                    dm.k_scale, dm.v_scale));
    return hipGetLastError();
}

}  // namespace icarus
