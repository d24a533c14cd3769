// Attention of single-token rows over sequences that share a prefix.
//
// softmax over a sequence's positions is put together from parts: of each part the largest score m, l = sum 2^(s - m) and o = sum 2^(s - m) v, joined by
// l = sum 2^(m_i - m) l_i, o likewise.  A unit is a range of positions with the rows that attend to all of it: the shared blocks of a group with the rows of all its sequences (they stand one
// after the other), or the rest of a sequence with its own.  k_prefix_plan cuts the units into items of about equal work -- a range of blocks and up to kItemTiles tiles of 16
// queries (rows x heads of a kv-head) --, k_prefix_attn gives each item and kv-head a workgroup, k_prefix_join adds up a row's parts.
#include "attn_tile.h"
#include "block_util.h"
#include "branch_ops.h"

#include <algorithm>
#include <atomic>

namespace icarus {
namespace {

struct PrefixUnit { int row0, rows, seq, b0, nb, len, chunks, slot; };  // its rows; the sequence whose table has the blocks b0 .. b0 + nb - 1; positions end; parts and the first one's place
struct PrefixItem { int row0, rows, j0, seq, b0, nb, len, slot; };      // j0: the first of its queries among the unit's
struct PrefixJoin { int row0, rows, n_shared, shared, shared_rows, n_own, own, pad; };  // a sequence's rows; place of part k of row r: shared + k * shared_rows + r, then own + k * rows + r - row0
constexpr int kPlanThreads = 1024, kMostBlocks = 1024;                   // blocks of an item, at most

struct PrefixPlan {
    PrefixUnit *units;  // [G] shared blocks of a group, [S] the rest of a sequence
    int *seq_group;     // [S], -1: none
    PrefixItem *items;
    int *n_items;
    PrefixJoin *join;   // [S]
    float *o;           // parts [slot][Hq][D], slot: unit's first + part * rows + row
    float2 *ml;         // [slot][Hq]: maximum in log2 units, sum
    int cap_items;
    int64_t cap_slots;
    int tiles, target, step;  // tiles of an item; items wanted to a kv-head; blocks of an item are a multiple of step
};

// Exclusive sum over the workgroup of one value per thread; *total: of all.
__device__ __forceinline__ int64_t plan_scan(int64_t v, int64_t *red, int64_t *total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) red[w] = x;
    __syncthreads();
    int64_t before = 0, sum = 0;
    for (int i = 0; i < kPlanThreads / 64; ++i) {
        if (i < w) before += red[i];
        sum += red[i];
    }
    *total = sum;
    return before + x - v;
}

__global__ void __launch_bounds__(kPlanThreads) k_prefix_plan(PrefixAttnArgs a, PrefixPlan p, int g, int Bk) {
    __shared__ int begin[kPlanThreads], end[kPlanThreads], least[kPlanThreads], first[kPlanThreads], live[kPlanThreads];
    __shared__ int64_t red[kPlanThreads / 64];
    const int t = threadIdx.x;
    const int64_t room = (int64_t)a.max_blocks * Bk;
    const auto len_of = [&](int s) { return (int)min((int64_t)max(a.kv_lens[s], 0), room); };
    const auto rows_of = [&](int s0, int s1, int *row0) {
        *row0 = min(max(a.row_start[s0], 0), a.R);
        return min(max(a.row_start[s1], *row0), a.R) - *row0;
    };
    for (int s = t; s < a.S; s += kPlanThreads) {
        p.seq_group[s] = -1;
        p.units[a.G + s] = PrefixUnit{0, 0, s, 0, 0, 0, 0, 0};
    }
    for (int g0 = 0; g0 < a.G; g0 += kPlanThreads) {
        const int n = min(kPlanThreads, a.G - g0);
        __syncthreads();
        if (t < n) {
            begin[t] = min(max(a.group_start[g0 + t], 0), a.S);
            end[t] = min(max(a.group_start[g0 + t + 1], begin[t]), a.S);
            least[t] = first[t] = INT32_MAX;
            live[t] = 0;
        }
        __syncthreads();
        for (int s = begin[0] + t; s < end[n - 1]; s += kPlanThreads) {
            int lo = 0, hi = n - 1;  // the last group that begins at or before s
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (begin[mid] <= s) lo = mid;
                else hi = mid - 1;
            }
            if (s >= end[lo]) continue;
            p.seq_group[s] = g0 + lo;
            const int len = len_of(s);
            if (len > 0) {
                atomicMin(&least[lo], len);
                atomicMin(&first[lo], s);
                atomicAdd(&live[lo], 1);
            }
        }
        __syncthreads();
        if (t < n) {
            PrefixUnit u{0, 0, first[t], 0, 0, 0, 0, 0};
            u.rows = rows_of(begin[t], end[t], &u.row0);
            const int shared = live[t] > 1 ? min(max(a.prefix_lens[g0 + t], 0), least[t]) / Bk : 0;  // one sequence reads all of its blocks by itself
            u.nb = u.rows ? shared : 0;
            u.len = shared * Bk;
            p.units[g0 + t] = u;
            least[t] = shared;
        }
        __syncthreads();
        for (int s = begin[0] + t; s < end[n - 1]; s += kPlanThreads) {
            const int group = p.seq_group[s] - g0;
            if (group < 0 || group >= n) continue;
            PrefixUnit u{0, 0, s, least[group], 0, len_of(s), 0, 0};
            u.rows = rows_of(s, s + 1, &u.row0);
            u.nb = u.rows ? max(u.len / Bk + (u.len % Bk != 0) - u.b0, 0) : 0;
            p.units[a.G + s] = u;
        }
    }
    __syncthreads();
    const int n_units = a.G + a.S;
    const auto groups_of = [&](const PrefixUnit &u) { return ((int)(((int64_t)u.rows * g + 15) / 16) + p.tiles - 1) / p.tiles; };
    int64_t work = 0, total;
    for (int i = t; i < n_units; i += kPlanThreads) {
        const PrefixUnit u = p.units[i];
        work += (int64_t)u.nb * groups_of(u);
    }
    plan_scan(work, red, &total);
    int per = (int)min((total + p.target - 1) / p.target, (int64_t)kMostBlocks);
    per = max((per + p.step - 1) / p.step, 1) * p.step;
    int64_t items = 0, slots = 0;
    for (int i0 = 0; i0 < n_units; i0 += kPlanThreads) {
        const int i = i0 + t;
        PrefixUnit u{};
        if (i < n_units) u = p.units[i];
        const int tg = groups_of(u);
        int mine = per;
        if (u.nb) {  // even parts
            const int chunks = (u.nb + per - 1) / per;
            mine = ((u.nb + chunks - 1) / chunks + p.step - 1) / p.step * p.step;
            u.chunks = (u.nb + mine - 1) / mine;
        }
        int64_t all_items, all_slots;
        const int64_t at = items + plan_scan((int64_t)u.chunks * tg, red, &all_items), slot = slots + plan_scan((int64_t)u.chunks * u.rows, red, &all_slots);
        if (at + (int64_t)u.chunks * tg > p.cap_items || slot + (int64_t)u.chunks * u.rows > p.cap_slots) u.chunks = 0;  // only where rows or groups overlap
        u.slot = (int)slot;
        if (i < n_units) p.units[i] = u;
        // the items of these units, a thread to an item
        begin[t] = (int)min(at, (int64_t)p.cap_items);
        end[t] = mine;
        __syncthreads();
        const int from = (int)min(items, (int64_t)p.cap_items), to = (int)min(items + all_items, (int64_t)p.cap_items);
        for (int k = from + t; k < to; k += kPlanThreads) {
            int lo = 0, hi = kPlanThreads - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (begin[mid] <= k) lo = mid;
                else hi = mid - 1;
            }
            const PrefixUnit v = p.units[i0 + lo];
            const int groups = max(groups_of(v), 1), chunk = (k - begin[lo]) / groups, b = chunk * end[lo];
            PrefixItem x{v.row0, v.rows, (k - begin[lo]) % groups * p.tiles * 16, v.seq, v.b0 + b, chunk < v.chunks ? min(end[lo], v.nb - b) : 0, v.len, v.slot + chunk * v.rows};
            p.items[k] = x;
        }
        __syncthreads();
        items += all_items;
        slots += all_slots;
    }
    if (t == 0) *p.n_items = (int)min(items, (int64_t)p.cap_items);
    for (int s = t; s < a.S; s += kPlanThreads) {
        PrefixJoin j{};
        const int group = p.seq_group[s];
        if (group >= 0) {
            const PrefixUnit u = p.units[a.G + s], v = p.units[group];
            j = PrefixJoin{u.row0, u.rows, v.chunks, v.slot - v.row0, v.rows, u.chunks, u.slot, 0};
            if (u.len == 0) j.n_shared = j.n_own = 0;  // an empty sequence among others: the shared parts are not its own
        }
        p.join[s] = j;
    }
}

// The same for up to THREADS sequences and groups: one of each to a thread, everything in registers and LDS after one round of reads.
__device__ __forceinline__ int sat(int64_t v) { return (int)min(v, (int64_t)1 << 30); }
template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_prefix_plan_small(PrefixAttnArgs a, PrefixPlan p, int g, int Bk) {
    constexpr int WAVES = THREADS / 64;
    __shared__ int begin[THREADS], end[THREADS], least[THREADS], first[THREADS], live[THREADS], row_at[THREADS + 1], at_item[2 * THREADS], red[4][WAVES];
    __shared__ int64_t red_work[WAVES];
    __shared__ PrefixUnit units[2 * THREADS];
    __shared__ int size_of[2 * THREADS];  // blocks of an item of the unit
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const bool is_seq = t < a.S, is_group = t < a.G;
    const int len = is_seq ? (int)min((int64_t)max(a.kv_lens[t], 0), (int64_t)a.max_blocks * Bk) : 0;
    const int row_here = is_seq ? min(max(a.row_start[t], 0), a.R) : 0, row_last = t == 0 ? min(max(a.row_start[a.S], 0), a.R) : 0;
    const int group_begin = is_group ? min(max(a.group_start[t], 0), a.S) : a.S;
    const int group_end = is_group ? min(max(a.group_start[t + 1], group_begin), a.S) : a.S;
    const int prefix = is_group ? max(a.prefix_lens[t], 0) : 0;
    begin[t] = group_begin;
    end[t] = group_end;
    least[t] = first[t] = INT32_MAX;
    live[t] = 0;
    if (is_seq) row_at[t] = row_here;
    if (t == 0) row_at[a.S] = row_last;
    __syncthreads();
    int group = -1;
    if (is_seq) {  // the last group that begins at or before this sequence
        int lo = 0, hi = a.G - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (begin[mid] <= t) lo = mid;
            else hi = mid - 1;
        }
        if (begin[lo] <= t && t < end[lo]) group = lo;
        if (group >= 0 && len > 0) {
            atomicMin(&least[group], len);
            atomicMin(&first[group], t);
            atomicAdd(&live[group], 1);
        }
    }
    __syncthreads();
    PrefixUnit u{}, v{};  // of the group, of the sequence
    if (is_group) {
        const int shared = live[t] > 1 ? min(prefix, least[t]) / Bk : 0;  // one sequence reads all of its blocks by itself
        u.row0 = row_at[group_begin];
        u.rows = max(row_at[group_end] - u.row0, 0);
        u.seq = first[t];
        u.nb = u.rows ? shared : 0;
        u.len = shared * Bk;
        least[t] = shared;
    }
    __syncthreads();
    if (group >= 0) {
        v.row0 = row_here;
        v.rows = max(row_at[t + 1] - row_here, 0);
        v.seq = t;
        v.b0 = least[group];
        v.len = len;
        v.nb = v.rows ? max(len / Bk + (len % Bk != 0) - v.b0, 0) : 0;
    }
    const auto groups_of = [&](const PrefixUnit &y) { return ((int)(((int64_t)y.rows * g + 15) / 16) + p.tiles - 1) / p.tiles; };
    const int tg_u = groups_of(u), tg_v = groups_of(v);
    int64_t work = (int64_t)u.nb * tg_u + (int64_t)v.nb * tg_v;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) work += __shfl_xor(work, o, 64);
    if (lane == 0) red_work[w] = work;
    __syncthreads();
    int64_t total = 0;
    for (int i = 0; i < WAVES; ++i) total += red_work[i];
    int per = (int)min((total + p.target - 1) / p.target, (int64_t)kMostBlocks);
    per = max((per + p.step - 1) / p.step, 1) * p.step;
    const auto cut = [&](PrefixUnit &y) {  // even parts
        if (y.nb == 0) return per;
        const int chunks = (y.nb + per - 1) / per, mine = ((y.nb + chunks - 1) / chunks + p.step - 1) / p.step * p.step;
        y.chunks = (y.nb + mine - 1) / mine;
        return mine;
    };
    size_of[t] = cut(u);
    size_of[THREADS + t] = cut(v);
    const int n[4] = {sat((int64_t)u.chunks * tg_u), sat((int64_t)v.chunks * tg_v), sat((int64_t)u.chunks * u.rows), sat((int64_t)v.chunks * v.rows)};
    int x[4] = {n[0], n[1], n[2], n[3]}, all[4];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int y = __shfl_up(x[k], o, 64);
            if (lane >= o) x[k] = min(x[k] + y, 1 << 30);
        }
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < 4; ++k) red[k][w] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        int before = 0, sum = 0;
        for (int i = 0; i < WAVES; ++i) {
            if (i < w) before = min(before + red[k][i], 1 << 30);
            sum = min(sum + red[k][i], 1 << 30);
        }
        x[k] = min(before + x[k], 1 << 30);  // with this thread's own
        all[k] = sum;
    }
    const int64_t item_u = (int64_t)x[0] - n[0], item_v = (int64_t)all[0] + x[1] - n[1], slot_u = (int64_t)x[2] - n[2], slot_v = (int64_t)all[2] + x[3] - n[3];
    if (item_u + n[0] > p.cap_items || slot_u + n[2] > p.cap_slots) u.chunks = 0;  // only where rows or groups overlap
    if (item_v + n[1] > p.cap_items || slot_v + n[3] > p.cap_slots) v.chunks = 0;
    u.slot = (int)slot_u;
    v.slot = (int)slot_v;
    at_item[t] = (int)min(item_u, (int64_t)p.cap_items);
    at_item[THREADS + t] = (int)min(item_v, (int64_t)p.cap_items);
    units[t] = u;
    units[THREADS + t] = v;
    __syncthreads();
    const int n_items = (int)min((int64_t)all[0] + all[1], (int64_t)p.cap_items);
    for (int k = t; k < n_items; k += THREADS) {
        int lo = 0, hi = 2 * THREADS - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (at_item[mid] <= k) lo = mid;
            else hi = mid - 1;
        }
        const PrefixUnit y = units[lo];
        const int groups = max(groups_of(y), 1), chunk = (k - at_item[lo]) / groups, size = size_of[lo], b = chunk * size;
        p.items[k] = PrefixItem{y.row0, y.rows, (k - at_item[lo]) % groups * p.tiles * 16, y.seq, y.b0 + b, chunk < y.chunks ? min(size, y.nb - b) : 0, y.len, y.slot + chunk * y.rows};
    }
    if (t == 0) *p.n_items = n_items;
    if (is_seq) {
        PrefixJoin j{};
        if (group >= 0) {
            const PrefixUnit &y = units[group];
            j = PrefixJoin{v.row0, v.rows, len ? y.chunks : 0, y.slot - y.row0, y.rows, len ? v.chunks : 0, v.slot, 0};
        }
        p.join[t] = j;
    }
}

// 16-byte LDS-direct load: lane i copies 16 bytes from its own global address to LDS byte lds_base + 16 i (lds_base wave-uniform, passed in m0); the load counts in vmcnt until the
// data is in LDS.
__device__ __forceinline__ void to_lds16(const void *g, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_base), "v"(g) : "memory");
}

// ---- matrix cores: bf16 storage, head_dim 128, blocks of 16 -------------------------------------------------------------
// Keys and values of a stage go straight to LDS as the fragments that the matrix cores take, the next stage's while this one is multiplied; two workgroups to a CU.  The waves
// share the item's tiles: of more than four, each wave has two and multiplies every group of the stage; of up to four, a pair of waves has each tile and each wave of it half of the groups,
// and the two states are put together at the end.
constexpr int kItemTiles = 8, kNT = 2;
template <bool KV8> constexpr int kStageGroups = KV8 ? 4 : 2;  // 32 tokens each: a stage is 32 KB

// One group of 32 tokens for N query tiles, its fragments read from LDS as they are needed: scores of all tiles, one look whether any softmax reference has to move (rare: see
// compute_group), the weights, and the values' product.  there: tokens of this lane's block (masked only).
//
// A weight of one bfloat16 (half a step, 2^-8) would add as much error, squared, as the output's own rounding; the weight is cut to 8 bits and the rest goes through a second
// product (2^-15).  The rest is greater than 0 (by 2^-20 of the weight) wherever the weight is, so that an infinite value stays what it is.  FP8 values, whose codes are float16
// numbers too: weights in float16 (2^-11), kLift powers of two up, to at most 2^14, so that only weights below 2^-20 of the reference lose bits to float16's least exponent.
constexpr float kLift = 6.f;
// By hand: for fmaxf the compiler first turns every score into itself, in case it were a signalling NaN.  Only for operands that no matrix instruction has just written: the compiler does
// not keep the distance that such a result needs before it is read in front of assembly (settled()).
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// Sixteen wait states behind the products: a result of a 16 x 16 x 32 product may be read after fewer.
__device__ __forceinline__ void settled(f32x4 (&s)[1][2]) { asm volatile("s_nop 15" : "+v"(s[0][0]), "+v"(s[0][1])); }
__device__ __forceinline__ void settled(f32x4 (&s)[2][2]) { asm volatile("s_nop 15" : "+v"(s[0][0]), "+v"(s[0][1]), "+v"(s[1][0]), "+v"(s[1][1])); }
template <int N, bool KV8, bool masked>
__device__ __forceinline__ void prefix_group(State<kNT> &st, const char *__restrict__ src, const bf16x8 (&qr)[kNT][kKS], int there, float scale_log2, int lane) {
    const int m = lane & 15, q = lane >> 4, t0 = 8 * (q & 1);
    f32x4 sc[N][2];
#pragma unroll
    for (int qt = 0; qt < N; ++qt)
        sc[qt][0] = sc[qt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (KV8) {
#pragma unroll
        for (int sl = 0; sl < 2; ++sl) {
            const uint4 r0 = *(const uint4 *)(src + sl * 1024 + lane * 16), r1 = *(const uint4 *)(src + (2 + sl) * 1024 + lane * 16);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bf16x8 k0 = h ? cvt8(r0.z, r0.w) : cvt8(r0.x, r0.y), k1 = h ? cvt8(r1.z, r1.w) : cvt8(r1.x, r1.y);
#pragma unroll
                for (int qt = 0; qt < N; ++qt) {
                    sc[qt][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qr[qt][2 * sl + h], sc[qt][0], 0, 0, 0);
                    sc[qt][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qr[qt][2 * sl + h], sc[qt][1], 0, 0, 0);
                }
            }
        }
    } else {
#pragma unroll
        for (int ks = 0; ks < kKS; ++ks) {
            const bf16x8 k0 = *(const bf16x8 *)(src + ks * 1024 + lane * 16), k1 = *(const bf16x8 *)(src + (kKS + ks) * 1024 + lane * 16);
#pragma unroll
            for (int qt = 0; qt < N; ++qt) {
                sc[qt][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qr[qt][ks], sc[qt][0], 0, 0, 0);
                sc[qt][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qr[qt][ks], sc[qt][1], 0, 0, 0);
            }
        }
    }
    float mx[N];
    bool move = false;
    settled(sc);
#pragma unroll
    for (int qt = 0; qt < N; ++qt) {
        if (masked)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (t0 + i >= there) sc[qt][i >> 2][i & 3] = -INFINITY;
        const f32x4 a = sc[qt][0], b = sc[qt][1];
        mx[qt] = max3(max3(a[0], a[1], a[2]), max3(a[3], b[0], b[1]), max3(b[2], b[3], b[3])) * scale_log2;
        move |= mx[qt] > st.m[qt] + kSlack;
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
            for (int dt = 0; dt < kDT; ++dt) st.o[dt][qt] *= c;
        }
    }
    uint4 hi[N], lo[N];
#pragma unroll
    for (int qt = 0; qt < N; ++qt) {
        const float m_ref = (st.m[qt] == -INFINITY ? 0.f : st.m[qt]) - (KV8 ? kLift : 0.f);  // nothing yet: every weight 0
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[qt][i >> 2][i & 3], scale_log2, -m_ref));
        st.l[qt] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));  // as they are
        if constexpr (KV8) {
            hi[qt] = make_uint4(pack_f16(e[0], e[1]), pack_f16(e[2], e[3]), pack_f16(e[4], e[5]), pack_f16(e[6], e[7]));
        } else {
            uint32_t p[4], rest[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t x = __float_as_uint(e[2 * i]) & 0xffff0000u, y = __float_as_uint(e[2 * i + 1]) & 0xffff0000u;
                p[i] = x >> 16 | y;
                rest[i] = pack_bf16(__builtin_fmaf(e[2 * i], 1.f + 0x1p-20f, -__uint_as_float(x)), __builtin_fmaf(e[2 * i + 1], 1.f + 0x1p-20f, -__uint_as_float(y)));
            }
            hi[qt] = make_uint4(p[0], p[1], p[2], p[3]);
            lo[qt] = make_uint4(rest[0], rest[1], rest[2], rest[3]);
        }
    }
    uint32_t keep[4];  // places behind the last token may hold anything
    if (masked) {
#pragma unroll
        for (int i = 0; i < 4; ++i) keep[i] = (t0 + 2 * i < there ? 0xffffu : 0u) | (t0 + 2 * i + 1 < there ? 0xffff0000u : 0u);
    }
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) {
        uint4 v;
        if constexpr (KV8) {
            const uint2 r = *(const uint2 *)(src + 4096 + (q >> 1) * 2048 + (16 * dt + m) * 16 + t0);
            v = cvt8_f16(r.x, r.y);
        } else {
            v = *(const uint4 *)(src + (2 * kKS + dt) * 1024 + lane * 16);
        }
        if (masked) v = make_uint4(v.x & keep[0], v.y & keep[1], v.z & keep[2], v.w & keep[3]);
#pragma unroll
        for (int qt = 0; qt < N; ++qt) {
            if constexpr (KV8) {
                st.o[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, hi[qt]), st.o[dt][qt], 0, 0, 0);
            } else {
                st.o[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, hi[qt]), st.o[dt][qt], 0, 0, 0);
                st.o[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, lo[qt]), st.o[dt][qt], 0, 0, 0);
            }
        }
    }
}

template <bool KV8>
__global__ void __launch_bounds__(256, 2) k_prefix_attn(PrefixAttnArgs a, PrefixPlan p, int Hq, int Hkv, float scale_log2, float v_scale) {
    constexpr int SG = kStageGroups<KV8>, SB = 2 * SG, kGroupBytes = KV8 ? 8192 : 16384, kStageBytes = SG * kGroupBytes;
    static_assert(2 * Image<kNT>::kBytes <= 2 * kStageBytes, "the states of two waves fit the ring");
    __shared__ __attribute__((aligned(1024))) char ring[2 * kStageBytes];
    __shared__ int ids[kMostBlocks + SB], found[4], part_id;
    const int i = blockIdx.x / Hkv, c = blockIdx.x % Hkv;
    if (i >= *p.n_items) return;
    const PrefixItem x = p.items[i];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, q = lane >> 4, g = Hq / Hkv;
    const int G = x.rows * g, tiles = min((G - x.j0 + 15) >> 4, kItemTiles);
    if (x.nb <= 0) return;
    // this wave's tiles
    const bool apart = tiles > 4, single = tiles <= 2;
    const int tile0 = apart ? 2 * w : single ? (w & 1) : 2 * (w & 1), n_mine = max(min(single ? 1 : 2, tiles - tile0), 0);
    bf16x8 qr[kNT][kKS];
#pragma unroll
    for (int qt = 0; qt < kNT; ++qt) {
        const int j = x.j0 + 16 * (tile0 + qt) + m;
        const bf16_t *qp = (const bf16_t *)a.q + ((size_t)(x.row0 + j / g) * Hq + c * g + j % g) * kD;
#pragma unroll
        for (int ks = 0; ks < kKS; ++ks) qr[qt][ks] = qt < n_mine && j < G ? *(const bf16x8 *)(qp + (KV8 ? 64 * (ks >> 1) + 16 * q + 8 * (ks & 1) : 32 * ks + 8 * q)) : zero8();
    }
    // The blocks, without those outside the pool: full ones, then the one that ends early, if there is one (the last).  Their order does not matter to the sums.
    const int part_n = min(kBk, x.len - (x.b0 + x.nb - 1) * kBk);
    int n_full = 0;
    if (threadIdx.x == 0) part_id = -1;
    for (int b0 = 0; b0 < x.nb; b0 += 256) {
        const int b = b0 + threadIdx.x, id = b < x.nb ? a.bt[(size_t)x.seq * a.max_blocks + x.b0 + b] : -1;
        const bool there = id >= 0 && id < a.num_blocks, full = there && (b < x.nb - 1 || part_n == kBk);
        const unsigned long long mask = __ballot(full);
        __syncthreads();
        if (lane == 0) found[w] = __popcll(mask);
        if (there && !full) part_id = id;
        __syncthreads();
        int at = n_full + __popcll(mask & ((1ull << lane) - 1));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k < w) at += found[k];
            n_full += found[k];
        }
        if (full) ids[at] = id;
    }
    n_full = __builtin_amdgcn_readfirstlane(n_full);
    const int last = __builtin_amdgcn_readfirstlane(part_id), n_blk = n_full + (last >= 0);
    if (threadIdx.x < SB) ids[n_full + threadIdx.x] = threadIdx.x == 0 && last >= 0 ? last : 0;  // behind the last block: something to load
    State<kNT> st;
#pragma unroll
    for (int qt = 0; qt < kNT; ++qt) {
        st.m[qt] = -INFINITY;
        st.l[qt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) st.o[dt][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const uint32_t ring0 = (uint32_t)(size_t)(__attribute__((address_space(3))) char *)ring;
    // This wave's quarter of a group: w = 0, 1 the key rows of tile w; w = 2, 3 value rows (bf16: four d tiles of both blocks; FP8: one block).
    const auto request = [&](int stage) {
        const uint32_t to = ring0 + (stage & 1) * kStageBytes;
#pragma unroll
        for (int gi = 0; gi < SG; ++gi) {
            const int *id2 = ids + stage * SB + 2 * gi;
            if constexpr (KV8) {
                const size_t head = (size_t)2 * kBk * kD;
                const int sel = w < 2 ? m >> 3 : w - 2;
                const uint8_t *blk = (const uint8_t *)a.pool + ((size_t)id2[sel] * Hkv + c) * head;
                const uint8_t *from = w < 2 ? blk + (8 * ((m >> 2) & 1) + (m & 3) + 4 * w) * kD + 16 * q : blk + kBk * kD + 16 * lane;
#pragma unroll
                for (int k = 0; k < 2; ++k) to_lds16(from + k * (w < 2 ? 64 : 1024), to + gi * kGroupBytes + (2 * w + k) * 1024);
            } else {
                const size_t head = (size_t)2 * kBk * kD;
                const int sel = w < 2 ? m >> 3 : q >> 1;
                const bf16_t *blk = (const bf16_t *)a.pool + ((size_t)id2[sel] * Hkv + c) * head;
                const bf16_t *from = w < 2 ? blk + (8 * ((m >> 2) & 1) + (m & 3) + 4 * w) * kD + 8 * q : blk + kBk * kD + (64 * (w - 2) + m) * kBk + 8 * (q & 1);
#pragma unroll
                for (int k = 0; k < 4; ++k) to_lds16(from + k * (w < 2 ? 32 : 16 * kBk), to + gi * kGroupBytes + (4 * w + k) * 1024);
            }
        }
    };
    const auto meet = [&] {  // what this wave brought has landed in LDS, and so has what the others brought
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
        __syncthreads();
    };
    const int stages = (n_blk + SB - 1) / SB, plain = n_full / SB;  // stages, and those without masks
    __syncthreads();  // ids
    if (stages) request(0);
    meet();
    const auto walk = [&](auto n_tiles, auto all) {
        constexpr int N = decltype(n_tiles)::value;
        constexpr bool ALL = decltype(all)::value;  // this wave takes all groups of a stage, else every other one
        const auto group = [&](auto masked, int s, int gi) {
            constexpr bool M = decltype(masked)::value;
            const int b = s * SB + 2 * gi + (q >> 1);  // this lane's block
            const int there = !M ? kBk : b < n_full ? kBk : b < n_blk ? part_n : 0;
            if constexpr (N > 0) prefix_group<N, KV8, M>(st, ring + (s & 1) * kStageBytes + gi * kGroupBytes, qr, there, scale_log2, lane);
        };
        int s = 0;
#pragma nounroll
        for (; s < plain; ++s) {
            if (s + 1 < stages) request(s + 1);
#pragma unroll
            for (int gi = 0; gi < (ALL ? SG : SG / 2); ++gi) group(std::false_type(), s, ALL ? gi : 2 * gi + (w >> 1));
            meet();
        }
#pragma nounroll
        for (; s < stages; ++s) {  // at most one
#pragma nounroll
            for (int gi = ALL ? 0 : w >> 1; gi < SG; gi += ALL ? 1 : 2)
                if (s * SB + 2 * gi < n_blk) group(std::true_type(), s, gi);
            meet();
        }
    };
    if (n_mine == 0) walk(std::integral_constant<int, 0>(), std::true_type());
    else if (apart && n_mine == 1) walk(std::integral_constant<int, 1>(), std::true_type());
    else if (apart) walk(std::integral_constant<int, 2>(), std::true_type());
    else if (n_mine == 1) walk(std::integral_constant<int, 1>(), std::false_type());
    else walk(std::integral_constant<int, 2>(), std::false_type());
    if (!apart) {  // the states of waves w and w + 2
        char *img = ring + (w & 1) * Image<kNT>::kBytes;
        if (w >= 2) image_store<kNT>(st, img, lane);
        __syncthreads();
        if (w >= 2) return;
        const float2 *ml = (const float2 *)(img + Image<kNT>::kO * 16);
#pragma unroll
        for (int qt = 0; qt < kNT; ++qt) {
            const float2 other = ml[qt * 64 + lane];
            const float mx = fmaxf(st.m[qt], other.x);
            const float f = st.m[qt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.m[qt] - mx), fo = other.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(other.x - mx);
            st.m[qt] = mx;
            st.l[qt] = f * st.l[qt] + fo * other.y;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) st.o[dt][qt] = f * st.o[dt][qt] + fo * ((const f32x4 *)img)[(dt * kNT + qt) * 64 + lane];
        }
    }
#pragma unroll
    for (int qt = 0; qt < kNT; ++qt) {
        float l = st.l[qt];
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        const int j = x.j0 + 16 * (tile0 + qt) + m;
        if (qt >= n_mine || j >= G) continue;
        const size_t at = (size_t)(x.slot + j / g) * Hq + c * g + j % g;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) *(f32x4 *)(p.o + at * kD + 16 * dt + 4 * q) = st.o[dt][qt] * v_scale;
        if (q == 0) p.ml[at] = make_float2(st.m[qt], l);
    }
}

bool on_matrix_cores(const Dims &dm) { return dm.bf16 && dm.D == kD && dm.Bk == kBk; }

// ---- block and head sizes that are multiples of 16: matrix cores in float32 ------------------------------------------------------
// For float32, head sizes other than 128 and blocks of more than 16 tokens.  An item has a tile of 16 queries; a wave takes sixteen tokens of a block in turn.  Products of 16 x 16 x 4 with the
// transposed operands, see k_block_attn_f32: scores of keys [token][channel] times queries [channel][query] leave lane t + 16 p query t's scores of tokens 4 p .. 4 p + 3, which are
// at once the right operand of the values' product, so nothing passes through LDS until the waves join.
template <typename T, typename KT, int DT, bool EXACT>  // tiles of 16 channels: at most DT, or DT exactly
__global__ void __launch_bounds__(256) k_prefix_attn_f32(PrefixAttnArgs a, PrefixPlan p, int Hq, int Hkv, int D_, int Bk, float scale_log2, float v_scale) {
    typedef typename Quad<KT>::raw Raw;
    __shared__ f32x4 image[2][DT][64];
    __shared__ int2 ids[kMostBlocks];  // block of the pool, and its tokens
    __shared__ float image_m[4][16], image_l[4][16];
    const int item = blockIdx.x / Hkv, c = blockIdx.x % Hkv;
    if (item >= *p.n_items) return;
    const PrefixItem x = p.items[item];
    if (x.nb <= 0) return;
    const int D = EXACT ? 16 * DT : D_, d16 = D / 16;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, p4 = 4 * (lane >> 4), g = Hq / Hkv;
    const int G = x.rows * g, parts = Bk / 16, units = x.nb * parts, step = 4 / parts, step_parts = 4 % parts;  // sixteen tokens of a block are a unit
    for (int b = threadIdx.x; b < x.nb; b += 256) {
        int2 v = make_int2(0, 0);
        const int id = a.bt[(size_t)x.seq * a.max_blocks + x.b0 + b];
        if (id >= 0 && id < a.num_blocks) v = make_int2(id, (int)min((int64_t)Bk, x.len - (int64_t)(x.b0 + b) * Bk));
        ids[b] = v;
    }
    const int j = min(x.j0 + t, G - 1);
    const size_t row = (size_t)(x.row0 + j / g) * Hq + c * g + j % g;
    float q[DT][4];
#pragma unroll
    for (int d = 0; d < DT; ++d)
        if (EXACT || d < d16) Quad<T>::get(*(const typename Quad<T>::raw *)((const T *)a.q + row * D + 16 * d + p4), q[d]);
    __syncthreads();
    f32x4 o[DT];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    const auto add = [&](int id, int first, int n) {  // n of the block's tokens, from `first` on
        const KT *blk = (const KT *)a.pool + ((size_t)id * Hkv + c) * 2 * Bk * D;
        const KT *kr = blk + (first + min(t, n - 1)) * D + p4, *vr = blk + (D + t) * Bk + first + p4;  // behind the last token: the last again
        Raw k[DT], v[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d)
            if (EXACT || d < d16) k[d] = *(const Raw *)(kr + 16 * d);
#pragma unroll
        for (int d = 0; d < DT; ++d)
            if (EXACT || d < d16) v[d] = *(const Raw *)(vr + (size_t)16 * Bk * d);
        f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            if (!EXACT && d >= d16) continue;
            float kf[4];
            Quad<KT>::get(k[d], kf);
#pragma unroll
            for (int u = 0; u < 4; ++u) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[u], q[d][u], sc, 0, 0, 0);
        }
        float most = -INFINITY, e[4];
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
            for (int d = 0; d < DT; ++d) o[d] *= f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            e[u] = sc[u] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sc[u] - m);
            l += e[u];
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            if (!EXACT && d >= d16) continue;
            float vf[4];
            Quad<KT>::get(v[d], vf);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (n < 16) vf[u] = p4 + u < n ? vf[u] : 0.f;  // places behind the last token may hold anything
                o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[u], e[u], o[d], 0, 0, 0);
            }
        }
    };
    int b = w / parts, part_of = w % parts;
    for (int u = w; u < units; u += 4) {
        const int id = __builtin_amdgcn_readfirstlane(ids[b].x), n = __builtin_amdgcn_readfirstlane(ids[b].y) - 16 * part_of;
        if (n > 0) add(id, 16 * part_of, min(16, n));
        b += step;
        part_of += step_parts;
        if (part_of >= parts) part_of -= parts, ++b;
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
    for (int d = 0; d < DT; ++d) o[d] *= f;
    const auto give = [&](int at) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
            if (EXACT || d < d16) image[at][d][lane] = o[d];
    };
    const auto take = [&](int at) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
            if (EXACT || d < d16) o[d] += image[at][d][lane];
    };
    if (w >= 2) give(w - 2);
    __syncthreads();
    if (w < 2) take(w);
    if (w == 1) give(1);  // its own place
    __syncthreads();
    if (w != 0) return;
    take(1);
    if (x.j0 + t >= G) return;
    const size_t at = (size_t)(x.slot + j / g) * Hq + c * g + j % g;
#pragma unroll
    for (int d = 0; d < DT; ++d)
        if (EXACT || d < d16) *(f32x4 *)(p.o + at * D + 16 * d + p4) = o[d] * v_scale;
    if (p4 == 0) p.ml[at] = make_float2(mx, sum);
}

// A row's parts put together, first the parts of the group's shared blocks, then those of its own: a wave to a head, four channels to a lane, so that D / 4 lanes take a part and the wave
// 256 / D of them at once (up to 256 channels).  Bound by its chain of two reads, so the first values are on their way before the maxima are known.
template <typename T>
__global__ void __launch_bounds__(256) k_prefix_join(PrefixAttnArgs a, PrefixPlan p, int Hq, int D) {
    const int h = blockIdx.z * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (h >= Hq) return;
    const PrefixJoin j = p.join[blockIdx.x];
    const int n = j.n_shared + j.n_own, lanes = D <= 64 ? 16 : D <= 128 ? 32 : 64, side = lane / lanes, sides = 64 / lanes, d = min((lane & (lanes - 1)) * 4, D - 4);
    for (int r = blockIdx.y; r < j.rows; r += gridDim.y) {
        const int row = j.row0 + r;
        const auto part = [&](int k) { return (size_t)(k < j.n_shared ? j.shared + k * j.shared_rows + row : j.own + (k - j.n_shared) * j.rows + r) * Hq + h; };
        float mx = -INFINITY, l = 0.f;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        for (int k0 = 0; k0 < n; k0 += 64) {
            const int cnt = min(64, n - k0);
            constexpr int AHEAD = 8;
            f32x4 o[AHEAD];
            const auto load = [&](int e0) {  // behind the last part: the last again, left out
#pragma unroll
                for (int e = 0; e < AHEAD; ++e) o[e] = *(const f32x4 *)(p.o + part(k0 + min((e0 + e) * sides + side, cnt - 1)) * D + d);
            };
            load(0);
            const float2 mine = lane < cnt ? p.ml[part(k0 + lane)] : make_float2(-INFINITY, 0.f);
            const float m_new = fmaxf(mx, wave_max(mine.x));
            const float f = mine.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mine.x - m_new), old = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx - m_new);
            l = l * old + wave_sum(f * mine.y);
            x *= old;
            mx = m_new;
            for (int e0 = 0; e0 * sides < cnt; e0 += AHEAD) {
                if (e0) load(e0);
#pragma unroll
                for (int e = 0; e < AHEAD; ++e) {
                    const int k = (e0 + e) * sides + side;
                    const float fk = __shfl(f, k & 63, 64);  // 0 behind the last
                    if (k < cnt) x += fk * o[e];
                }
            }
        }
        for (int q = lanes; q < 64; q <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], q, 64);
        const float inv = l > 0.f ? 1.f / l : 0.f;  // a NaN stays one: the sums of values are NaN then too
        x *= inv;
        if (side == 0 && (lane & (lanes - 1)) * 4 < D) {
            T *out = (T *)a.out + ((size_t)row * Hq + h) * D + d;
            if constexpr (sizeof(T) == 2) *(uint2 *)out = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
            else *(f32x4 *)out = x;
        }
    }
}

// Sizes that hold whatever the lengths are.  Items of a kv-head: a unit of n blocks and t tile groups has t * ceil(n / per) of them, and per is at least the sum of
// n * t over all units by `target`, or kMostBlocks.  Rows of a tile group: at most tiles * 16 / g and one more.
bool plan_for(const Dims &dm, int S, int G, int R, int max_blocks, PrefixPlan &p) {  // false: more than a launch counts
    const bool mfma = on_matrix_cores(dm);
    const int g = dm.Hq / dm.Hkv;
    p = PrefixPlan{};
    p.tiles = mfma ? kItemTiles : 1;
    p.step = mfma ? (dm.kv8 ? 2 * kStageGroups<true> : 2 * kStageGroups<false>) : std::max(1, 8 * 16 / dm.Bk);
    p.target = std::max(1, (mfma ? 512 : 1024) / dm.Hkv);
    const int64_t groups = 2 * (((int64_t)R * g + 15) / 16 / p.tiles + 1) + G + S;  // tile groups of all units, at most
    const int64_t items = std::max<int64_t>(p.target, groups * ((int64_t)max_blocks / kMostBlocks + 1)) + 2 * groups;
    if (items * dm.Hkv >= 1 << 24) return false;
    p.cap_items = (int)items;
    const int64_t most_parts = std::max<int64_t>(p.target, (int64_t)max_blocks / kMostBlocks + 1) + 2;
    p.cap_slots = std::min<int64_t>(2 * (int64_t)R * most_parts, (int64_t)p.cap_items * (p.tiles * 16 / g + 1));
    return p.cap_slots <= INT32_MAX;
}

}  // namespace

bool prefix_attn_fast(const Dims &dm) { return dm.Bk % 16 == 0 && dm.D % 16 == 0; }

static size_t place(const Dims &dm, int S, int G, PrefixPlan &p, char *ws) {
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        char *const r = ws + at;
        at += (bytes + 255) / 256 * 256;
        return r;
    };
    p.n_items = (int *)take(4);
    p.units = (PrefixUnit *)take((size_t)(G + S) * sizeof(PrefixUnit));
    p.seq_group = (int *)take((size_t)S * 4);
    p.items = (PrefixItem *)take((size_t)p.cap_items * sizeof(PrefixItem));
    p.join = (PrefixJoin *)take((size_t)S * sizeof(PrefixJoin));
    p.ml = (float2 *)take((size_t)p.cap_slots * dm.Hq * 8);
    p.o = (float *)take((size_t)p.cap_slots * dm.Hq * dm.D * 4);
    return at;
}

size_t prefix_attn_workspace(const Dims &dm, int S, int G, int R, int max_blocks) {
    if (!prefix_attn_fast(dm) || S == 0 || G == 0 || R == 0) return 256;
    PrefixPlan p;
    return plan_for(dm, S, G, R, max_blocks, p) ? place(dm, S, G, p, nullptr) + 256 : 0;
}

template <typename T, typename KT>
static hipError_t launch_f32(const Dims &dm, const PrefixAttnArgs &a, const PrefixPlan &p, hipStream_t st) {
    const dim3 grid((unsigned)p.cap_items * dm.Hkv);
    const float scale_log2 = kLog2e / sqrtf((float)dm.D) * (sizeof(KT) == 1 ? dm.k_scale : 1.f), v_scale = sizeof(KT) == 1 ? dm.v_scale : 1.f;
#define PREFIX_ATTN_F32(DT, EXACT) hipLaunchKernelGGL((k_prefix_attn_f32<T, KT, DT, EXACT>), grid, dim3(256), 0, st, a, p, dm.Hq, dm.Hkv, dm.D, dm.Bk, scale_log2, v_scale)
    if (dm.D == 64) PREFIX_ATTN_F32(4, true);
    else if (dm.D == 128) PREFIX_ATTN_F32(8, true);
    else if (dm.D < 128) PREFIX_ATTN_F32(8, false);
    else PREFIX_ATTN_F32(16, false);
#undef PREFIX_ATTN_F32
    return hipGetLastError();
}

hipError_t launch_prefix_attn(const Dims &dm, const PrefixAttnArgs &a, void *workspace, hipStream_t st) {
    PrefixPlan p;
    if (!plan_for(dm, a.S, a.G, a.R, a.max_blocks, p)) return hipErrorInvalidValue;  // its workspace has size 0, so no call gets here
    place(dm, a.S, a.G, p, (char *)workspace);
    const int g = dm.Hq / dm.Hkv, most = std::max(a.S, a.G);
    if (most <= 256) hipLaunchKernelGGL(k_prefix_plan_small<256>, dim3(1), dim3(256), 0, st, a, p, g, dm.Bk);
    else if (most <= 512) hipLaunchKernelGGL(k_prefix_plan_small<512>, dim3(1), dim3(512), 0, st, a, p, g, dm.Bk);
    else hipLaunchKernelGGL(k_prefix_plan, dim3(1), dim3(kPlanThreads), 0, st, a, p, g, dm.Bk);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (on_matrix_cores(dm)) {
        const dim3 grid((unsigned)p.cap_items * dm.Hkv);
        const float scale_log2 = kLog2e / sqrtf((float)kD) * (dm.kv8 ? dm.k_scale : 1.f);
        if (dm.kv8) hipLaunchKernelGGL(k_prefix_attn<true>, grid, dim3(256), 0, st, a, p, dm.Hq, dm.Hkv, scale_log2, dm.v_scale);
        else hipLaunchKernelGGL(k_prefix_attn<false>, grid, dim3(256), 0, st, a, p, dm.Hq, dm.Hkv, scale_log2, 1.f);
        e = hipGetLastError();
    } else {
        DISPATCH_TK(dm.bf16, dm.kv8, e = (launch_f32<T, KT>(dm, a, p, st)));
    }
    if (e != hipSuccess) return e;
    const int rows = std::min(64, std::max(1, 2 * ((a.R + a.S - 1) / a.S)));
    DISPATCH_T(dm.bf16, hipLaunchKernelGGL(k_prefix_join<T>, dim3(a.S, rows, (dm.Hq + 3) / 4), dim3(256), 0, st, a, p, dm.Hq, dm.D));
    return hipGetLastError();
}

}  // namespace icarus
