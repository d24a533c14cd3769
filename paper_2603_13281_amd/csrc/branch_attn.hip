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

namespace icarus {
namespace {

struct PrefixUnit { int row0, rows, seq, b0, nb, len, chunks, slot; };  // its rows; the sequence whose table has the blocks b0 .. b0 + nb - 1; positions end; parts and the first one's place
struct PrefixItem { int row0, rows, j0, seq, b0, nb, len, slot; };      // j0: the first of its queries among the unit's
struct PrefixJoin { int row0, rows, n_shared, shared, shared_rows, n_own, own, pad; };  // a sequence's rows; place of part k of row r: shared + k * shared_rows + r, then own + k * rows + r - row0
constexpr int kPlanThreads = 1024, kMostBlocks = 1024;                   // blocks of an item, at most
constexpr int kMostParts = (1 << 30) - 1;                                // where sums of items and parts stop: two of them fit an int, and no workspace holds so many
constexpr float kItemCost = 5.f, kAlone = 0.55f, kRounds = 0.6f;         // of the choice of an item's size: an item's cost beside its blocks, in blocks; a last round of at most one to a CU; weight of the rounds

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

// The rows of sequence u are among those of its group v.  They are not where row_start decreases: the group's parts have no places for them then.
__device__ __forceinline__ bool within(const PrefixUnit &u, const PrefixUnit &v) { return u.row0 >= v.row0 && u.row0 + u.rows <= v.row0 + v.rows; }

// For more than 512 sequences or groups.  Items have even shares, their sizes are not weighed as k_prefix_plan_small does: sequences of two rows and up to 500 tokens of their own behind one prefix of
// 8192, us of plan and items: 520 of them here 15 + 298, 500 there 14 + 307; eight groups behind 1024 to 8192 tokens, up to nine rows, 520 16 + 474, 496 13 + 423 for a seventh less of the products.
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
            if (u.len == 0) j.n_shared = j.n_own = 0;      // an empty sequence among others: the shared parts are not its own
            if (!within(u, v)) j.n_shared = 0;
        }
        p.join[s] = j;
    }
}

// The same for up to THREADS sequences and groups: one of each to a thread, everything in registers and LDS after one round of reads.  Bound by its chain: 8 sequences 5.9 us, 64 sequences of 8
// groups 8.3 us.
__device__ __forceinline__ int sat(int64_t v) { return (int)min(v, (int64_t)kMostParts); }
template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_prefix_plan_small(PrefixAttnArgs a, PrefixPlan p, int g, int Bk) {
    constexpr int WAVES = THREADS / 64;
    __shared__ int begin[THREADS], end[THREADS], least[THREADS], first[THREADS], live[THREADS], row_at[THREADS + 1], at_item[2 * THREADS], red[4][WAVES];
    __shared__ int64_t red_work[WAVES];
    __shared__ PrefixUnit units[2 * THREADS];
    __shared__ int size_of[2 * THREADS];  // blocks of an item of the unit
    __shared__ float4 red_size[WAVES][16];
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
    const int even = (int)min((total + p.target - 1) / p.target, (int64_t)kMostBlocks);
    int per = max((even + p.step - 1) / p.step, 1) * p.step;
    if (even > 2 * p.step && even < kMostBlocks) {
        // The largest size of an item.  Even shares would be `even` blocks, but a unit is cut into whole items, and a few more than run at once cost a round.  Of sixteen sizes the one is taken
        // whose sum is least, in blocks: all work over the workgroups that run at once, and kRounds times the rounds of the large items, a last round of at most one to a CU counting kAlone.  Over 16
        // sets of sequences (9 to 140 units, 600 to 25600 blocks) and eleven sizes each, called on one state after the other, this choice was 1.8 % behind the best one timed, 7.5 % at most; even shares 3.6 and 11 %.
        if (is_group) size_of[t] = u.nb, at_item[t] = tg_u;
        if (is_seq) size_of[a.G + t] = v.nb, at_item[a.G + t] = tg_v;
        __syncthreads();
        const int k = t & 15;
        const int most = min((int)ceilf(even * __builtin_amdgcn_exp2f(0.12f * (k - 6)) / p.step) * p.step, kMostBlocks);
        const float inv = __builtin_amdgcn_rcpf(most);
        float all_work = 0.f, large = 0.f, longest = 0.f;
        for (int i = t >> 4; i < a.G + a.S; i += THREADS / 16) {
            const float nb = size_of[i], tg = at_item[i];
            const float chunks = fmaxf(ceilf(nb * inv - 1e-4f), 1.f), size = nb * __builtin_amdgcn_rcpf(chunks), items = nb > 0.f ? tg * chunks : 0.f;
            all_work += items * (size + kItemCost);
            large += size > 0.3f * most ? items : 0.f;
            longest = fmaxf(longest, size);
        }
        const auto over = [&](auto op, float x) {  // the lanes of the same size
            x = op(x, __shfl_xor(x, 16, 64));
            return op(x, __shfl_xor(x, 32, 64));
        };
        const auto sum = [](float x, float y) { return x + y; };
        const auto max_of = [](float x, float y) { return fmaxf(x, y); };
        all_work = over(sum, all_work), large = over(sum, large), longest = over(max_of, longest);
        if (lane < 16) red_size[w][lane] = make_float4(all_work, large, longest, 0.f);
        __syncthreads();
        all_work = large = longest = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const float4 r = red_size[i][k];
            all_work += r.x, large += r.y, longest = fmaxf(longest, r.z);
        }
        const float rounds = large / p.target, full = floorf(rounds), rest = rounds - full;
        const float time = all_work / p.target + kRounds * (full + (rest <= 0.f ? 0.f : rest <= 0.5f ? kAlone : 1.f)) * (longest + kItemCost);
        float least = time;
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) least = fminf(least, __shfl_xor(least, o, 64));
        per = __shfl(most, __ffsll(__ballot(time == least)) - 1, 64);
    }
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
            if (lane >= o) x[k] = min(x[k] + y, kMostParts);
        }
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < 4; ++k) red[k][w] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        int before = 0, sum = 0;
        for (int i = 0; i < WAVES; ++i) {
            if (i < w) before = min(before + red[k][i], kMostParts);
            sum = min(sum + red[k][i], kMostParts);
        }
        x[k] = min(before + x[k], kMostParts);  // with this thread's own
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
            j = PrefixJoin{v.row0, v.rows, len && within(v, y) ? y.chunks : 0, y.slot - y.row0, y.rows, len ? v.chunks : 0, v.slot, 0};
        }
        p.join[t] = j;
    }
}

// 16-byte LDS-direct load: lane i copies 16 bytes from byte `at` (its own) behind g (the wave's) to LDS byte lds_base + 16 i (the wave's, passed in m0); the load counts in vmcnt until the
// data is in LDS.
__device__ __forceinline__ void to_lds16(const char *g, uint32_t at, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_base), "v"(at), "s"(g) : "memory");
}

// Sequence s with all of its blocks and rows as one item, for tables of at most kMostBlocks blocks; false: it is in no group, or has no rows.
__device__ __forceinline__ bool whole_sequence(const PrefixAttnArgs &a, int s, int Bk, PrefixItem &x) {
    x.row0 = min(max(a.row_start[s], 0), a.R);
    x.rows = min(max(a.row_start[s + 1], x.row0), a.R) - x.row0;
    x.seq = s;
    x.b0 = 0;
    x.len = (int)min((int64_t)max(a.kv_lens[s], 0), (int64_t)a.max_blocks * Bk);
    x.nb = x.len / Bk + (x.len % Bk != 0);
    x.slot = 0;
    return a.group_start[0] <= s && s < a.group_start[a.G] && x.rows > 0;
}

// ---- matrix cores: bf16 storage, head_dim 128, blocks of 16 -------------------------------------------------------------
// Products of 32 x 32 x 16 (operand layout of lane l, h = l / 32: A[row l % 32][k 8h .. 8h + 7], B[k 8h .. 8h + 7][col l % 32], C[row 8 (i / 4) + 4h + i % 4][col l % 32], i = 0 .. 15): beside one
// of them, 32 cycles, a SIMD issues six vector instructions, beside two of 16 x 16 x 32 four.  Scores are keys [token][channel] times queries [channel][query]; row r of a group of two blocks is
// token 8 (r / 4 % 2) + 4 (r / 8 % 2) + r % 4 of block r / 16, so that a lane's scores 8 s + e are tokens 8h + e of block s: at once the right operand of the values' product, whose
// left operand is a row piece of the transposed block.
//
// Keys and values go straight to LDS; two workgroups to a CU.  An item's queries are up to four tiles of 32, and a wave has one of them.
//   Three or four tiles: a group is a slot of a ring, requested some groups ahead by a quarter by each wave, and every wave multiplies every group.  While a group's weights are formed on the vector
//   units, the scores of the next one are multiplied.
//   One or two tiles, where each product is used less often than its operands are read from HBM: every wave (or two waves, one for each tile) takes groups of its own, into a part of LDS of its own,
//   without barriers -- a group's keys are in registers before its scores are formed, and their places are taken by the next group's at once --, and the states are put together at the end.
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
constexpr int kItemTiles = 8;  // of 16 queries
template <bool KV8> constexpr int kSlots = KV8 ? 8 : 4;
template <bool KV8> constexpr int kGroupBytes = KV8 ? 8192 : 16384;

struct PrefixState {
    f32x16 o[4];  // sums of values of four tiles of 32 channels
    float m, l;   // reference in log2 units, the same in both halves of the wave; sum of this half's weights
};

// A group in LDS.  Keys: rows of 8 chunks of 16 bytes (bf16: two such rows to a token, 4096 bytes apart), chunk c of row r in place c ^ (r / 2 % 8), so that lanes that read one chunk of
// 16 rows, 256 bytes in all, meet all banks.  Then values: of each block, bf16 [tile of 32 channels][lane] as the products take them, FP8 [channel][token].
struct PrefixPlaces { int key[4], value; };  // of this lane's chunks of keys 2 j + h; of its values
template <bool KV8>
__device__ __forceinline__ PrefixPlaces prefix_places(int lane) {
    const int r = lane & 31, h = lane >> 5;
    PrefixPlaces x;
#pragma unroll
    for (int j = 0; j < 4; ++j) x.key[j] = r * 128 + ((2 * j + h) ^ (r >> 1 & 7)) * 16;
    x.value = KV8 ? 4096 + r * 16 + 8 * h : 8192 + lane * 16;
    return x;
}

// The fragments are read well ahead of the products that take them: a wave issues in order, and one that waits for LDS at each product has nothing under way meanwhile.
template <bool KV8> struct PrefixKeys { uint4 f[KV8 ? 4 : 8]; };
template <bool KV8>
__device__ __forceinline__ void prefix_keys(PrefixKeys<KV8> &k, const char *__restrict__ src, const PrefixPlaces &at) {
#pragma unroll
    for (int j = 0; j < (KV8 ? 4 : 8); ++j) k.f[j] = *(const uint4 *)(src + at.key[j & 3] + (j >> 2) * 4096);
}
template <bool KV8> struct PrefixValues { typename std::conditional<KV8, uint2, uint4>::type f[4]; };  // of one block
template <bool KV8>
__device__ __forceinline__ void prefix_block(PrefixValues<KV8> &v, const char *__restrict__ src, const PrefixPlaces &at, int s) {
#pragma unroll
    for (int x = 0; x < 4; ++x) v.f[x] = *(const typename std::conditional<KV8, uint2, uint4>::type *)(src + at.value + s * (KV8 ? 2048 : 4096) + x * (KV8 ? 512 : 1024));
}
// Scores of a group, raw.
template <bool KV8>
__device__ __forceinline__ void prefix_scores(f32x16 &sc, const PrefixKeys<KV8> &k, const bf16x8 (&qr)[8]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
    for (int j = 0; j < (KV8 ? 4 : 8); ++j) {
        if constexpr (KV8) {
            sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cvt8(k.f[j].x, k.f[j].y), qr[2 * j], sc, 0, 0, 0);
            sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cvt8(k.f[j].z, k.f[j].w), qr[2 * j + 1], sc, 0, 0, 0);
        } else {
            sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k.f[j]), qr[j], sc, 0, 0, 0);
        }
    }
}

// By hand: for fmaxf the compiler first turns every score into itself, in case it were a signalling NaN.  Only for operands that no matrix instruction has just written: the compiler does
// not keep the distance that such a result needs before it is read in front of assembly (settled()).
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// Twenty wait states behind the products: any result may be read after fewer.
__device__ __forceinline__ void settled(f32x16 &s) { asm volatile("s_nop 15\n\ts_nop 3" : "+v"(s)); }

// One look whether the softmax reference has to move (rare: see compute_group).  there: tokens of the two blocks (masked only).
template <bool masked>
__device__ __forceinline__ void prefix_reference(PrefixState &st, f32x16 &sc, int there0, int there1, float scale_log2, int lane) {
    const int t0 = 8 * (lane >> 5);
    settled(sc);
    if (masked)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (t0 + i % 8 >= (i < 8 ? there0 : there1)) sc[i] = -INFINITY;
    const float a = max3(sc[0], sc[1], sc[2]), b = max3(sc[3], sc[4], sc[5]), c = max3(sc[6], sc[7], sc[8]), d = max3(sc[9], sc[10], sc[11]), e = max3(sc[12], sc[13], sc[14]);
    float mx = max3(max3(a, b, c), max3(d, e, sc[15]), sc[15]) * scale_log2;
    if (__builtin_expect(__any(mx > st.m + kSlack), 0)) {
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(st.m, mx), f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m - m_new);
        st.m = m_new;
        st.l *= f;
#pragma unroll
        for (int x = 0; x < 4; ++x) st.o[x] *= f;
    }
}

// Weights of a group and the values' product.
//
// A weight of one bfloat16 (half a step, 2^-8) would add as much error, squared, as the output's own rounding; the weight is cut to 8 bits and the rest goes through a second
// product (2^-15).  The rest is greater than 0 (by 2^-20 of the weight) wherever the weight is, so that an infinite value stays what it is.  FP8 values, whose codes are float16
// numbers too: weights in float16 (2^-11), kLift powers of two up, to at most 2^14, so that only weights below 2^-20 of the reference lose bits to float16's least exponent.
constexpr float kLift = 6.f;
struct PrefixWeights { uint4 hi, lo; };  // of one block's 8 tokens of this lane
template <bool KV8>
__device__ __forceinline__ PrefixWeights prefix_weights(PrefixState &st, const f32x16 &sc, int s, float scale_log2) {
    const float m_ref = (st.m == -INFINITY ? 0.f : st.m) - (KV8 ? kLift : 0.f);  // nothing yet: every weight 0
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[8 * s + i], scale_log2, -m_ref));
    st.l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));  // as they are
    PrefixWeights p;
    if constexpr (KV8) {
        p.hi = p.lo = make_uint4(pack_f16(e[0], e[1]), pack_f16(e[2], e[3]), pack_f16(e[4], e[5]), pack_f16(e[6], e[7]));
    } else {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = __float_as_uint(e[2 * i]) & 0xffff0000u, y = __float_as_uint(e[2 * i + 1]) & 0xffff0000u;
            hi[i] = __builtin_amdgcn_perm(__float_as_uint(e[2 * i + 1]), __float_as_uint(e[2 * i]), 0x07060302u);
            lo[i] = pack_bf16(__builtin_fmaf(e[2 * i], 1.f + 0x1p-20f, -__uint_as_float(x)), __builtin_fmaf(e[2 * i + 1], 1.f + 0x1p-20f, -__uint_as_float(y)));
        }
        p.hi = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        p.lo = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
    return p;
}
// there: tokens of the block (masked only: places behind the last one may hold anything).
template <bool KV8, bool masked>
__device__ __forceinline__ void prefix_product(PrefixState &st, const PrefixWeights &p, const PrefixValues<KV8> &vf, int there, int lane) {
    const int t0 = 8 * (lane >> 5);
    uint32_t keep[4];
    if (masked) {
#pragma unroll
        for (int i = 0; i < 4; ++i) keep[i] = (t0 + 2 * i < there ? 0xffffu : 0u) | (t0 + 2 * i + 1 < there ? 0xffff0000u : 0u);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        uint4 v;
        if constexpr (KV8) v = cvt8_f16(vf.f[x].x, vf.f[x].y);
        else v = vf.f[x];
        if (masked) v = make_uint4(v.x & keep[0], v.y & keep[1], v.z & keep[2], v.w & keep[3]);
        if constexpr (KV8) {
            st.o[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, p.hi), st.o[x], 0, 0, 0);
        } else {
            st.o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p.hi), st.o[x], 0, 0, 0);
            st.o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p.lo), st.o[x], 0, 0, 0);
        }
    }
}

// What bounds it (heads of 128, 8 kv-heads; share of the cycles in which the matrix pipe is busy).  32 queries of a kv-head over 32000 tokens: HBM and the latency of an item's first and last
// groups, 135 MB in 31 us, 4.4 TB/s (23 %).  8 groups with tails of up to 2000 tokens: both in turn, 451 MB and 29 GFLOP in 113 us, 4.0 TB/s (30 %).  1000 queries over 8192 tokens: 35 GFLOP, half
// as many again for the weights' second part, in 68 us (44 %).  1150 queries over two FP8 prefixes of 32768 tokens: 157 GFLOP in 184 us, 0.85 PFLOP/s (45 %), where a large product of bf16 in
// the library reaches 1.23; products alone between the barriers keep the pipe 72 to 80 % busy, the rest goes to the codes' conversion, to LDS and to the older of a CU's two workgroups, which is
// served first and leaves the younger one alone for the last third.  With bf16 values 38 registers spill (34 where DIRECT): none within the loops of whole groups, but the walk's end reads some back.
template <bool KV8, bool DIRECT>  // DIRECT: an item is a whole sequence, and the sums go to out
__global__ void __launch_bounds__(256, 2) k_prefix_attn(PrefixAttnArgs a, PrefixPlan p, int Hq, int Hkv, float scale_log2, float v_scale) {
    constexpr int SLOTS = kSlots<KV8>, BYTES = kGroupBytes<KV8>, ES = KV8 ? 1 : 2;
    __shared__ __attribute__((aligned(1024))) char ring[SLOTS * BYTES];
    static_assert(SLOTS * BYTES == 4 * 16384, "a state to a wave");
    __shared__ __attribute__((aligned(8))) int ids[kMostBlocks + 2];
    __shared__ int found[4], part_id;
    __shared__ float2 state_ml[4][64];
    const int i = blockIdx.x / Hkv, c = blockIdx.x % Hkv, g = Hq / Hkv;
    PrefixItem x;
    if constexpr (DIRECT) {
        if (!whole_sequence(a, i, kBk, x)) return;
        x.j0 = blockIdx.y * kItemTiles * 16;
        if (x.j0 >= x.rows * g) return;
    } else {
        const int n_items = *p.n_items;
        x = p.items[i];
        if (i >= n_items || x.nb <= 0) return;
    }
    const int lane = threadIdx.x & 63, h = lane >> 5, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = x.rows * g, tiles = min((G - x.j0 + 31) >> 5, kItemTiles / 2);
    const bool narrow = tiles <= 2;
    const int tile = narrow ? w & (tiles - 1) : w, j = x.j0 + 32 * tile + (lane & 31);
    bf16x8 qr[8];
    {
        const bf16_t *qp = (const bf16_t *)a.q + ((size_t)(x.row0 + j / g) * Hq + c * g + j % g) * kD;
#pragma unroll
        for (int k = 0; k < 8; ++k) qr[k] = tile < tiles && j < G ? *(const bf16x8 *)(qp + (KV8 ? 32 * (k >> 1) + 16 * h + 8 * (k & 1) : 16 * k + 8 * h)) : zero8();
    }
    // The blocks, without those outside the pool: full ones, then the one that ends early, if there is one (the last).  Their order does not matter to the sums.
    const int part_n = min(kBk, x.len - (x.b0 + x.nb - 1) * kBk);
    int n_full = 0;
    if (threadIdx.x == 0) part_id = -1;
    if (DIRECT && x.nb <= 0) __syncthreads();
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
    const int last = __builtin_amdgcn_readfirstlane(part_id), n_blk = n_full + (last >= 0), n_grp = (n_blk + 1) / 2;
    if (threadIdx.x < 2) ids[n_full + threadIdx.x] = threadIdx.x == 0 && last >= 0 ? last : 0;  // behind the last block: something to load
    PrefixState st;
    st.m = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int k = 0; k < 16; ++k) st.o[t][k] = 0.f;
    const PrefixPlaces at = prefix_places<KV8>(lane);
    // Where this lane's 16 bytes of a load stand in a block.  Keys: eight rows of 128 bytes to a load; the next eight rows are 4 tokens on.  Values: a KB to a load.
    const int r8 = lane >> 3, chunk = (lane & 7) ^ (r8 >> 1), token = 8 * (r8 >> 2) + (r8 & 3);
    const int key = token * kD * ES + chunk * 16, on = 4 * kD * ES + ((chunk ^ 4) - chunk) * 16;
    const int value = kBk * kD * ES + (KV8 ? 16 * lane : 32 * (lane & 31) + 16 * h);
    const char *const pool = (const char *)a.pool + (size_t)c * (2 * kBk * kD * ES);
    const size_t stride = (size_t)Hkv * 2 * kBk * kD * ES;
    const uint32_t ring0 = (uint32_t)(size_t)(__attribute__((address_space(3))) char *)ring;
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the queries are here, so the waits below count the requests alone
    __syncthreads();                     // ids
    const auto blocks_of_group = [&](int grp) {  // wave-uniform
        const int2 v = *(const int2 *)(ids + 2 * grp);
        return make_int2(__builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y));
    };
    const auto tokens_of = [&](int b) { return b < n_full ? kBk : b < n_blk ? part_n : 0; };
    const auto put = [&](const f32x16 &o, int t, float l) {  // sums of channel tile t; l: sum of the weights
        if constexpr (DIRECT) {
            const float inv = l > 0.f ? v_scale / l : 0.f;  // a NaN stays one: the sums of values are NaN then too
            bf16_t *const to = (bf16_t *)a.out + ((size_t)(x.row0 + j / g) * Hq + c * g + j % g) * kD + 32 * t + 4 * h;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                *(uint2 *)(to + 8 * k) = make_uint2(pack_bf16(o[4 * k] * inv, o[4 * k + 1] * inv), pack_bf16(o[4 * k + 2] * inv, o[4 * k + 3] * inv));
            return;
        }
        const size_t to = (size_t)(x.slot + j / g) * Hq + c * g + j % g;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            *(f32x4 *)(p.o + to * kD + 32 * t + 8 * k + 4 * h) = f32x4{o[4 * k] * v_scale, o[4 * k + 1] * v_scale, o[4 * k + 2] * v_scale, o[4 * k + 3] * v_scale};
    };
    const auto put_ml = [&](float m, float l) { if constexpr (!DIRECT) p.ml[(size_t)(x.slot + j / g) * Hq + c * g + j % g] = make_float2(m, l); };

    if (narrow) {
        constexpr int LOADS = KV8 ? 4 : 8;  // of a group's keys, and of its values
        const int step = 4 / tiles, first = w / tiles;  // one tile: groups w, w + 4, ..; two: w / 2, w / 2 + 2, ..
        const uint32_t to = ring0 + w * 16384;
        const char *const src = ring + w * 16384;
        const auto request_keys = [&](int2 b) {
            const char *const from0 = pool + b.x * stride, *const from1 = pool + b.y * stride;
#pragma unroll
            for (int k = 0; k < LOADS; ++k) to_lds16((k & 3) < 2 ? from0 : from1, key + (k & 1) * on + (k >> 2) * 128, to + k * 1024);
        };
        const auto request_values = [&](int2 b) {
            const char *const from0 = pool + b.x * stride, *const from1 = pool + b.y * stride;
#pragma unroll
            for (int k = 0; k < LOADS; ++k) to_lds16(k < LOADS / 2 ? from0 : from1, value + (k & (LOADS / 2 - 1)) * 1024, to + (LOADS + k) * 1024);
        };
        if (first < n_grp) {
            const int2 b = blocks_of_group(first);
            request_keys(b);
            request_values(b);
        }
#pragma nounroll
        for (int k = first; k < n_grp; k += step) {
            const bool more = k + step < n_grp;
            const int2 b = blocks_of_group(more ? k + step : k);
            const int there0 = tokens_of(2 * k), there1 = tokens_of(2 * k + 1);
            PrefixKeys<KV8> kf;
            PrefixValues<KV8> vf[2];
            f32x16 sc;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");  // the keys have landed, the values may be under way
            prefix_keys<KV8>(kf, src, at);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // and are in registers
            if (more) request_keys(b);
            prefix_scores<KV8>(sc, kf, qr);
            prefix_reference<true>(st, sc, there0, there1, scale_log2, lane);
            if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            prefix_block<KV8>(vf[0], src, at, 0);
            prefix_block<KV8>(vf[1], src, at, 1);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) request_values(b);
            prefix_product<KV8, true>(st, prefix_weights<KV8>(st, sc, 0, scale_log2), vf[0], there0, lane);
            prefix_product<KV8, true>(st, prefix_weights<KV8>(st, sc, 1, scale_log2), vf[1], there1, lane);
        }
        // The states of the waves that have the same tile: each leaves its own in LDS, in its own part, and takes 4 / step of the channels.
        f32x4 *const mine = (f32x4 *)(ring + w * 16384);
        state_ml[w][lane] = make_float2(st.m, st.l);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int k = 0; k < 4; ++k) mine[(4 * t + k) * 64 + lane] = f32x4{st.o[t][4 * k], st.o[t][4 * k + 1], st.o[t][4 * k + 2], st.o[t][4 * k + 3]};
        __syncthreads();
        float m = -INFINITY, l = 0.f, f[4];
        for (int k = 0; k < step; ++k) m = fmaxf(m, state_ml[tile + k * tiles][lane].x);
        for (int k = 0; k < step; ++k) {
            const float2 v = state_ml[tile + k * tiles][lane];
            f[k] = v.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(v.x - m);
            l += f[k] * v.y;
        }
        l += __shfl_xor(l, 32, 64);
        if (j >= G) return;
        for (int t = first; t < 4; t += step) {
            f32x16 o;
#pragma unroll
            for (int k = 0; k < 16; ++k) o[k] = 0.f;
            for (int y = 0; y < step; ++y)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const f32x4 v = ((const f32x4 *)(ring + (tile + y * tiles) * 16384))[(4 * t + k) * 64 + lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[4 * k + e] += f[y] * v[e];
                }
            put(o, t, l);
        }
        if (first == 0 && h == 0) put_ml(m, l);
        return;
    }

    constexpr int LOADS = KV8 ? 2 : 4;
    int2 pair = make_int2(0, 0);  // the blocks of the group that is requested next, read ahead: what an address waits for, every product behind it waits for
    // This wave's quarter of a group.  w = 0, 1: keys, bf16 half w of all 32 rows, FP8 the rows of block w; w = 2, 3: the values of block w - 2.
    const auto request = [&](int grp) {
        const uint32_t to = ring0 + (grp & (SLOTS - 1)) * BYTES + LOADS * 1024 * w;
        const char *const from0 = pool + pair.x * stride, *const from1 = pool + pair.y * stride;
        if (w < 2 && !KV8) {  // rows 0 .. 15 are the first block's
            to_lds16(from0, key + 128 * w, to);
            to_lds16(from0, key + 128 * w + on, to + 1024);
            to_lds16(from1, key + 128 * w, to + 2048);
            to_lds16(from1, key + 128 * w + on, to + 3 * 1024);
        } else {
            const char *const from = w & 1 ? from1 : from0;
#pragma unroll
            for (int k = 0; k < LOADS; ++k) to_lds16(from, w < 2 ? key + k * on : value + k * 1024, to + k * 1024);
        }
    };
    // All that this wave requested of group k has landed (of `ahead` younger groups it may be under way), and behind the barrier what the other waves requested too.
    const auto landed = [&](int k, auto younger) {
        constexpr int ahead = decltype(younger)::value;
        static_assert(ahead * LOADS < 16, "one field of the wait's count");
        if (k + ahead < n_grp) __builtin_amdgcn_s_waitcnt(0x0f70 | ahead * LOADS);
        else __builtin_amdgcn_s_waitcnt(0x0f70);
        __syncthreads();
    };
    const auto slot = [&](int k) { return ring + (k & (SLOTS - 1)) * BYTES; };
    const auto next_slot = [&](int k, auto all) {  // group k - SLOTS is in every wave's registers; all: k < n_grp
        if constexpr (decltype(all)::value) {
            __builtin_amdgcn_s_waitcnt(0x0f70 | (SLOTS - 3) * LOADS);
            __syncthreads();
            request(k);
        } else {
            landed(k - SLOTS + 2, std::integral_constant<int, SLOTS - 3>());
            if (k < n_grp) request(k);
        }
    };
    if (n_grp > 0) {
        for (int k = 0; k < min(SLOTS, n_grp); ++k) {
            pair = blocks_of_group(k);
            request(k);
        }
        pair = blocks_of_group(min(SLOTS, n_grp - 1));
        landed(1, std::integral_constant<int, SLOTS - 2>());
    }
    if (tile >= tiles) {
        for (int k = 0; k + 1 < n_grp; ++k) {
            next_slot(k + SLOTS, std::false_type());
            pair = blocks_of_group(min(k + SLOTS + 1, n_grp - 1));
        }
        return;
    }
    if (n_grp > 0) {
        f32x16 now, next;
        PrefixKeys<KV8> kf;
        PrefixValues<KV8> v0, v1;
        prefix_keys<KV8>(kf, slot(0), at);
        prefix_scores<KV8>(now, kf, qr);
        prefix_keys<KV8>(kf, slot(1), at);  // of no use where there is one group
        prefix_block<KV8>(v0, slot(0), at, 0);
        // A group's weights are formed beside products that do not wait for them: those of its first block beside the next group's scores, those of the second beside the first one's values.
        // Fragments are read a part ahead, and the barrier stands where the last of a group have been.
        const auto step = [&](int k, f32x16 &x0, f32x16 &x1, auto all) {
            prefix_block<KV8>(v1, slot(k), at, 1);
            const int2 ahead = *(const int2 *)(ids + 2 * min(k + SLOTS + 1, n_grp - 1));
            __builtin_amdgcn_sched_barrier(0);
            prefix_reference<false>(st, x0, kBk, kBk, scale_log2, lane);
            prefix_scores<KV8>(x1, kf, qr);
            const PrefixWeights p0 = prefix_weights<KV8>(st, x0, 0, scale_log2);
            prefix_product<KV8, false>(st, p0, v0, kBk, lane);
            PrefixWeights p1 = prefix_weights<KV8>(st, x0, 1, scale_log2);
            asm volatile("" : "+v"(p1.hi.x), "+v"(p1.hi.y), "+v"(p1.hi.z), "+v"(p1.hi.w), "+v"(p1.lo.x), "+v"(p1.lo.y), "+v"(p1.lo.z), "+v"(p1.lo.w));  // here, not where they are needed
            __builtin_amdgcn_sched_barrier(0);
            next_slot(k + SLOTS, all);
            prefix_keys<KV8>(kf, slot(k + 2), at);
            prefix_block<KV8>(v0, slot(k + 1), at, 0);
            pair = make_int2(__builtin_amdgcn_readfirstlane(ahead.x), __builtin_amdgcn_readfirstlane(ahead.y));
            __builtin_amdgcn_sched_barrier(0);
            prefix_product<KV8, false>(st, p1, v1, kBk, lane);
        };
        int k = 0;
#pragma nounroll
        for (; k + 1 + SLOTS < n_grp; k += 2) {
            step(k, now, next, std::true_type());
            step(k + 1, next, now, std::true_type());
        }
#pragma nounroll
        for (; k + 2 < n_grp; k += 2) {
            step(k, now, next, std::false_type());
            step(k + 1, next, now, std::false_type());
        }
        const auto end = [&](f32x16 &y) {  // the last group, of which a block may end early or be missing
            const int there0 = tokens_of(2 * (n_grp - 1)), there1 = tokens_of(2 * n_grp - 1);
            prefix_block<KV8>(v1, slot(n_grp - 1), at, 1);
            prefix_reference<true>(st, y, there0, there1, scale_log2, lane);
            prefix_product<KV8, true>(st, prefix_weights<KV8>(st, y, 0, scale_log2), v0, there0, lane);
            prefix_product<KV8, true>(st, prefix_weights<KV8>(st, y, 1, scale_log2), v1, there1, lane);
        };
        if (k + 1 < n_grp) {
            step(k, now, next, std::false_type());
            end(next);
        } else {
            end(now);
        }
    }
    const float l = st.l + __shfl_xor(st.l, 32, 64);
    if (j >= G) return;
#pragma unroll
    for (int t = 0; t < 4; ++t) put(st.o[t], t, l);
    if (h == 0) put_ml(st.m, l);
}

bool on_matrix_cores(const Dims &dm) { return dm.bf16 && dm.D == kD && dm.Bk == kBk; }

// ---- block and head sizes that are multiples of 16: matrix cores in float32 ------------------------------------------------------
// For float32, head sizes other than 128 and blocks of more than 16 tokens.  An item has a tile of 16 queries; a wave takes sixteen tokens of a block in turn.  Products of 16 x 16 x 4 with the
// transposed operands, see k_block_attn_f32: scores of keys [token][channel] times queries [channel][query] leave lane t + 16 p query t's scores of tokens 4 p .. 4 p + 3, which are
// at once the right operand of the values' product, so nothing passes through LDS until the waves join.  Bound by the float32 products, a sixteenth of the 16-bit rate, where there are many
// queries; in a short call by its chain (3 sequences of up to 130 tokens, 4 heads of 64: 6 us).  32 query and 8 kv-heads, 128 sequences over 8192 tokens, 256 rows: float32 heads of 128, 35 GFLOP, 463 us;
// bf16 heads of 64 230 us, of 256 1606, blocks of 32 tokens 420, where the 16-bit products take 68 for blocks of 16.
template <typename T, typename KT, int DT, bool EXACT, bool DIRECT>  // tiles of 16 channels: at most DT, or DT exactly
__global__ void __launch_bounds__(256) k_prefix_attn_f32(PrefixAttnArgs a, PrefixPlan p, int Hq, int Hkv, int D_, int Bk, float scale_log2, float v_scale) {
    typedef typename Quad<KT>::raw Raw;
    __shared__ f32x4 image[2][DT][64];
    __shared__ int2 ids[kMostBlocks];  // block of the pool, and its tokens
    __shared__ float image_m[4][16], image_l[4][16];
    const int item = blockIdx.x / Hkv, c = blockIdx.x % Hkv, g = Hq / Hkv;
    PrefixItem x;
    if constexpr (DIRECT) {
        if (!whole_sequence(a, item, Bk, x)) return;
        x.j0 = blockIdx.y * 16;
        if (x.j0 >= x.rows * g) return;
    } else {
        const int n_items = *p.n_items;
        x = p.items[item];
        if (item >= n_items || x.nb <= 0) return;
    }
    const int D = EXACT ? 16 * DT : D_, d16 = D / 16;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, p4 = 4 * (lane >> 4);
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
    if constexpr (DIRECT) {
        const float inv = sum > 0.f ? v_scale / sum : 0.f;  // a NaN stays one: the sums of values are NaN then too
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            if (!EXACT && d >= d16) continue;
            T *out = (T *)a.out + row * D + 16 * d + p4;
            if constexpr (sizeof(T) == 2) *(uint2 *)out = make_uint2(pack_bf16(o[d][0] * inv, o[d][1] * inv), pack_bf16(o[d][2] * inv, o[d][3] * inv));
            else *(f32x4 *)out = o[d] * inv;
        }
        return;
    }
    const size_t at = (size_t)(x.slot + j / g) * Hq + c * g + j % g;
#pragma unroll
    for (int d = 0; d < DT; ++d)
        if (EXACT || d < d16) *(f32x4 *)(p.o + at * D + 16 * d + p4) = o[d] * v_scale;
    if (p4 == 0) p.ml[at] = make_float2(mx, sum);
}

// A row's parts put together, first the parts of the group's shared blocks, then those of its own: a wave to a head, four channels to a lane, so that D / 4 lanes take a part and the wave
// 256 / D of them at once (up to 256 channels).  Bound by its chain of two reads, so the first values are on their way before the maxima are known
// (16 rows 4.7 us, 300 rows with up to 12 parts 13 us).
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

// Sizes that hold whatever the lengths are.  Items of a kv-head: a unit of n blocks and t tile groups has t * ceil(n / per) of them, and per is at least half the sum of
// n * t over all units by `target`, or kMostBlocks.  Rows of a tile group: at most tiles * 16 / g and one more.
bool plan_for(const Dims &dm, int S, int G, int R, int max_blocks, PrefixPlan &p) {  // false: more than a launch counts
    const bool mfma = on_matrix_cores(dm);
    const int g = dm.Hq / dm.Hkv;
    p = PrefixPlan{};
    p.tiles = mfma ? kItemTiles : 1;
    p.step = mfma ? 4 : std::max(1, 8 * 16 / dm.Bk);
    p.target = std::max(1, (mfma ? 512 : 1024) / dm.Hkv);
    const int64_t groups = 2 * (((int64_t)R * g + 15) / 16 / p.tiles + 1) + G + S;  // tile groups of all units, at most
    const int64_t items = std::max<int64_t>(p.target * 5 / 3, groups * ((int64_t)max_blocks / kMostBlocks + 1)) + 2 * groups;
    if (items * dm.Hkv >= 1 << 24) return false;
    p.cap_items = (int)items;
    const int64_t most_parts = std::max<int64_t>(p.target * 5 / 3, (int64_t)max_blocks / kMostBlocks + 1) + 2;
    p.cap_slots = std::min<int64_t>(2 * (int64_t)R * most_parts, (int64_t)p.cap_items * (p.tiles * 16 / g + 1));
    return p.cap_slots < kMostParts;  // heads of 128 alone come near it: 500 GB
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

// Tables so short that one launch in which every sequence reads all of its own costs less than three that read the shared blocks once.  1 to 128 sequences that share all but 30 tokens, 8 kv-heads,
// us for three and for one launch, one sequence and 128 of them: 512 tokens 19 and 37 to 12 and 26, 1024 tokens 19 and 39 to 14 and 37, 2048 tokens 18 and 42 to 22 and 61 (FP8 cache the same way).
// Without matrix cores: 256 tokens 16 and 17 to 12 and 12, 512 tokens 16 and 17 to 12 and 18, 1024 tokens 16 and 20 to 20 and 30.  Not timed beyond 1024 sequences x kv-heads.
static int direct_tiles(const Dims &dm, const PrefixAttnArgs &a) {  // tile groups of the launch, 0: not this way
    const int64_t tiles = ((int64_t)a.R * (dm.Hq / dm.Hkv) + 15) / 16, groups = on_matrix_cores(dm) ? (tiles + kItemTiles - 1) / kItemTiles : tiles;
    const int64_t tokens = (int64_t)a.max_blocks * dm.Bk, items = (int64_t)a.S * dm.Hkv;
    return tokens <= (on_matrix_cores(dm) ? 1024 : 512) && items <= 1024 && items * groups <= 8192 ? (int)groups : 0;
}

template <typename T, typename KT>
static hipError_t launch_f32(const Dims &dm, const PrefixAttnArgs &a, const PrefixPlan &p, int direct, hipStream_t st) {
    const dim3 grid(direct ? (unsigned)a.S * dm.Hkv : (unsigned)p.cap_items * dm.Hkv, direct ? direct : 1);
    const float scale_log2 = kLog2e / sqrtf((float)dm.D) * (sizeof(KT) == 1 ? dm.k_scale : 1.f), v_scale = sizeof(KT) == 1 ? dm.v_scale : 1.f;
#define PREFIX_ATTN_F32(DT, EXACT)                                                                                                                                                    \
    do {                                                                                                                                                                               \
        if (direct) hipLaunchKernelGGL((k_prefix_attn_f32<T, KT, DT, EXACT, true>), grid, dim3(256), 0, st, a, p, dm.Hq, dm.Hkv, dm.D, dm.Bk, scale_log2, v_scale);                    \
        else hipLaunchKernelGGL((k_prefix_attn_f32<T, KT, DT, EXACT, false>), grid, dim3(256), 0, st, a, p, dm.Hq, dm.Hkv, dm.D, dm.Bk, scale_log2, v_scale);                          \
    } while (0)
    if (dm.D == 64) PREFIX_ATTN_F32(4, true);
    else if (dm.D == 128) PREFIX_ATTN_F32(8, true);
    else if (dm.D < 128) PREFIX_ATTN_F32(8, false);
    else PREFIX_ATTN_F32(16, false);
#undef PREFIX_ATTN_F32
    return hipGetLastError();
}

template <bool DIRECT>
static hipError_t launch_mfma(const Dims &dm, const PrefixAttnArgs &a, const PrefixPlan &p, dim3 grid, hipStream_t st) {
    const float scale_log2 = kLog2e / sqrtf((float)kD) * (dm.kv8 ? dm.k_scale : 1.f);
    if (dm.kv8) hipLaunchKernelGGL((k_prefix_attn<true, DIRECT>), grid, dim3(256), 0, st, a, p, dm.Hq, dm.Hkv, scale_log2, dm.v_scale);
    else hipLaunchKernelGGL((k_prefix_attn<false, DIRECT>), grid, dim3(256), 0, st, a, p, dm.Hq, dm.Hkv, scale_log2, 1.f);
    return hipGetLastError();
}

hipError_t launch_prefix_attn(const Dims &dm, const PrefixAttnArgs &a, void *workspace, hipStream_t st) {
    PrefixPlan p;
    hipError_t e = hipSuccess;
    if (const int direct = direct_tiles(dm, a)) {
        p = PrefixPlan{};
        if (on_matrix_cores(dm)) return launch_mfma<true>(dm, a, p, dim3((unsigned)a.S * dm.Hkv, direct), st);
        DISPATCH_TK(dm.bf16, dm.kv8, e = (launch_f32<T, KT>(dm, a, p, direct, st)));
        return e;
    }
    if (!plan_for(dm, a.S, a.G, a.R, a.max_blocks, p)) return hipErrorInvalidValue;  // its workspace has size 0, so no call gets here
    place(dm, a.S, a.G, p, (char *)workspace);
    const int g = dm.Hq / dm.Hkv, most = std::max(a.S, a.G);
    if (most <= 256) hipLaunchKernelGGL(k_prefix_plan_small<256>, dim3(1), dim3(256), 0, st, a, p, g, dm.Bk);
    else if (most <= 512) hipLaunchKernelGGL(k_prefix_plan_small<512>, dim3(1), dim3(512), 0, st, a, p, g, dm.Bk);
    else hipLaunchKernelGGL(k_prefix_plan, dim3(1), dim3(kPlanThreads), 0, st, a, p, g, dm.Bk);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (on_matrix_cores(dm)) e = launch_mfma<false>(dm, a, p, dim3((unsigned)p.cap_items * dm.Hkv), st);
    else DISPATCH_TK(dm.bf16, dm.kv8, e = (launch_f32<T, KT>(dm, a, p, 0, st)));
    if (e != hipSuccess) return e;
    const int rows = std::min(64, std::max(1, 2 * ((a.R + a.S - 1) / a.S)));
    DISPATCH_T(dm.bf16, hipLaunchKernelGGL(k_prefix_join<T>, dim3(a.S, rows, (dm.Hq + 3) / 4), dim3(256), 0, st, a, p, dm.Hq, dm.D));
    return hipGetLastError();
}

}  // namespace icarus
