// Operators with lengths on the device: growth of the sequences, rotation and append, bounds of the keys, choice of the
// blocks.  Everything a kernel indexes with -- lengths, slots, block ids -- comes from device memory and is checked
// where it is used.
#include "block_ops.h"
#include "device_util.h"

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

// ---- growth of the sequences ------------------------------------------------------------------------------------------
// Two sums over the sequences decide everything: rows before a sequence, and blocks taken before it.  Every workgroup
// forms both over all sequences (8-12 bytes each, from L2) and writes its own range of rows, so that one launch does and no
// workgroup waits for another.  Sums saturate just past the largest value that is told apart (max_rows, n_free), so that no length overflows them.
constexpr int kExtThreads = 256, kExtPer = 4, kExtSeg = kExtThreads * kExtPer;  // sequences of a round

__host__ __device__ __forceinline__ int blocks_of(int tokens, int Bk) { return tokens / Bk + (tokens % Bk != 0); }

// Exclusive saturating prefix sum of one value per thread; *total: of all.
__device__ __forceinline__ int scan_sat(int v, int cap, int *red, int *total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x = min(x + y, cap);
    }
    __syncthreads();
    if (lane == 63) red[w] = x;
    __syncthreads();
    int before = 0, sum = 0;
    for (int i = 0; i < kExtThreads / 64; ++i) {
        if (i < w) before = min(before + red[i], cap);
        sum = min(sum + red[i], cap);
    }
    *total = sum;
    const int up = __shfl_up(x, 1, 64);
    return min(before + (lane ? up : 0), cap);
}

__global__ void __launch_bounds__(kExtThreads) k_extend(ExtendArgs a, int rows_per_wg) {
    __shared__ int row_begin[kExtSeg], row_end[kExtSeg], first_id[kExtSeg], ctx[kExtSeg], fresh[kExtSeg], red[kExtThreads / 64];
    const int row_cap = a.max_rows + 1, id_cap = a.n_free + 1;
    const int r0 = blockIdx.x * rows_per_wg, r1 = min(a.max_rows, r0 + rows_per_wg);
    const bool lead = blockIdx.x == 0;
    const int head = min(max(*a.free_used, 0), a.n_free);
    int rows_before = 0, ids_before = head, used = head, refused = 0;
    for (int s0 = 0; s0 < a.S; s0 += kExtSeg) {
        int n[kExtPer], c[kExtPer], nw[kExtPer], need[kExtPer], sum = 0, total;
        bool ok[kExtPer];
#pragma unroll
        for (int j = 0; j < kExtPer; ++j) {
            const int s = s0 + threadIdx.x * kExtPer + j;
            const bool in = s < a.S;
            c[j] = in ? a.ctx_lens[s] : 0;
            nw[j] = in ? a.new_lens[s] : 0;
            const int m = in && a.streams ? a.streams[s] : 0;
            const int64_t end = (int64_t)c[j] + nw[j];
            ok[j] = c[j] >= 0 && nw[j] >= 0 && m >= 0 && end <= a.max_position && end <= (int64_t)a.max_blocks * a.Bk;
            n[j] = nw[j] > 0 ? (int)min((int64_t)nw[j] + max(m, 0), (int64_t)row_cap) : 0;
            sum = min(sum + n[j], row_cap);
        }
        const int round0 = rows_before;
        int at = min(rows_before + scan_sat(sum, row_cap, red, &total), row_cap);
        rows_before = min(rows_before + total, row_cap);
        sum = 0;
#pragma unroll
        for (int j = 0; j < kExtPer; ++j) {
            const int i = threadIdx.x * kExtPer + j;
            if (lead && s0 + i < a.S) a.row_start[s0 + i] = min(at, a.max_rows);
            row_begin[i] = at;
            at = min(at + n[j], row_cap);
            row_end[i] = at;
            ok[j] = ok[j] && (n[j] == 0 || at <= a.max_rows);
            need[j] = ok[j] ? blocks_of(c[j] + nw[j], a.Bk) - blocks_of(c[j], a.Bk) : 0;
            sum = min(sum + need[j], id_cap);
        }
        int id = min(ids_before + scan_sat(sum, id_cap, red, &total), id_cap);
        ids_before = min(ids_before + total, id_cap);
#pragma unroll
        for (int j = 0; j < kExtPer; ++j) {
            const int i = threadIdx.x * kExtPer + j;
            first_id[i] = id;
            id = min(id + need[j], id_cap);
            ok[j] = ok[j] && (need[j] == 0 || id <= a.n_free);
            ctx[i] = c[j];
            fresh[i] = ok[j] ? nw[j] : -1;
            if (s0 + i < a.S) {
                if (ok[j] && need[j]) used = id;  // of the last sequence that takes blocks: ids grow from one to the next
                refused += !ok[j];
                if (lead) a.kv_lens[s0 + i] = ok[j] ? c[j] + nw[j] : c[j];
            }
        }
        __syncthreads();
        // this workgroup's rows among the round's
        const int last = min(kExtSeg, a.S - s0) - 1, stop = min(r1, row_end[last]);
        for (int r = max(r0, round0) + threadIdx.x; r < stop; r += kExtThreads) {
            int lo = 0, hi = last;  // the first sequence that ends behind row r holds it
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (row_end[mid] > r) hi = mid;
                else lo = mid + 1;
            }
            const int i = r - row_begin[lo], news = fresh[lo];
            int pos = -1;
            int64_t slot = -1;
            if (news >= 0) {
                pos = ctx[lo] + min(i, news - 1);
                if (i < news) {
                    const int column = pos / a.Bk, off = pos - column * a.Bk, old = blocks_of(ctx[lo], a.Bk);
                    int32_t *entry = a.bt + (size_t)(s0 + lo) * a.max_blocks + column;
                    int b = column < old ? *entry : a.free_ids[first_id[lo] + column - old];
                    if (b < 0 || b >= a.num_blocks) b = -1;
                    if (off == 0) *entry = b;  // a block's first token brings it in
                    if (b >= 0) slot = (int64_t)b * a.Bk + off;
                }
            }
            a.row_seq[r] = news >= 0 ? s0 + lo : -1;
            a.row_pos[r] = pos;
            a.row_slot[r] = slot;
        }
        __syncthreads();
    }
    for (int r = max(r0, rows_before) + threadIdx.x; r < r1; r += kExtThreads) {
        a.row_seq[r] = -1;
        a.row_pos[r] = -1;
        a.row_slot[r] = -1;
    }
    if (!lead) return;
    __shared__ int most[kExtThreads / 64];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        used = max(used, __shfl_xor(used, o, 64));
        refused += __shfl_xor(refused, o, 64);
    }
    if ((threadIdx.x & 63) == 0) {
        most[threadIdx.x >> 6] = used;
        red[threadIdx.x >> 6] = refused;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kExtThreads / 64; ++i) {
            used = max(used, most[i]);
            refused += red[i];
        }
        a.counts[0] = used;
        a.counts[1] = refused;
        a.row_start[a.S] = min(rows_before, a.max_rows);
    }
}

// ---- rotation and append ------------------------------------------------------------------------------------------------
// Turns of pair i at a position, pos * theta^(-2i/D) / 2 pi, in float64: a far position keeps the fraction of its last turn.
__device__ __forceinline__ void turn_of(int pos, double turns_per_pos, float *cs, float *sn) {
    const double t = (double)pos * turns_per_pos;
    const float half_turns = (float)(2.0 * (t - rint(t)));  // -1 .. 1, rounded last
    *cs = cospif(half_turns);
    *sn = sinpif(half_turns);
}
__device__ __forceinline__ double turns_per_position(int i, int D, double log2_theta) {
    return exp2(-(2.0 * (double)i / (double)D) * log2_theta) * 0.15915494309189533577;
}

// Any head size: a wave to a head of a row, a pair to a lane.
template <typename T, typename KT>
__global__ void __launch_bounds__(256) k_append(AppendArgs a, int Hq, int Hkv, int D, int Bk, double log2_theta, float eps, int qk_norm,
                                                float k_scale, float v_scale) {
    const int row = blockIdx.x, h = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, half = D >> 1;
    if (h >= Hq + 2 * Hkv) return;
    const int pos = a.row_pos[row];
    if (pos < 0) return;
    const int64_t slot = a.row_slot[row];
    const bool write = slot >= 0 && slot < a.n_slots;
    if (h >= Hq && !write) return;
    const T *src = (const T *)a.qkv + (size_t)row * a.ld + (size_t)h * D;
    const size_t blk = write ? (size_t)slot / Bk : 0, off = write ? (size_t)slot % Bk : 0;
    KT *pool = (KT *)a.pool;
    if (h >= Hq + Hkv) {
        KT *dst = pool + ((blk * Hkv + (h - Hq - Hkv)) * 2 + 1) * Bk * D + off;  // V plane [D][Bk]
        for (int i = lane; i < D; i += 64) KVElem<KT>::st(dst + (size_t)i * Bk, Elem<T>::ld(src + i), v_scale);
        return;
    }
    float inv = 1.f;
    if (qk_norm) {
        float ss = 0.f;
        for (int i = lane; i < D; i += 64) { const float v = Elem<T>::ld(src + i); ss += v * v; }
        inv = rsqrtf(wave_sum(ss) / (float)D + eps);
    }
    for (int i = lane; i < half; i += 64) {
        float x = Elem<T>::ld(src + i), y = Elem<T>::ld(src + i + half), cs, sn, rx, ry;
        if (qk_norm) {
            const T *w = (const T *)(h < Hq ? a.q_norm : a.k_norm);
            x = x * inv * Elem<T>::ld(w + i);
            y = y * inv * Elem<T>::ld(w + i + half);
        }
        turn_of(pos, turns_per_position(i, D, log2_theta), &cs, &sn);
        rotate_pair(x, y, cs, sn, &rx, &ry);
        if (h < Hq) {
            T *dst = (T *)a.q_out + ((size_t)row * Hq + h) * D;
            Elem<T>::st(dst + i, rx);
            Elem<T>::st(dst + i + half, ry);
        } else {
            KT *dst = pool + ((blk * Hkv + (h - Hq)) * 2) * Bk * D + off * D;  // K plane [Bk][D]
            KVElem<KT>::st(dst + i, rx, k_scale);
            KVElem<KT>::st(dst + i + half, ry, k_scale);
        }
    }
}

// ---- bounds of the keys ---------------------------------------------------------------------------------------------------
// Exponent e of the smallest 2^e, -40 <= e <= 40, with 127 * 2^e >= x (x >= 0 and finite).  With both exponents of a score in this range
// its value, a whole number below 2^23 times 2^(-80 .. 80), is an exact float.
__device__ __forceinline__ int step_exponent(float x) {
    const int e = __builtin_amdgcn_frexp_expf(x) - (__builtin_amdgcn_frexp_mantf(x) > 127.f / 128.f ? 6 : 7);
    return x > 0.f ? min(max(e, -40), 40) : -40;
}
__device__ __forceinline__ float finite_or_edge(float x) {
    if (!(x == x)) return 0.f;
    return fminf(fmaxf(x, -3.402823466e38f), 3.402823466e38f);
}
__device__ __forceinline__ int8_t code_of(float rounded) { return (int8_t)(int)fminf(fmaxf(rounded, -127.f), 127.f); }
template <typename KT> __device__ __forceinline__ float key_value(const KT *p) { return finite_or_edge(KVElem<KT>::ld(p, 1.f)); }

// Any shape: a wave to a block and kv-head, a channel to a lane.
template <typename KT>
__global__ void __launch_bounds__(256) k_bounds(BoundsArgs a, int Hkv, int D, int Bk) {
    const int s = blockIdx.x, c = blockIdx.z * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (c >= Hkv) return;
    const int from = max(a.from_lens[s], 0), to = (int)min((int64_t)max(a.to_lens[s], 0), (int64_t)a.max_blocks * Bk);
    if (from >= to) return;
    for (int b = from / Bk + blockIdx.y; b * (int64_t)Bk < to; b += gridDim.y) {
        const int id = a.bt[(size_t)s * a.max_blocks + b];
        if (id < 0 || id >= a.num_blocks) continue;
        const int n = min(Bk, to - b * Bk);
        const KT *k = (const KT *)a.pool + ((size_t)id * Hkv + c) * 2 * Bk * D;
        float hi[4], lo[4], most = 0.f;  // head sizes up to 256
        for (int j = 0; j * 64 + lane < D; ++j) {
            hi[j] = -INFINITY;
            lo[j] = INFINITY;
            for (int t = 0; t < n; ++t) {
                const float v = key_value(k + (size_t)t * D + j * 64 + lane);
                hi[j] = fmaxf(hi[j], v);
                lo[j] = fminf(lo[j], v);
            }
            most = fmaxf(most, fmaxf(fabsf(hi[j]), fabsf(lo[j])));
        }
        const int e = step_exponent(wave_max(most));
        int8_t *dst = a.codes + ((size_t)id * Hkv + c) * 2 * D;
        for (int j = 0; j * 64 + lane < D; ++j) {
            dst[j * 64 + lane] = code_of(ceilf(ldexpf(hi[j], -e)));
            dst[D + j * 64 + lane] = code_of(floorf(ldexpf(lo[j], -e)));
        }
        if (lane == 0) a.scales[(size_t)id * Hkv + c] = ldexpf(1.f, e);
    }
}

// ---- choice of the blocks ---------------------------------------------------------------------------------------------------
// A score as a number whose order is that of the floats; forced blocks above all of them.
constexpr uint32_t kForced = 0xffffffffu;
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Any even head size: a thread to a block, the queries of a batch in LDS as codes [queries][2 D / 4 words], the positive parts before the negative ones.
constexpr int kScoreBatch = 16;
template <typename T>
__global__ void __launch_bounds__(256) k_scores(SelectArgs a, int Hq, int Hkv, int D, int Bk) {
    __shared__ int qs[kScoreBatch][128];
    __shared__ float qstep[kScoreBatch];
    const int s = blockIdx.x / Hkv, c = blockIdx.x % Hkv, g = Hq / Hkv, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int nb = min(blocks_of(max(a.kv_lens[s], 0), Bk), a.max_blocks);
    if ((int)blockIdx.y * 256 >= nb) return;
    const int row0 = min(max(a.row_start[s], 0), a.R), n = (min(max(a.row_start[s + 1], row0), a.R) - row0) * g;
    const int b = blockIdx.y * 256 + threadIdx.x;
    const int id = b < nb ? a.bt[(size_t)s * a.max_blocks + b] : -1;
    const bool good = id >= 0 && id < a.num_blocks;
    const size_t rec = good ? (size_t)id * Hkv + c : 0;
    const int *code = (const int *)(a.codes + rec * 2 * D);
    const int words = D / 2;
    float best = -INFINITY;
    for (int q0 = 0; q0 < n; q0 += kScoreBatch) {
        const int cnt = min(kScoreBatch, n - q0);
        __syncthreads();
        for (int j = w; j < cnt; j += 4) {
            const T *q = (const T *)a.q + ((size_t)(row0 + (q0 + j) / g) * Hq + c * g + (q0 + j) % g) * D;
            float most = 0.f;
            for (int i = lane; i < D; i += 64) most = fmaxf(most, fabsf(finite_or_edge(Elem<T>::ld(q + i))));
            const int e = step_exponent(wave_max(most));
            int8_t *dst = (int8_t *)qs[j];
            for (int i = lane; i < D; i += 64) {
                const int v = code_of(rintf(ldexpf(finite_or_edge(Elem<T>::ld(q + i)), -e)));
                dst[i] = (int8_t)max(v, 0);
                dst[D + i] = (int8_t)min(v, 0);
            }
            if (lane == 0) qstep[j] = ldexpf(1.f, e);
        }
        __syncthreads();
        if (!good) continue;
        int acc[kScoreBatch];
#pragma unroll
        for (int j = 0; j < kScoreBatch; ++j) acc[j] = 0;
        for (int i = 0; i < words; ++i) {
            const int k = code[i];
#pragma unroll
            for (int j = 0; j < kScoreBatch; ++j) acc[j] = __builtin_amdgcn_sdot4(k, qs[j][i], acc[j], false);
        }
#pragma unroll
        for (int j = 0; j < kScoreBatch; ++j)
            if (j < cnt) best = fmaxf(best, (float)acc[j] * qstep[j]);
    }
    if (b >= nb) return;
    uint32_t key = order_key(good ? (n ? best * a.scales[rec] : 0.f) : -INFINITY);
    if (b < a.first || b >= nb - a.last) key = kForced;
    ((uint32_t *)a.scores)[((size_t)s * Hkv + c) * a.max_blocks + b] = key;
}

// The top_k largest keys of a sequence and kv-head, lowest index first among equal ones: the k-th largest key is found eight bits at a
// time from counts in LDS (whole numbers: their order does not matter), then one pass in the order of the blocks writes the list.
__global__ void __launch_bounds__(256) k_pick(SelectArgs a, int Hkv, int Bk) {
    __shared__ int hist[256], wave_gt[4], wave_eq[4], chosen[2];
    const int s = blockIdx.x / Hkv, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int nb = min(blocks_of(max(a.kv_lens[s], 0), Bk), a.max_blocks), k = min(a.top_k, nb);
    const uint32_t *keys = (const uint32_t *)a.scores + (size_t)blockIdx.x * a.max_blocks;
    int32_t *out = a.blocks + (size_t)blockIdx.x * a.top_k;
    if (threadIdx.x == 0 && blockIdx.x % Hkv == 0) a.counts[s] = k;
    for (int i = k + threadIdx.x; i < a.top_k; i += 256) out[i] = -1;
    if (nb <= a.top_k) {
        for (int i = threadIdx.x; i < nb; i += 256) out[i] = i;
        return;
    }
    uint32_t prefix = 0;  // the bits of the k-th largest key found so far
    int left = k;         // its rank among the keys that share them
    for (int shift = 24; shift >= 0; shift -= 8) {
        hist[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < nb; i += 256) {
            const uint32_t key = keys[i];
            if (shift == 24 || (key >> (shift + 8)) == prefix) atomicAdd(&hist[(key >> shift) & 255], 1);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int bin = 255, above = 0;
            while (above + hist[bin] < left) above += hist[bin--];
            chosen[0] = bin;
            chosen[1] = above;
        }
        __syncthreads();
        prefix = prefix << 8 | (uint32_t)chosen[0];
        left -= chosen[1];
    }
    // `left` of the keys equal to `prefix` are taken, and all larger ones
    int at = 0, eq_before = 0;
    for (int i0 = 0; i0 < nb; i0 += 256) {
        const int i = i0 + threadIdx.x;
        const uint32_t key = i < nb ? keys[i] : 0;
        const bool gt = i < nb && key > prefix, eq = i < nb && key == prefix;
        const unsigned long long m_gt = __ballot(gt), m_eq = __ballot(eq), below = (1ull << lane) - 1;
        __syncthreads();
        if (lane == 0) {
            wave_gt[w] = __popcll(m_gt);
            wave_eq[w] = __popcll(m_eq);
        }
        __syncthreads();
        int gts = 0, eqs = 0, all_gt = 0, all_eq = 0;
        for (int j = 0; j < 4; ++j) {
            if (j < w) { gts += wave_gt[j]; eqs += wave_eq[j]; }
            all_gt += wave_gt[j];
            all_eq += wave_eq[j];
        }
        gts += __popcll(m_gt & below);
        eqs += __popcll(m_eq & below);
        const int rank = eq_before + eqs;  // among the equal ones
        if (gt || (eq && rank < left)) out[at + gts + min(rank, left) - min(eq_before, left)] = i;
        at += all_gt + min(eq_before + all_eq, left) - min(eq_before, left);
        eq_before += all_eq;
    }
}

}  // namespace

hipError_t launch_extend(const ExtendArgs &a, hipStream_t st) {
    const int rows_per_wg = 512;
    const int wgs = a.max_rows > rows_per_wg ? (a.max_rows + rows_per_wg - 1) / rows_per_wg : 1;
    hipLaunchKernelGGL(k_extend, dim3(wgs), dim3(kExtThreads), 0, st, a, rows_per_wg);
    return hipGetLastError();
}

hipError_t launch_append(const Dims &dm, const AppendArgs &a, hipStream_t st) {
    DISPATCH_TK(dm.bf16, dm.kv8, hipLaunchKernelGGL((k_append<T, KT>), dim3(a.R, (dm.Hq + 2 * dm.Hkv + 3) / 4), dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.D,
                                                    dm.Bk, log2(dm.theta), dm.eps, dm.qk_norm, dm.k_scale, dm.v_scale));
    return hipGetLastError();
}

hipError_t launch_bounds(const Dims &dm, const BoundsArgs &a, hipStream_t st) {
    const int most = a.max_new > 0 ? min(a.max_blocks, (a.max_new - 1) / dm.Bk + 2) : a.max_blocks;
    DISPATCH_TK(dm.bf16, dm.kv8, {
        (void)sizeof(T);
        hipLaunchKernelGGL(k_bounds<KT>, dim3(a.S, min(most, 65535), (dm.Hkv + 3) / 4), dim3(256), 0, st, a, dm.Hkv, dm.D, dm.Bk);
    });
    return hipGetLastError();
}

hipError_t launch_select(const Dims &dm, const SelectArgs &a, hipStream_t st) {
    DISPATCH_T(dm.bf16, hipLaunchKernelGGL(k_scores<T>, dim3(a.S * dm.Hkv, (a.max_blocks + 255) / 256), dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.D, dm.Bk));
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_pick, dim3(a.S * dm.Hkv), dim3(256), 0, st, a, dm.Hkv, dm.Bk);
    return hipGetLastError();
}

}  // namespace icarus
