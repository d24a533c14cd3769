// Operators with lengths on the device: growth of the sequences, rotation and append, bounds of the keys, choice of the
// blocks.  Everything a kernel indexes with -- lengths, slots, block ids -- comes from device memory and is checked
// where it is used.
#include "block_ops.h"
#include "block_util.h"

#include <algorithm>
#include <type_traits>

namespace icarus {
namespace {

// ---- growth of the sequences ------------------------------------------------------------------------------------------
// Two sums over the sequences decide everything: rows before a sequence, and blocks taken before it.  Every workgroup
// forms both over all sequences (8-12 bytes each, from L2) and writes its own range of rows, so that one launch does and no
// workgroup waits for another.  Sums saturate just past the largest value that is told apart (max_rows, n_free), so that no length overflows them.
// Bound by its chain of reads, sums and barriers: 64 sequences, 374 rows 5.3 us; 256 sequences, 62208 rows 6.2 us (two rows to a thread 7.1, four 8.8).
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

__global__ void __launch_bounds__(kExtThreads) k_extend(ExtendArgs a) {
    __shared__ int row_begin[kExtSeg], row_end[kExtSeg], first_id[kExtSeg], ctx[kExtSeg], fresh[kExtSeg], red[kExtThreads / 64];
    const int row_cap = a.max_rows + 1, id_cap = a.n_free + 1;
    const int r0 = blockIdx.x * kExtThreads, r1 = min(a.max_rows, r0 + kExtThreads);
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
            need[j] = ok[j] ? min(blocks_of(c[j] + nw[j], a.Bk) - blocks_of(c[j], a.Bk), id_cap) : 0;
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
// Cosine and sine of pos * theta^(-2i/D), in float64 and rounded once: a far position keeps the fraction of its last turn.  A cache entry must not depend on which
// call appended it, so the angles, and the order in which a norm's squares are summed, are those of the kernels behind icarus_prefill_kv and icarus_decode_step.
__device__ __forceinline__ double frequency_of(int i, int D, double log2_theta) { return exp2(-(2.0 * (double)i / (double)D) * log2_theta); }
__device__ __forceinline__ void angle_of(int pos, double frequency, float *cs, float *sn) {
    double s, c;
    sincos((double)pos * frequency, &s, &c);
    *cs = (float)c;
    *sn = (float)s;
}

// Any head size and block size, rows at any distance: a wave to a head of a row, a pair to a lane, V written element by element (16384 rows of 48 heads of 128,
// 402 MB: 366 us; 356 rows of them 7.8 us; angles taken by every wave for itself 455 and 9.8).
template <typename T, typename KT>
__global__ void __launch_bounds__(256) k_append(AppendArgs a, int Hq, int Hkv, int D, int Bk, double log2_theta, float eps, int qk_norm,
                                                float k_scale, float v_scale) {
    __shared__ float cos_t[128], sin_t[128];
    const int row = a.first + blockIdx.x, h = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, half = D >> 1;
    const int pos = a.row_pos[row];
    if (pos < 0) return;
    if ((int)blockIdx.y * 4 < Hq + Hkv) {  // the row's angles, for the four heads
        for (int i = threadIdx.x; i < half; i += 256) angle_of(pos, frequency_of(i, D, log2_theta), cos_t + i, sin_t + i);
        __syncthreads();
    }
    if (h >= Hq + 2 * Hkv) return;
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
        float x = Elem<T>::ld(src + i), y = Elem<T>::ld(src + i + half), rx, ry;
        if (qk_norm) {
            const T *w = (const T *)(h < Hq ? a.q_norm : a.k_norm);
            x = x * inv * Elem<T>::ld(w + i);
            y = y * inv * Elem<T>::ld(w + i + half);
        }
        rotate_pair(x, y, cos_t[i], sin_t[i], &rx, &ry);
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

// Head sizes 64, 128 and 256, blocks of 16.  Bound by HBM where there are many rows, by the chain of its reads where there are few.
// A workgroup takes a window of 16 rows and a part of their rotated heads or of their values.  LPH = D / 8 lanes hold a head, four pairs to a lane, so that both halves of a
// row of 128 bfloat16 are read and written as whole lines; a lane keeps its row's angles for all heads of the part.
// V goes into the pool transposed: a run of rows that are consecutive places of one block is put together in LDS and written as one row of the block per
// channel, 32 bytes at once where the run fills the block.  A run belongs to the window in which it starts, wherever it ends, so that prompts which begin
// inside a block are written in whole blocks too.
// The values have workgroups of their own, whose chain of reads runs beside the other.  16384 rows of 48 heads of 128 (402 MB): 92 us, 4.4 TB/s (a wave to a head
// 366); 1145 rows of 80 heads into an FP8 cache (44 MB): 15.4 us (48); 356 rows of 48 heads 5.6 us (7.8).  With angles in float32 half turns, which differ from the other
// kernels' in the last bit, 92, 14.5 and 5.3, and then with the values after the rotation in one workgroup 97, 18 and 6.9.
template <typename KT> __device__ __forceinline__ void put4(KT *p, const float (&v)[4], float scale);
template <> __device__ __forceinline__ void put4(bf16_t *p, const float (&v)[4], float) { *(uint2 *)p = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])); }
template <> __device__ __forceinline__ void put4(float *p, const float (&v)[4], float) { *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]); }
template <> __device__ __forceinline__ void put4(fp8_t *p, const float (&v)[4], float scale) {
    *(uint32_t *)p = f32_to_fp8(v[0] / scale) | f32_to_fp8(v[1] / scale) << 8 | f32_to_fp8(v[2] / scale) << 16 | f32_to_fp8(v[3] / scale) << 24;
}

constexpr int kWindow = 16;
// What a wave wrote to LDS is what it reads next: an order for the compiler, the hardware keeps it anyway.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// Squares of a head whose pairs (x, y) 4 l .. 4 l + 3 lane l of its D / 8 holds, in the order of a wave that adds elements i, i + 64, .. in lane i and then lanes 32, 16, .. 1 apart.
template <int D> __device__ __forceinline__ float sum_of_squares(const float (&x)[4], const float (&y)[4]) {
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (D == 64) {  // two lanes' squares: each is rounded
            float a = x[e] * x[e], b = y[e] * y[e];
            asm("" : "+v"(a), "+v"(b));
            p[e] = a + b;
        } else if constexpr (D == 128) {
            p[e] = __builtin_fmaf(y[e], y[e], x[e] * x[e]);
        } else {  // pairs i and i + 64 of one lane, whose values lie 16 lanes apart here: both lanes add them in the order of i
            static_assert(D == 256, "");
            const bool up = threadIdx.x & 16;
            const float x2 = __shfl_xor(x[e], 16, 64), y2 = __shfl_xor(y[e], 16, 64);
            const float a = up ? x2 : x[e], b = up ? x[e] : x2, c = up ? y2 : y[e], d = up ? y[e] : y2;
            p[e] = __builtin_fmaf(d, d, __builtin_fmaf(c, c, __builtin_fmaf(b, b, a * a)));
        }
#pragma unroll
        for (int o = D == 64 ? 4 : 8; o > 0; o >>= 1) p[e] += __shfl_xor(p[e], o, 64);
    }
    return (p[0] + p[2]) + (p[1] + p[3]);
}

template <typename T, typename KT, int D>
__global__ void __launch_bounds__(256) k_append_window(AppendArgs a, int Hq, int Hkv, int parts, double log2_theta, float eps, int qk_norm, float k_scale, float v_scale) {
    constexpr int Bk = 16, LPH = D / 8, HALF = D / 2, ROWS = 256 / LPH, VW = 16 / sizeof(T);  // ROWS: heads of a pass; VW: elements of 16 bytes
    __shared__ double frequency[HALF];
    __shared__ __attribute__((aligned(16))) T tile[4][Bk][D];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r0 = a.first + blockIdx.x * kWindow;
    const int n_rot = Hq + Hkv;
    if ((int)blockIdx.y < parts) {
        for (int i = threadIdx.x; i < HALF; i += 256) frequency[i] = frequency_of(i, D, log2_theta);
        __syncthreads();
        // Rotated heads of this part, [h0, h1): with fewer than 16 lanes to a head the lanes of a row take neighbouring heads.
        constexpr int HPR = ROWS > kWindow ? ROWS / kWindow : 1;  // heads of a row at a time
        const int h0 = n_rot * blockIdx.y / parts, h1 = n_rot * (blockIdx.y + 1) / parts;
        const int sub = threadIdx.x / LPH, i4 = 4 * (threadIdx.x % LPH);
        for (int rr = sub / HPR; rr < kWindow; rr += ROWS / HPR) {
            const int row = r0 + rr, pos = row < a.R ? a.row_pos[row] : -1;
            if (pos < 0) continue;
            const int64_t slot = a.row_slot[row];
            const bool write = slot >= 0 && slot < a.n_slots;
            float cs[4], sn[4], wq[2][4], wk[2][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) angle_of(pos, frequency[i4 + e], &cs[e], &sn[e]);
            if (qk_norm)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    Quad<T>::get(*(const typename Quad<T>::raw *)((const T *)a.q_norm + h * HALF + i4), wq[h]);
                    Quad<T>::get(*(const typename Quad<T>::raw *)((const T *)a.k_norm + h * HALF + i4), wk[h]);
                }
            const T *src = (const T *)a.qkv + (size_t)row * a.ld + i4;
            KT *kdst = (KT *)a.pool + (write ? ((size_t)(slot / Bk) * Hkv * 2 * Bk + (size_t)(slot % Bk)) * D : 0) + i4;
            const int end = write ? h1 : min(h1, Hq);  // a stream's key heads are not read
            constexpr int U = 4;  // heads whose reads are under way together
            for (int hu = h0 + sub % HPR; hu < end; hu += U * HPR) {
                typename Quad<T>::raw lo[U], up[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const T *p = src + (size_t)min(hu + u * HPR, end - 1) * D;
                    lo[u] = *(const typename Quad<T>::raw *)p;
                    up[u] = *(const typename Quad<T>::raw *)(p + HALF);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int h = hu + u * HPR;
                    if (h >= end) break;
                    float x[4], y[4], rx[4], ry[4];
                    Quad<T>::get(lo[u], x);
                    Quad<T>::get(up[u], y);
                    if (qk_norm) {
                        const float inv = rsqrtf(sum_of_squares<D>(x, y) / (float)D + eps);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            x[e] = x[e] * inv * (h < Hq ? wq[0][e] : wk[0][e]);
                            y[e] = y[e] * inv * (h < Hq ? wq[1][e] : wk[1][e]);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) rotate_pair(x[e], y[e], cs[e], sn[e], &rx[e], &ry[e]);
                    if (h < Hq) {
                        T *dst = (T *)a.q_out + ((size_t)row * Hq + h) * D + i4;
                        put4(dst, rx, 1.f);
                        put4(dst + HALF, ry, 1.f);
                    } else {
                        KT *dst = kdst + (size_t)(h - Hq) * 2 * Bk * D;
                        put4(dst, rx, k_scale);
                        put4(dst + HALF, ry, k_scale);
                    }
                }
            }
        }
        return;
    }
    // V: lane l < 32 looks at row r0 + l; the rows behind the window matter for runs that start in it.
    const int v_part = blockIdx.y - parts, v_parts = gridDim.y - parts, v0 = Hkv * v_part / v_parts, n_v = Hkv * (v_part + 1) / v_parts - v0;
    int64_t slot = -1, before = -1;
    if (lane < 32) {
        auto place = [&](int row) {
            if (row < 0 || row >= a.R || a.row_pos[row] < 0) return (int64_t)-1;
            const int64_t x = a.row_slot[row];
            return x < a.n_slots ? x : (int64_t)-1;
        };
        slot = place(r0 + lane);
        before = place(r0 + lane - 1);
    }
    const bool there = slot >= 0, goes_on = there && before >= 0 && slot == before + 1 && slot % Bk != 0;
    const uint32_t going = (uint32_t)__ballot(goes_on);
    uint32_t starts = (uint32_t)__ballot(there && !goes_on) & 0xffffu;
    const int n_runs = __popc(starts);
    if (n_runs == 0) return;
    int at = w;  // of the runs x heads of this part
    for (int run = 0; run < n_runs; ++run, starts &= starts - 1) {
        const int l = __ffs((int)starts) - 1, n = 1 + __builtin_ctz(~(going >> l >> 1));  // a run ends at a block's end: at most 16
        const int64_t first = ((int64_t)__shfl((int)(slot >> 32), l, 64) << 32) | (uint32_t)__shfl((int)slot, l, 64);
        const size_t blk = (size_t)(first / Bk);
        const int off = (int)(first % Bk);
        for (; at < (run + 1) * n_v; at += 4) {
            const int c = v0 + at - run * n_v;
            const T *src = (const T *)a.qkv + (size_t)(r0 + l) * a.ld + (size_t)(Hq + Hkv + c) * D;
            KT *dst = (KT *)a.pool + ((blk * Hkv + c) * 2 + 1) * Bk * D;
            if (n == 1) {
                for (int d = lane; d < D; d += 64) KVElem<KT>::st(dst + d * Bk + off, Elem<T>::ld(src + d), v_scale);
                continue;
            }
            constexpr int CH = D / VW;  // 16-byte pieces of a row
#pragma unroll
            for (int i = 0; i < Bk * CH / 64; ++i) {
                const int t = (i * 64 + lane) / CH, d = (i * 64 + lane) % CH * VW;
                if (t < n) *(uint4 *)&tile[w][t][d] = *(const uint4 *)(src + (size_t)t * a.ld + d);
            }
            wave_fence();  // the tile is this wave's own, and a wave's LDS accesses go in order
            for (int d = lane; d < D; d += 64) {
                if (n == Bk) {
                    if constexpr (sizeof(KT) == 1) {
                        uint32_t o[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            o[i] = 0;
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[i] |= f32_to_fp8(Elem<T>::ld(&tile[w][4 * i + e][d]) / v_scale) << 8 * e;
                        }
                        *(uint4 *)(dst + d * Bk) = make_uint4(o[0], o[1], o[2], o[3]);
                    } else {
                        constexpr int PER = 4 / sizeof(KT);  // elements of a word: the same type on both sides, the bits are moved as they are
                        uint32_t o[Bk / PER];
#pragma unroll
                        for (int i = 0; i < Bk / PER; ++i) {
                            if constexpr (PER == 2) o[i] = (uint32_t)tile[w][2 * i][d] | (uint32_t)tile[w][2 * i + 1][d] << 16;
                            else o[i] = __float_as_uint(tile[w][i][d]);
                        }
#pragma unroll
                        for (int i = 0; i < Bk / PER / 4; ++i) ((uint4 *)(dst + d * Bk))[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    }
                } else {
                    for (int t = 0; t < n; ++t) KVElem<KT>::st(dst + d * Bk + off + t, Elem<T>::ld(&tile[w][t][d]), v_scale);
                }
            }
            wave_fence();
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

// Any shape: a wave to a block and kv-head, a channel to a lane (16384 blocks of 8 heads of 128, 571 MB: 338 us).
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

// Blocks of 16, head sizes 64, 128 and 256: a wave to the keys of a block and kv-head, which it reads as they lie, four channels of a token to a lane; a lane sees 4 to 16 of
// the tokens, and lanes of the same channels meet by exchanges in registers.  Bound by HBM (half of a block's lines), with the vector units close behind: with
// 16 bytes to a lane there were twice the exchanges and the reads waited for them.  bfloat16 pairs stay pairs: as whole numbers of 16 bits whose order is that of the values two
// are compared at a time.  16384 blocks of 8 heads of 128 (537 MB of keys, 4 KB of every 8 KB, and 34 MB out): 121 us, 4.7 TB/s (16 bytes to a lane: 129).
typedef short s16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ s16x2_t ordered(uint32_t u) {  // two bfloat16 -> whole numbers in their order; its own inverse
    const s16x2_t x = __builtin_bit_cast(s16x2_t, u);
    return x ^ ((x >> 15) & s16x2_t{0x7fff, 0x7fff});
}

// op over lanes that are O apart, O = 16 or 32, in both of them.
template <int O, typename V, typename Op> __device__ __forceinline__ V with_lane(V x, Op op) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    if constexpr (O == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return op(__builtin_bit_cast(V, (uint32_t)r[0]), __builtin_bit_cast(V, (uint32_t)r[1]));
    } else {
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        return op(__builtin_bit_cast(V, (uint32_t)r[0]), __builtin_bit_cast(V, (uint32_t)r[1]));
    }
}
// The largest of the wave's lanes, in each of them; inside 16 lanes as operands of the maximum itself.
__device__ __forceinline__ float max_of_lanes(float x) {
    auto step = [&](auto ctrl) { x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true))); };
    step(std::integral_constant<int, 0xb1>());   // quad 1 0 3 2
    step(std::integral_constant<int, 0x4e>());   // quad 2 3 0 1
    step(std::integral_constant<int, 0x141>());  // mirrored in 8
    step(std::integral_constant<int, 0x140>());  // mirrored in 16
    auto most = [](float a, float b) { return fmaxf(a, b); };
    return with_lane<32>(with_lane<16>(x, most), most);
}

template <typename KT, int D>
__global__ void __launch_bounds__(256) k_bounds_wave(BoundsArgs a, int Hkv) {
    constexpr int Bk = 16, LPT = D / 4, TPI = 64 / LPT, NI = Bk / TPI;  // lanes of a token, tokens of a read, reads
    typedef typename Quad<KT>::raw raw;
    const int s = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6, t0 = lane / LPT;
    const int from = max(a.from_lens[s], 0), to = (int)min((int64_t)max(a.to_lens[s], 0), (int64_t)a.max_blocks * Bk);
    if (from >= to) return;
    const int b_end = (to - 1) / Bk + 1;
    const int32_t *bt = a.bt + (size_t)s * a.max_blocks;
    int b = from / Bk + blockIdx.y, id = b < b_end ? bt[b] : -1;
    for (; b < b_end; b += gridDim.y) {
        const int here = id, n = min(Bk, to - b * Bk);
        if (b + (int)gridDim.y < b_end) id = bt[b + gridDim.y];
        if (here < 0 || here >= a.num_blocks) continue;
        for (int c = w; c < Hkv; c += 4) {
            const size_t rec = (size_t)here * Hkv + c;
            const raw *src = (const raw *)((const KT *)a.pool + rec * 2 * Bk * D) + lane % LPT;
            raw r[NI];  // behind the last token: the last again
#pragma unroll
            for (int i = 0; i < NI; ++i) r[i] = src[min(i * TPI + t0, n - 1) * LPT];
            float hi[4], lo[4];
            auto by_value = [&] {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    hi[e] = -INFINITY;
                    lo[e] = INFINITY;
                }
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    float v[4];
                    Quad<KT>::get(r[i], v);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = finite_or_edge(v[e]);
                        hi[e] = fmaxf(hi[e], x);
                        lo[e] = fminf(lo[e], x);
                    }
                }
                auto most = [](float x, float y) { return fmaxf(x, y); };
                auto least = [](float x, float y) { return fminf(x, y); };
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (LPT <= 16) {
                        hi[e] = with_lane<16>(hi[e], most);
                        lo[e] = with_lane<16>(lo[e], least);
                    }
                    if constexpr (LPT <= 32) {
                        hi[e] = with_lane<32>(hi[e], most);
                        lo[e] = with_lane<32>(lo[e], least);
                    }
                }
            };
            if constexpr (sizeof(KT) == 2) {
                s16x2_t h[2], l[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    h[e] = s16x2_t{-32768, -32768};
                    l[e] = s16x2_t{32767, 32767};
                }
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const s16x2_t x = ordered(e ? r[i].y : r[i].x);
                        h[e] = __builtin_elementwise_max(h[e], x);
                        l[e] = __builtin_elementwise_min(l[e], x);
                    }
                auto most = [](s16x2_t x, s16x2_t y) { return __builtin_elementwise_max(x, y); };
                auto least = [](s16x2_t x, s16x2_t y) { return __builtin_elementwise_min(x, y); };
                bool odd = false;  // an infinity or a NaN
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if constexpr (LPT <= 16) {
                        h[e] = with_lane<16>(h[e], most);
                        l[e] = with_lane<16>(l[e], least);
                    }
                    if constexpr (LPT <= 32) {
                        h[e] = with_lane<32>(h[e], most);
                        l[e] = with_lane<32>(l[e], least);
                    }
                    odd |= max(h[e][0], h[e][1]) >= 0x7f80 || min(l[e][0], l[e][1]) <= -0x7f81;
                }
                if (__any(odd)) {
                    by_value();
                } else {
                    Quad<bf16_t>::get(make_uint2(__builtin_bit_cast(uint32_t, ordered(__builtin_bit_cast(uint32_t, h[0]))),
                                                 __builtin_bit_cast(uint32_t, ordered(__builtin_bit_cast(uint32_t, h[1])))), hi);
                    Quad<bf16_t>::get(make_uint2(__builtin_bit_cast(uint32_t, ordered(__builtin_bit_cast(uint32_t, l[0]))),
                                                 __builtin_bit_cast(uint32_t, ordered(__builtin_bit_cast(uint32_t, l[1])))), lo);
                }
            } else {
                by_value();
            }
            float most = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) most = fmaxf(most, fmaxf(fabsf(hi[e]), fabsf(lo[e])));
            const int e2 = step_exponent(max_of_lanes(most));
            const float inv = ldexpf(1.f, -e2);
            // The first token's lanes write the largest, the second's the smallest: floor(x) = -ceil(-x), so that one way serves both.
            auto put = [&](bool low) {
                const float turn = low ? -inv : inv;
                uint32_t word = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int x = (int)fminf(fmaxf(ceilf((low ? lo : hi)[e] * turn), -127.f), 127.f);
                    word |= (uint32_t)(uint8_t)(low ? -x : x) << 8 * e;
                }
                ((uint32_t *)(a.codes + rec * 2 * D))[(low ? LPT : 0) + lane % LPT] = word;
            };
            if constexpr (TPI > 1) {
                if (t0 < 2) put(t0 == 1);
            } else {
                put(false);
                put(true);
            }
            if (lane == 0) a.scales[rec] = ldexpf(1.f, e2);
        }
    }
}

// ---- choice of the blocks ---------------------------------------------------------------------------------------------------
// A score as a number whose order is that of the floats.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// Blocks of a sequence that a choice is made from: [first, nb - last) of them compete, the others are taken.
__device__ __forceinline__ int n_blocks_of(const SelectArgs &a, int s, int Bk) { return min(blocks_of(max(a.kv_lens[s], 0), Bk), a.max_blocks); }

// Scores on the matrix cores, head sizes 64, 128, 192, 256: a wave to 16 * TB blocks.  Codes of a block are the columns of 16x16x64 products in 8 bits, a query's positive
// parts (as many as the largest keys) and negative parts (smallest keys) the rows.  In both operands a lane holds 16 bytes of one row or column,
// which is how codes lie in memory and what a lane quantises by itself: a query's 16 channels of one step, the same for both parts.  The four waves
// quantise a tile of 16 queries each and share them; their codes are on the way meanwhile.  Each workgroup is one chain of reads (length, ids, codes), so many small ones at a
// time do best: 64 sequences of 1024-16384 tokens, 1-8 agents (73 MB) 19 us with five waves to a SIMD, 21 with four, 28 with six (the registers do not hold the codes);
// 23 us where a workgroup goes on to further blocks with the next codes on their way.
typedef int i32x4 __attribute__((ext_vector_type(4)));
template <typename T> __device__ __forceinline__ void load16(const T *p, float (&v)[16]) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 r = *(const uint4 *)(p + 8 * h);
            const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[8 * h + 2 * i] = __uint_as_float(u[i] << 16);
                v[8 * h + 2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
            }
        }
    } else {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const float4 r = *(const float4 *)(p + 4 * h);
            v[4 * h] = r.x; v[4 * h + 1] = r.y; v[4 * h + 2] = r.z; v[4 * h + 3] = r.w;
        }
    }
}
// Four rounded multiples of 2^-e: the bytes of their positive and of their negative parts.  The conversion to whole numbers makes 0 of a NaN and
// saturates, so values need no looking at before.
__device__ __forceinline__ void quantise4(const float *v, float inv, int *up, int *down) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    s16x2 h[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int x, y;
        asm("v_cvt_i32_f32 %0, %1" : "=v"(x) : "v"(rintf(v[2 * k] * inv)));
        asm("v_cvt_i32_f32 %0, %1" : "=v"(y) : "v"(rintf(v[2 * k + 1] * inv)));
        h[k] = __builtin_bit_cast(s16x2, __builtin_amdgcn_cvt_pk_i16(x, y));
    }
    const s16x2 most = {127, 127}, none = {0, 0}, least = {-127, -127};
    const uint32_t u0 = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_elementwise_max(h[0], none), most));
    const uint32_t u1 = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_elementwise_max(h[1], none), most));
    const uint32_t d0 = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_elementwise_min(h[0], none), least));
    const uint32_t d1 = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_elementwise_min(h[1], none), least));
    *up = (int)__builtin_amdgcn_perm(u1, u0, 0x06040200);  // bytes 0 and 2 of both words
    *down = (int)__builtin_amdgcn_perm(d1, d0, 0x06040200);
}
// A sequence's queries of one kv-head: n of them, query j in row row0 + j / g, head c * g + j % g.
template <typename T> struct Stack {
    const T *q;
    int row0, n, g, c, Hq;
    __device__ __forceinline__ Stack(const SelectArgs &a, int s, int c_, int Hq_, int Hkv) : q((const T *)a.q), g(Hq_ / Hkv), c(c_), Hq(Hq_) {
        row0 = min(max(a.row_start[s], 0), a.R);
        n = (min(max(a.row_start[s + 1], row0), a.R) - row0) * g;
    }
};
// Queries j0 .. j0 + 15 (behind the last: the last again) as rows of the products: rows[step][lane], steps[query].
template <typename T, int KS>
__device__ __forceinline__ void quantise_tile(const Stack<T> &x, int j0, i32x4 (*rows)[64], float *steps, int lane) {
    constexpr int D = KS * 32, H = KS / 2;
    const int m = lane & 15, q4 = lane >> 4, j = min(j0 + m, x.n - 1);
    const T *q = x.q + ((size_t)(x.row0 + j / x.g) * x.Hq + x.c * x.g + j % x.g) * D + 16 * q4;
    float v[H][16], most = 0.f;
#pragma unroll
    for (int ks = 0; ks < H; ++ks) load16(q + 64 * ks, v[ks]);
#pragma unroll
    for (int ks = 0; ks < H; ++ks)
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(v[ks][i]));  // a NaN is passed over
    most = fmaxf(most, __shfl_xor(most, 16, 64));
    most = fmaxf(most, __shfl_xor(most, 32, 64));
    const int e = step_exponent(fminf(most, 3.402823466e38f));
    const float inv = ldexpf(1.f, -e);
#pragma unroll
    for (int ks = 0; ks < H; ++ks) {
        i32x4 up, down;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int u, d;
            quantise4(v[ks] + 4 * i, inv, &u, &d);
            up[i] = u;
            down[i] = d;
        }
        rows[ks][lane] = up;
        rows[ks + H][lane] = down;
    }
    if (q4 == 0) steps[m] = ldexpf(1.f, e);
}
// Codes of blocks b0 .. b0 + 16 TB - 1, a column to a lane; scale 0: no such block in the pool.
template <int KS, int TB> struct Codes {
    i32x4 code[TB][KS];
    float scale[TB];
    __device__ __forceinline__ void load(const SelectArgs &a, int s, int c, int Hkv, int b0, int nb, int lane) {
        constexpr int D = KS * 32;
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            const int b = b0 + 16 * t + (lane & 15), id = b < nb ? a.bt[(size_t)s * a.max_blocks + b] : -1;
            const bool good = id >= 0 && id < a.num_blocks;
            const size_t rec = good ? (size_t)id * Hkv + c : 0;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) code[t][ks] = *(const i32x4 *)(a.codes + rec * 2 * D + 64 * ks + 16 * (lane >> 4));
            scale[t] = good ? a.scales[rec] : 0.f;
        }
    }
    // the largest of a tile's scores, so far; lanes 16 apart have other queries of the same block
    __device__ __forceinline__ void score(float (&best)[TB], const i32x4 (*rows)[64], const float *steps, int lane) const {
        i32x4 sum[TB];
#pragma unroll
        for (int t = 0; t < TB; ++t) sum[t] = i32x4{0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const i32x4 r = rows[ks][lane];
#pragma unroll
            for (int t = 0; t < TB; ++t) sum[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(r, code[t][ks], sum[t], 0, 0, 0);
        }
        const float4 st = *(const float4 *)(steps + 4 * (lane >> 4));
#pragma unroll
        for (int t = 0; t < TB; ++t)
            best[t] = fmaxf(fmaxf(fmaxf(best[t], (float)sum[t][0] * st.x), fmaxf((float)sum[t][1] * st.y, (float)sum[t][2] * st.z)), (float)sum[t][3] * st.w);
    }
    __device__ __forceinline__ uint32_t key(int t, float best, int n) const {
        best = fmaxf(best, __shfl_xor(best, 16, 64));
        best = fmaxf(best, __shfl_xor(best, 32, 64));
        return order_key(scale[t] > 0.f ? (n ? best * scale[t] : 0.f) : -INFINITY);
    }
};

template <typename T, int KS, int TB>
__global__ void __launch_bounds__(256, KS <= 4 ? 5 : 1) k_scores_mfma(SelectArgs a, int Hq, int Hkv, int Bk) {
    __shared__ i32x4 rows[4][KS][64];  // four tiles of queries
    __shared__ __attribute__((aligned(16))) float steps[4][16];
    const int pair = blockIdx.x, s = pair / Hkv, c = pair - s * Hkv, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int nb = n_blocks_of(a, s, Bk);
    if ((int)blockIdx.y * 64 * TB >= nb - a.last || nb <= a.top_k) return;  // all of them are taken
    const int b0 = (blockIdx.y * 4 + w) * 16 * TB;
    const Stack<T> x(a, s, c, Hq, Hkv);
    Codes<KS, TB> codes;
    codes.load(a, s, c, Hkv, b0, nb, lane);
    float best[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) best[t] = -INFINITY;
    for (int j0 = 0; j0 < x.n; j0 += 64) {
        if (j0 + 16 * w < x.n) quantise_tile<T, KS>(x, j0 + 16 * w, rows[w], steps[w], lane);
        __syncthreads();
        for (int j = 0; j < min(4, (x.n - j0 + 15) / 16); ++j) codes.score(best, rows[j], steps[j], lane);
        __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < TB; ++t) {
        const uint32_t key = codes.key(t, best[t], x.n);
        const int b = b0 + 16 * t + lane;
        if (lane < 16 && b < nb) ((uint32_t *)a.scores)[(size_t)pair * key_pitch(a.max_blocks) + b] = key;
    }
}

// Any even head size: a thread to a block, the queries of a batch in LDS as codes [queries][2 D / 4 words], the positive parts before the negative ones
// (64 sequences as above: 114 us).
constexpr int kScoreBatch = 16;
template <typename T>
__global__ void __launch_bounds__(256) k_scores(SelectArgs a, int Hq, int Hkv, int D, int Bk) {
    __shared__ int qs[kScoreBatch][128];
    __shared__ float qstep[kScoreBatch];
    const int s = blockIdx.x / Hkv, c = blockIdx.x % Hkv, g = Hq / Hkv, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int nb = n_blocks_of(a, s, Bk);
    if ((int)blockIdx.y * 256 >= nb || nb <= a.top_k) return;
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
    ((uint32_t *)a.scores)[((size_t)s * Hkv + c) * key_pitch(a.max_blocks) + b] = order_key(good ? (n ? best * a.scales[rec] : 0.f) : -INFINITY);
}

// The choice of a sequence and kv-head: of the keys that compete the k largest, lowest index first among equal ones.  The k-th largest is found eight bits at
// a time from counts in LDS (whole numbers: their order does not matter), from the highest bit in which the keys differ at all on until all keys that agree so far
// are taken; then each thread knows how many of its neighbouring blocks are taken, and one sum over the workgroup says where they go.  Scores share most of their
// first bits, so eight lanes in turn count in places of their own (32 lists of 7500: 12.2 -> 8.7 us).  Bound by its dependent steps: 8 lists of 2048 5.9 us.
// KPT: keys of a thread, in registers (0: read again in every pass, for any number).
template <int THREADS, int KPT>
__device__ __forceinline__ void pick(const SelectArgs &a, int nb, const uint32_t *keys, int32_t *out) {
    constexpr int WAVES = THREADS / 64, COPIES = 8;
    __shared__ __attribute__((aligned(16))) int hist[256][COPIES], count[256];
    __shared__ int part[WAVES];
    __shared__ uint32_t low[WAVES], high[WAVES];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int b_end = nb - a.last;  // [first, b_end) compete
    const int per = KPT ? KPT : ((nb + THREADS - 1) / THREADS + 3) & ~3, i0 = threadIdx.x * per;
    uint4 key[KPT ? KPT / 4 : 1];
    const auto competes = [&](int i) { return i >= a.first && i < b_end; };
#pragma unroll
    for (int j = 0; j < KPT / 4; ++j)
        if (i0 + 4 * j < nb) key[j] = *(const uint4 *)(keys + i0 + 4 * j);
    const auto quad = [&](const uint4 &x, int i, auto &&f) {  // what competes of keys i .. i + 3
        if (competes(i)) f(x.x);
        if (competes(i + 1)) f(x.y);
        if (competes(i + 2)) f(x.z);
        if (competes(i + 3)) f(x.w);
    };
    const auto each = [&](auto &&f) {
        if constexpr (KPT > 0) {
#pragma unroll
            for (int j = 0; j < KPT / 4; ++j) quad(key[j], i0 + 4 * j, f);
        } else {
            for (int i = 4 * threadIdx.x; i < nb; i += 4 * THREADS) quad(*(const uint4 *)(keys + i), i, f);
        }
    };
    uint32_t lo = 0xffffffffu, hi = 0;
    each([&](uint32_t x) {
        lo = min(lo, x);
        hi = max(hi, x);
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
    }
    if (lane == 0) {
        low[w] = lo;
        high[w] = hi;
    }
    for (int i = threadIdx.x; i < 256 * COPIES / 4; i += THREADS) ((int4 *)hist)[i] = make_int4(0, 0, 0, 0);
    __syncthreads();
    for (int i = 0; i < WAVES; ++i) {
        lo = min(lo, low[i]);
        hi = max(hi, high[i]);
    }
    int left = a.top_k - a.first - a.last;  // how many of the competing ones are taken; more than `left` compete
    int shift = lo == hi ? 0 : 32 - __clz((int)(lo ^ hi));
    uint32_t prefix = shift == 32 ? 0 : hi >> shift;  // the bits of the key in question that are known, all above `shift`
    while (shift > 0 && left > 0) {
        const int next = max(0, shift - 8);
        const uint32_t mask = (1u << (shift - next)) - 1;
        each([&](uint32_t x) {
            if (shift == 32 || x >> shift == prefix) atomicAdd(&hist[(x >> next) & mask][lane % COPIES], 1);
        });
        __syncthreads();
        if (threadIdx.x < 256) {
            const int4 x = ((const int4 *)hist[threadIdx.x])[0], y = ((const int4 *)hist[threadIdx.x])[1];
            count[255 - threadIdx.x] = x.x + x.y + x.z + x.w + y.x + y.y + y.z + y.w;
            ((int4 *)hist[threadIdx.x])[0] = make_int4(0, 0, 0, 0);
            ((int4 *)hist[threadIdx.x])[1] = make_int4(0, 0, 0, 0);
        }
        __syncthreads();
        // each wave for itself, four bins to a lane from the top: the bin in which the count reaches `left`
        const int4 h = ((const int4 *)count)[lane];
        const int sum = h.x + h.y + h.z + h.w;
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(upto, o, 64);
            if (lane >= o) upto += y;
        }
        const int at = __ffsll((unsigned long long)__ballot(upto >= left)) - 1;
        int above = upto - sum, bin = 255 - 4 * lane, here = h.x;
        if (above + here < left) above += here, --bin, here = h.y;
        if (above + here < left) above += here, --bin, here = h.z;
        if (above + here < left) above += here, --bin, here = h.w;
        prefix = prefix << (shift - next) | (uint32_t)__shfl(bin, at, 64);
        left -= __shfl(above, at, 64);
        shift = next;
        if (__shfl(here, at, 64) == left) break;
    }
    // With left > 0 `prefix` is the key of the last ones taken down to bit `shift`: `left` of those equal to it there are, and all larger ones.
    // With none to take, none is larger.
    const bool any = a.top_k > a.first + a.last;
    const auto above = [&](uint32_t x) { return any && x >> shift > prefix; };
    const auto equal = [&](uint32_t x) { return any && x >> shift == prefix; };
    const auto mine = [&](auto &&f) {  // of this thread's neighbours
        const auto one = [&](int i, uint32_t x) {
            if (i < nb) f(i, !competes(i) || above(x), competes(i) && equal(x));
        };
#pragma unroll KPT ? KPT / 4 : 1
        for (int j = 0; j < (KPT ? KPT / 4 : per / 4); ++j) {
            const int i = i0 + 4 * j;
            if (i >= nb) continue;
            const uint4 x = KPT ? key[KPT ? j : 0] : *(const uint4 *)(keys + i);
            one(i, x.x);
            one(i + 1, x.y);
            one(i + 2, x.z);
            one(i + 3, x.w);
        }
    };
    int gt = 0, eq = 0;
    mine([&](int, bool more, bool same) {
        gt += more;
        eq += same;
    });
    // both counts in one word: a workgroup has fewer than 65536 keys where they are in registers; else two sums
    const auto sum_before = [&](int v) {
        int x = v;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(x, o, 64);
            if (lane >= o) x += y;
        }
        __syncthreads();
        if (lane == 63) part[w] = x;
        __syncthreads();
        for (int i = 0; i < w; ++i) x += part[i];
        return x - v;
    };
    int at, eq_at;
    if (KPT) {
        const int both = sum_before(gt | eq << 16);
        at = both & 0xffff;
        eq_at = (int)((uint32_t)both >> 16);
    } else {
        at = sum_before(gt);
        eq_at = sum_before(eq);
    }
    at += min(eq_at, left);
    mine([&](int i, bool more, bool same) {
        if (more || (same && eq_at < left)) out[at++] = i;
        eq_at += same;
    });
}

// What needs no choice: the length of the list, its end, and a list of all blocks.  True: done.
template <int THREADS>
__device__ __forceinline__ bool all_taken(const SelectArgs &a, int pair, int s, int Hkv, int nb, int32_t *out) {
    const int k = min(a.top_k, nb);
    if (threadIdx.x == 0 && pair == s * Hkv) a.counts[s] = k;
    for (int i = k + threadIdx.x; i < a.top_k; i += THREADS) out[i] = -1;
    if (nb > a.top_k) return false;
    for (int i = threadIdx.x; i < nb; i += THREADS) out[i] = i;
    return true;
}

template <int THREADS, int KPT>
__global__ void __launch_bounds__(THREADS) k_pick(SelectArgs a, int Hkv, int Bk) {
    const int pair = blockIdx.x, s = pair / Hkv, nb = n_blocks_of(a, s, Bk);
    int32_t *out = a.blocks + (size_t)pair * a.top_k;
    if (all_taken<THREADS>(a, pair, s, Hkv, nb, out)) return;
    pick<THREADS, KPT>(a, nb, (const uint32_t *)a.scores + (size_t)pair * key_pitch(a.max_blocks), out);
}

// Both at once where a sequence has few blocks, head sizes 64 and 128: a workgroup to a sequence and kv-head, keys in LDS.  Replayed from a graph, 8 heads of 128, up to
// 9 rows x 4 heads: 1 sequence of 125 blocks 7.3 us, of 250 8.0 (two kernels 8.1 and 8.4), 64 of 250 12.7 (15.9), 64 of 506 17.9 (21.8); but 1 of 506 11.3 (9.2), one
// workgroup's reads of all its codes, and 64 of 1012 26.4 (25.4).
constexpr int kOnceThreads = 512, kOnceBlocks = 512, kOnceTiles = 5;
template <typename T, int KS>
__global__ void __launch_bounds__(kOnceThreads) k_select(SelectArgs a, int Hq, int Hkv, int Bk) {
    constexpr int TB = 2, STEP = kOnceThreads / 64 * 16 * TB;
    __shared__ i32x4 rows[kOnceTiles][KS][64];
    __shared__ __attribute__((aligned(16))) float steps[kOnceTiles][16];
    __shared__ __attribute__((aligned(16))) uint32_t keys[kOnceBlocks];
    const int pair = blockIdx.x, s = pair / Hkv, c = pair - s * Hkv, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int nb = n_blocks_of(a, s, Bk);
    int32_t *out = a.blocks + (size_t)pair * a.top_k;
    if (all_taken<kOnceThreads>(a, pair, s, Hkv, nb, out)) return;
    const Stack<T> x(a, s, c, Hq, Hkv);
    for (int j0 = 0; j0 == 0 || j0 < x.n; j0 += 16 * kOnceTiles) {  // without queries once too: the keys say which blocks there are
        const int tiles = max(0, min(kOnceTiles, (x.n - j0 + 15) / 16));
        int b0 = w * 16 * TB;
        Codes<KS, TB> codes;
        codes.load(a, s, c, Hkv, b0, nb, lane);
        if (j0) __syncthreads();
        for (int t = w; t < tiles; t += kOnceThreads / 64) quantise_tile<T, KS>(x, j0 + 16 * t, rows[t], steps[t], lane);
        __syncthreads();
        for (; b0 < nb - a.last; b0 += STEP) {
            float best[TB];
#pragma unroll
            for (int t = 0; t < TB; ++t) best[t] = -INFINITY;
            for (int j = 0; j < tiles; ++j) codes.score(best, rows[j], steps[j], lane);
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const uint32_t key = codes.key(t, best[t], x.n);
                const int b = b0 + 16 * t + lane;
                if (lane < 16 && b < nb) keys[b] = j0 ? max(keys[b], key) : key;
            }
            if (b0 + STEP < nb - a.last) codes.load(a, s, c, Hkv, b0 + STEP, nb, lane);
        }
    }
    __syncthreads();
    pick<kOnceThreads, 4>(a, nb, keys, out);
}

}  // namespace

hipError_t launch_extend(const ExtendArgs &a, hipStream_t st) {
    const int wgs = a.max_rows > kExtThreads ? (a.max_rows + kExtThreads - 1) / kExtThreads : 1;  // a row to a thread
    hipLaunchKernelGGL(k_extend, dim3(wgs), dim3(kExtThreads), 0, st, a);
    return hipGetLastError();
}

template <typename T, typename KT>
static bool append_window(const Dims &dm, const AppendArgs &a, int rows, hipStream_t st) {
    if (dm.Bk != 16 || a.ld * (int64_t)sizeof(T) % 16) return false;
    const int windows = (rows + kWindow - 1) / kWindow;
    // Of the heads: four workgroups to a CU, as long as a part has a rotated head for every wave's turn.  5300 rows of 80 heads 54 us (1 to a CU 68, 16 to a CU 58),
    // 1145 rows 15.4 (1 to a CU 19.7), 16384 rows of 48 heads 92 (16 to a CU 98).
    int parts = 1;
    while (windows * parts < 1024 && 2 * parts <= (dm.Hq + dm.Hkv + 3) / 4) parts *= 2;
    const dim3 grid(windows, parts + std::min(parts, dm.Hkv));
    const double l2t = log2(dm.theta);
    switch (dm.D) {
    case 64: hipLaunchKernelGGL((k_append_window<T, KT, 64>), grid, dim3(256), 0, st, a, dm.Hq, dm.Hkv, parts, l2t, dm.eps, dm.qk_norm, dm.k_scale, dm.v_scale); return true;
    case 128: hipLaunchKernelGGL((k_append_window<T, KT, 128>), grid, dim3(256), 0, st, a, dm.Hq, dm.Hkv, parts, l2t, dm.eps, dm.qk_norm, dm.k_scale, dm.v_scale); return true;
    case 256:
        if constexpr (sizeof(T) == 2) {  // four tiles of float32 pass what static LDS holds
            hipLaunchKernelGGL((k_append_window<T, KT, 256>), grid, dim3(256), 0, st, a, dm.Hq, dm.Hkv, parts, l2t, dm.eps, dm.qk_norm, dm.k_scale, dm.v_scale);
            return true;
        }
        return false;
    default: return false;
    }
}

hipError_t launch_append(const Dims &dm, bool generic, AppendArgs a, hipStream_t st) {
    constexpr int kRows = 1 << 23;  // of a launch, whole windows: its work items in one direction have to be fewer than 2^32
    for (a.first = 0; a.first < a.R; a.first += kRows) {
        const int rows = std::min(kRows, a.R - a.first);
        bool done = false;
        if (!generic) DISPATCH_TK(dm.bf16, dm.kv8, done = (append_window<T, KT>(dm, a, rows, st)));
        if (!done)
            DISPATCH_TK(dm.bf16, dm.kv8, hipLaunchKernelGGL((k_append<T, KT>), dim3(rows, (dm.Hq + 2 * dm.Hkv + 3) / 4), dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.D,
                                                            dm.Bk, log2(dm.theta), dm.eps, dm.qk_norm, dm.k_scale, dm.v_scale));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

constexpr int kBoundsWgs = 4096;
template <typename KT>
static bool bounds_wave(const Dims &dm, const BoundsArgs &a, dim3 grid, hipStream_t st) {
    if (dm.Bk != 16) return false;
    switch (dm.D) {
    case 64: hipLaunchKernelGGL((k_bounds_wave<KT, 64>), grid, dim3(256), 0, st, a, dm.Hkv); return true;
    case 128: hipLaunchKernelGGL((k_bounds_wave<KT, 128>), grid, dim3(256), 0, st, a, dm.Hkv); return true;
    case 256: hipLaunchKernelGGL((k_bounds_wave<KT, 256>), grid, dim3(256), 0, st, a, dm.Hkv); return true;
    default: return false;
    }
}

hipError_t launch_bounds(const Dims &dm, bool generic, const BoundsArgs &a, hipStream_t st) {
    const int64_t most = a.max_new > 0 ? std::min<int64_t>(a.max_blocks, (a.max_new - 1) / dm.Bk + 2) : a.max_blocks;  // blocks of a sequence, about
    // workgroups to a sequence: a block to each, until there are 16 to a CU; what is left goes round (4 to a CU: 124 us for the above, 32: 119)
    const int per_seq = (int)std::min<int64_t>(most, std::max<int64_t>(1, (kBoundsWgs + a.S - 1) / a.S));
    bool done = false;
    if (!generic) DISPATCH_TK(dm.bf16, dm.kv8, { (void)sizeof(T); done = bounds_wave<KT>(dm, a, dim3(a.S, per_seq), st); });
    if (!done)
        DISPATCH_TK(dm.bf16, dm.kv8, {
            (void)sizeof(T);
            hipLaunchKernelGGL(k_bounds<KT>, dim3(a.S, per_seq, (dm.Hkv + 3) / 4), dim3(256), 0, st, a, dm.Hkv, dm.D, dm.Bk);
        });
    return hipGetLastError();
}

template <typename T, int TB>
static bool scores_mfma(const Dims &dm, const SelectArgs &a, hipStream_t st) {
    const dim3 grid(a.S * dm.Hkv, (a.max_blocks + 64 * TB - 1) / (64 * TB));
    switch (dm.D) {
    case 64: hipLaunchKernelGGL((k_scores_mfma<T, 2, TB>), grid, dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.Bk); return true;
    case 128: hipLaunchKernelGGL((k_scores_mfma<T, 4, TB>), grid, dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.Bk); return true;
    case 192: hipLaunchKernelGGL((k_scores_mfma<T, 6, TB>), grid, dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.Bk); return true;
    case 256: hipLaunchKernelGGL((k_scores_mfma<T, 8, TB>), grid, dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.Bk); return true;
    default: return false;
    }
}

template <typename T>
static bool select_at_once(const Dims &dm, const SelectArgs &a, hipStream_t st) {
    const dim3 grid(a.S * dm.Hkv), threads(kOnceThreads);
    switch (dm.D) {
    case 64: hipLaunchKernelGGL((k_select<T, 2>), grid, threads, 0, st, a, dm.Hq, dm.Hkv, dm.Bk); return true;
    case 128: hipLaunchKernelGGL((k_select<T, 4>), grid, threads, 0, st, a, dm.Hq, dm.Hkv, dm.Bk); return true;
    default: return false;
    }
}

hipError_t launch_select(const Dims &dm, bool generic, const SelectArgs &a, hipStream_t st) {
    bool done = false;
    const int64_t pairs = (int64_t)a.S * dm.Hkv;
    if (!generic && a.max_blocks <= (pairs < 128 ? kOnceBlocks / 2 : kOnceBlocks)) {  // few lists: two kernels spread the codes of each over the chip
        DISPATCH_T(dm.bf16, done = (select_at_once<T>(dm, a, st)));
        if (done) return hipGetLastError();
    }
    if (a.max_blocks > a.top_k) {  // else all blocks are taken
        // 128 blocks to a workgroup share its queries, 64 fill the chip sooner: 1 sequence, 8 kv-heads, 2048 blocks 6.6 and 5.7 us; 64 sequences 18.6 and 20.7
        const bool few = pairs * ((a.max_blocks + 127) / 128) <= 256;
        if (!generic) DISPATCH_T(dm.bf16, done = (few ? scores_mfma<T, 1>(dm, a, st) : scores_mfma<T, 2>(dm, a, st)));
        if (!done)
            DISPATCH_T(dm.bf16, hipLaunchKernelGGL(k_scores<T>, dim3(a.S * dm.Hkv, (a.max_blocks + 255) / 256), dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.D, dm.Bk));
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 grid(a.S * dm.Hkv);
    // The fewest threads that hold the keys of the widest list: 512 lists of up to 1024 blocks 6.3 us (512 threads 7.1, 1024 10.4); 8 of 2048 5.9 us (256 threads with
    // 8 keys 7.9, 1024 7.7); 32 of 7500 8.7 us (keys read again 16); 8 of 31250 23 us (keys read again 43).
    if (a.max_blocks <= 1024) hipLaunchKernelGGL((k_pick<256, 4>), grid, dim3(256), 0, st, a, dm.Hkv, dm.Bk);
    else if (a.max_blocks <= 2048) hipLaunchKernelGGL((k_pick<512, 4>), grid, dim3(512), 0, st, a, dm.Hkv, dm.Bk);
    else if (a.max_blocks <= 8192) hipLaunchKernelGGL((k_pick<1024, 8>), grid, dim3(1024), 0, st, a, dm.Hkv, dm.Bk);
    else if (a.max_blocks <= 32768) hipLaunchKernelGGL((k_pick<1024, 32>), grid, dim3(1024), 0, st, a, dm.Hkv, dm.Bk);
    else hipLaunchKernelGGL((k_pick<1024, 0>), grid, dim3(1024), 0, st, a, dm.Hkv, dm.Bk);
    return hipGetLastError();
}

}  // namespace icarus
