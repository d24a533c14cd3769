// Sequences that branch: choice of a group's best continuations, tables of the children, copies of blocks, and attention for any shape.  Everything a
// kernel indexes with -- parents, lengths, block ids, rows -- comes from device memory and is checked where it is used.
#include "block_util.h"
#include "branch_ops.h"

#include <algorithm>

namespace icarus {
namespace {

// ---- choice of the continuations ------------------------------------------------------------------------------------------
// Two launches.  k_beam_part reads a part of a beam's logits once: its largest logit, its sum of exponentials and its `width` largest logits, of which no other of the
// part's can be among the group's best.  k_beam_merge puts the parts of a group together.
//
// Sums and scores are float64: two beams' candidates are told apart by the difference of their normalisers, and with sums in float32 the order of a group would
// depend on how the row was split.  A logit and a number below it as the order of the logits, equal ones by the lowest token: packed in 64 bits.
constexpr int kBeamThreads = 256, kBeamList = 1024;

__device__ __forceinline__ uint32_t order_key(float x) {  // larger numbers have larger keys
    const uint32_t u = __float_as_uint(x);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
// A logit as it counts: NaN as minus infinity, plus infinity as the largest finite number.  The median of three, which is their minimum where one is NaN; by hand, since the compiler takes
// it for a minimum of the outer two.  A signalling NaN is made a quiet one first: the minimum of it and minus infinity would be a quiet NaN, and the next minimum the largest number.
__device__ __forceinline__ float clean_logit(float x) {
    float r;
    asm("v_med3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(__builtin_canonicalizef(x)), "v"(-INFINITY), "v"(3.402823466e38f));
    return r;
}
__device__ __forceinline__ float max_of_3(float a, float b, float c) {  // by hand: for fmaxf the compiler first turns what clean_logit gives into itself
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// exp(d) for d <= 0, to 2^-39 of itself; below -700, minus infinity included, 2^-1010, which no sum of ours notices: exp(d) = 2^n exp(r), |r| <= ln 2 / 2, the polynomial that meets exp at the nine Chebyshev nodes of that interval.
__device__ __forceinline__ double exp_of(double d) {
    d = fmax(d, -700.0);
    const double n = rint(d * 1.4426950408889634074), r = __builtin_fma(n, -0.69314718055994530942, d);
    double p = 2.4876164180131435e-05;
    p = __builtin_fma(p, r, 0.00019915867076303128);
    p = __builtin_fma(p, r, 0.0013888821677344278);
    p = __builtin_fma(p, r, 0.008333266097680215);
    p = __builtin_fma(p, r, 0.04166666689095846);
    p = __builtin_fma(p, r, 0.16666666891047124);
    p = __builtin_fma(p, r, 0.49999999999797934);
    p = __builtin_fma(p, r, 0.9999999999797851);
    p = __builtin_fma(p, r, 1.0);
    return __builtin_ldexp(p, (int)n);
}
__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ double wave_max_f64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o, 64));
    return v;
}

// A number that at least W of the wave's 64 reach, and not many more.  Up to 16: of sixteen runs of four lanes the largest each, and of those the least that fewer than W exceed; else of W runs
// (the next power of two) the least.  A part of 8192 logits lists 27 of them for 8 beams, by runs alone 53.
template <int CTRL>
__device__ __forceinline__ float lane_of(float x) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, true)); }
__device__ __forceinline__ float reached_by(float x, int W) {
    int run = W > 1 && W <= 16 ? 4 : 64;
    while (W > 16 && run > 1 && 64 / run < W) run >>= 1;
    const auto join = [&](float y, int size) { x = size <= run ? fmaxf(x, y) : fminf(x, y); };
    join(lane_of<0xb1>(x), 2);  // lane ^ 1
    join(lane_of<0x4e>(x), 4);  // lane ^ 2
    if (W > 1 && W <= 16) {
        int above = 0;
        const auto row = [&](float y) {  // the four runs of a row of 16 lanes, each turned past this one
            above += (y > x) + (lane_of<0x124>(y) > x) + (lane_of<0x128>(y) > x) + (lane_of<0x12c>(y) > x);
        };
        row(x);
        row(__shfl_xor(x, 16, 64));
        row(__shfl_xor(x, 32, 64));
        row(__shfl_xor(x, 48, 64));
        if (above >= W) x = INFINITY;
    }
    join(lane_of<0x141>(x), 8);   // of the other four of eight, all alike
    join(lane_of<0x140>(x), 16);  // of the other eight of sixteen
    join(__shfl_xor(x, 16, 64), 32);
    join(__shfl_xor(x, 32, 64), 64);
    return x;
}

// Row of logits that a beam takes, -1: none.
__device__ __forceinline__ int beam_row(const BeamArgs &a, int s) {
    int row = s;
    if (a.row_start) {
        const int end = a.row_start[s + 1];
        row = end > a.row_start[s] ? end - 1 : -1;
    }
    return row >= 0 && row < a.R ? row : -1;
}

struct BeamParts {
    double2 *sums;   // [G * W][parts]: largest logit, sum of exp(x - largest)
    uint64_t *best;  // [G * W][parts][W]: key << 32 | ~token, descending; 0: none
    int parts;
};

// A workgroup loads its part, then adds up exponentials, then ranks, and with few rounds of workgroups these phases do not hide one another: 460 rows of 128256 float32 logits (236 MB) take 66 us,
// nearer the sum than the larger one of the read (without the exponentials 40 us, 5.9 TB/s) and the arithmetic (17 instructions of float64 to a logit, 26 us at the full rate, and seven others);
// without the candidates 53.  Instructions alone are not what bounds it: three of the 17 less changed nothing.  More waves to a SIMD spill or wait (66 -> 76).  120 rows of 50021 bfloat16 logits (12 MB)
// take 13.6 us in one round of 840 workgroups: the chain of one of them.
template <typename T, int PER>  // logits of a thread
__global__ void __launch_bounds__(kBeamThreads) k_beam_part(BeamArgs a, BeamParts out) {
    constexpr int VE = 16 / sizeof(T), NV = PER / VE;
    constexpr int SEG = kBeamList / 4;  // a list to a wave
    __shared__ uint64_t list[kBeamList];
    __shared__ float wmax[4], wbound[4];
    __shared__ double wsum[4];
    __shared__ int listed[4];
    const int s = blockIdx.y, part = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6;
    const int row = beam_row(a, s);
    if (row < 0 || (a.done && a.done[s])) return;
    // Which thread takes a logit goes by the token alone: equal rows have equal sums wherever they begin, and their beams tie.
    const T *x0 = (const T *)a.logits + (size_t)row * a.ld;
    struct __attribute__((packed, aligned(sizeof(T)))) Vec { uint32_t u[4]; };  // rows begin at any element
    const int first = part * NV * kBeamThreads;
    float x[PER];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int e = (first + j * kBeamThreads + t) * VE;
        if (e + VE <= a.vocab) {
            const Vec r = *(const Vec *)(x0 + e);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (sizeof(T) == 4) {
                    x[j * VE + k] = __uint_as_float(r.u[k]);
                } else {
                    x[j * VE + 2 * k] = __uint_as_float(r.u[k] << 16);
                    x[j * VE + 2 * k + 1] = __uint_as_float(r.u[k] & 0xffff0000u);
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < VE; ++k) x[j * VE + k] = e + k < a.vocab ? Elem<T>::ld(x0 + e + k) : -INFINITY;
        }
    }
    const auto token_of = [&](int i) { return (first + i / VE * kBeamThreads + t) * VE + i % VE; };
    float mine = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = clean_logit(x[i]);
#pragma unroll
    for (int i = 0; i < PER; i += 2) mine = max_of_3(mine, x[i], x[i + 1]);
    const float wave_most = reached_by(mine, 1), bound_w = reached_by(mine, a.W);
    if (lane == 0) {
        wmax[w] = wave_most;
        wbound[w] = bound_w;
    }
    __syncthreads();
    const float most = fmaxf(fmaxf(wmax[0], wmax[1]), fmaxf(wmax[2], wmax[3]));
    const float least = fmaxf(fmaxf(fmaxf(wbound[0], wbound[1]), fmaxf(wbound[2], wbound[3])), -3.402823466e38f);  // at least W logits reach it, or all that count
    uint64_t *best = out.best + ((size_t)s * out.parts + part) * a.W;
    if (most == -INFINITY) {
        if (t < a.W) best[t] = 0;
        if (t == 0) out.sums[(size_t)s * out.parts + part] = make_double2(-INFINITY, 0.0);
        return;
    }
    double sum = 0.0, sum1 = 0.0;
    const double most_d = most;
#pragma unroll
    for (int i = 0; i < PER; i += 2) {
        sum += exp_of((double)x[i] - most_d);
        sum1 += exp_of((double)x[i + 1] - most_d);
    }
    sum = wave_sum_f64(sum + sum1);
    int n = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const unsigned long long mask = __ballot(x[i] >= least);
        if (mask) {  // few
            const int at = n + __popcll(mask & ((1ull << lane) - 1));
            if ((mask >> lane & 1) && at < SEG) list[w * SEG + at] = (uint64_t)order_key(x[i] + 0.f) << 32 | ~(uint32_t)token_of(i);  // -0 equals 0
            n += __popcll(mask);
        }
    }
    if (lane == 0) {
        wsum[w] = sum;
        listed[w] = n;
    }
    __syncthreads();
    if (t == 0) out.sums[(size_t)s * out.parts + part] = make_double2((double)most, (wsum[0] + wsum[1]) + (wsum[2] + wsum[3]));
    const int n0 = listed[0], n1 = listed[1], n2 = listed[2], n3 = listed[3], all = n0 + n1 + n2 + n3;
    if (max(max(n0, n1), max(n2, n3)) <= SEG) {  // the place of each in the order: how many are larger; several lanes to one, each of which looks at a share of the lists
        int lanes = 64;
        while (lanes > 1 && lanes * n > 64) lanes >>= 1;
        const int share = lane & (lanes - 1);
        for (int i = lane / lanes; i < n; i += 64 / lanes) {
            const uint64_t v = list[w * SEG + i];
            int rank = 0;
            for (int k = 0; k < 4; ++k)
                for (int j = share; j < listed[k]; j += lanes) rank += list[k * SEG + j] > v;
            for (int o = 1; o < lanes; o <<= 1) rank += __shfl_xor(rank, o, 64);
            if (share == 0 && rank < a.W) best[rank] = v;
        }
        if (t >= all && t < a.W) best[t] = 0;
        return;
    }
    __syncthreads();
    // Many equal logits: one after the other.
    uint64_t last = ~0ull;
    for (int k = 0; k < a.W; ++k) {
        uint64_t v = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint64_t c = (uint64_t)order_key(x[i] + 0.f) << 32 | ~(uint32_t)token_of(i);
            if (x[i] > -INFINITY && c < last && c > v) v = c;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const uint64_t y = __shfl_xor(v, o, 64);
            v = y > v ? y : v;
        }
        __syncthreads();
        if (lane == 0) list[w] = v;
        __syncthreads();
        v = list[0];
        for (int i = 1; i < 4; ++i) v = list[i] > v ? list[i] : v;
        last = v;
        if (t == 0) best[k] = v;
    }
}

// A candidate and its place: larger scores first, then the lowest beam, then the larger logit, then the lowest token.
struct Candidate {
    double score;
    uint64_t what;  // as BeamParts::best; done: the end token's
    int beam;
    __device__ __forceinline__ bool before(const Candidate &o) const {
        if (score != o.score) return score > o.score;
        if (beam != o.beam) return beam < o.beam;
        return what > o.what;
    }
};

// A workgroup to a group; the candidates that fit stay in registers, on their way before the normalisers are summed: what the kernel waits for is its chain of reads and sums (64 groups of 8
// beams with 16 parts 7.4 us, one group of 4 beams with 63 parts 5.8 us).
constexpr int kMergeThreads = 512, kMergeWaves = kMergeThreads / 64, kMergeHeld = 4;
__global__ void __launch_bounds__(kMergeThreads) k_beam_merge(BeamArgs a, BeamParts in) {
    __shared__ double add[kBeamMost], top[kBeamMost];  // a logit x of the beam scores (x - top) + add: large logits cancel before the rest is added
    __shared__ int kind[kBeamMost];                    // 0: no continuations, 1: live, 2: done
    __shared__ Candidate list[kBeamList];
    __shared__ int rank[kBeamList];
    __shared__ float wbound[kMergeWaves];
    __shared__ int count;
    const int g = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6, W = a.W;
    const int per_beam = in.parts * W, n_all = W * per_beam;
    const uint64_t *best = in.best + (size_t)g * n_all;
    uint64_t held[kMergeHeld];
#pragma unroll
    for (int k = 0; k < kMergeHeld; ++k) held[k] = best[min(t + k * kMergeThreads, n_all - 1)];
    for (int b = w; b < W; b += kMergeWaves) {
        const int s = g * W + b;
        const float score = a.scores[s];
        const int done = a.done ? a.done[s] : 0;
        const double2 first = in.sums[(size_t)s * in.parts + min(lane, in.parts - 1)];  // of a beam that is not live: anything
        int k = score - score != 0.f ? 0 : done ? 2 : beam_row(a, s) >= 0 ? 1 : 0;  // a finished beam needs no row
        double most = -INFINITY, sum = 0.0;
        if (k == 1) {
            most = lane < in.parts ? first.x : -INFINITY;
            for (int p = lane + 64; p < in.parts; p += 64) most = fmax(most, in.sums[(size_t)s * in.parts + p].x);
            most = wave_max_f64(most);
            if (lane < in.parts && first.y > 0.0) sum = first.y * exp_of(first.x - most);
            for (int p = lane + 64; p < in.parts; p += 64) {
                const double2 v = in.sums[(size_t)s * in.parts + p];
                if (v.y > 0.0) sum += v.y * exp_of(v.x - most);
            }
            sum = wave_sum_f64(sum);
            if (most == -INFINITY) k = 0;
        }
        if (lane == 0) {
            kind[b] = k;
            add[b] = k == 1 ? (double)score - log(sum) : (double)score;
            top[b] = most;
        }
    }
    if (t == 0) count = 0;
    for (int i = t; i < kBeamList; i += kMergeThreads) rank[i] = 0;
    __syncthreads();
    const auto make = [&](int i, uint64_t what, Candidate &c) {
        c.beam = i / per_beam;
        const int k = kind[c.beam];
        if (k == 0 || (k == 2 && i != c.beam * per_beam)) return false;
        if (k == 2) {
            c.what = (uint64_t)0x80000000u << 32 | ~(uint32_t)a.eos;
            c.score = add[c.beam];
            return true;
        }
        c.what = what;
        c.score = ((double)of_key((uint32_t)(what >> 32)) - top[c.beam]) + add[c.beam];
        return what != 0;
    };
    const auto below = [](double v) {  // a float that is not above v
        const float f = (float)v;
        return (double)f > v ? nextafterf(f, -INFINITY) : f;
    };
    const auto each = [&](auto &&f) {  // all candidates of this thread
        Candidate c;
#pragma unroll
        for (int k = 0; k < kMergeHeld; ++k)
            if (t + k * kMergeThreads < n_all && make(t + k * kMergeThreads, held[k], c)) f(c);
        for (int i = t + kMergeHeld * kMergeThreads; i < n_all; i += kMergeThreads)
            if (make(i, best[i], c)) f(c);
    };
    float mine = -INFINITY;
    each([&](const Candidate &c) { mine = fmaxf(mine, below(c.score)); });
    const float bound_w = reached_by(mine, W);
    if (lane == 0) wbound[w] = bound_w;
    __syncthreads();
    float bound = wbound[0];
#pragma unroll
    for (int k = 1; k < kMergeWaves; ++k) bound = fmaxf(bound, wbound[k]);
    each([&](const Candidate &c) {
        if (below(c.score) < bound) return;
        const int at = atomicAdd(&count, 1);
        if (at < kBeamList) list[at] = c;
    });
    __syncthreads();
    const int n = count;
    const auto put = [&](int place, const Candidate &v) {
        const int s = g * W + place, token = (int)~(uint32_t)v.what;
        a.parents[s] = v.beam;
        a.tokens[s] = token;
        a.scores_out[s] = (float)v.score;
        if (a.done_out) a.done_out[s] = kind[v.beam] == 2 || token == a.eos;
    };
    const auto none = [&](int place) {
        const int s = g * W + place;
        a.parents[s] = -1;
        a.tokens[s] = -1;
        a.scores_out[s] = -INFINITY;
        if (a.done_out) a.done_out[s] = 0;
    };
    if (n <= kBeamList) {  // the place of each: how many are better; each wave counts among its share
        for (int i = lane; i < n; i += 64) {
            const Candidate v = list[i];
            int better = 0;
            for (int j = w; j < n; j += kMergeWaves) better += list[j].before(v);
            if (better) atomicAdd(&rank[i], better);
        }
        __syncthreads();
        for (int i = t; i < n; i += kMergeThreads)
            if (rank[i] < W) put(rank[i], list[i]);
        if (t >= n && t < W) none(t);
        return;
    }
    Candidate last{INFINITY, ~0ull, -1};
    for (int k = 0; k < W; ++k) {
        Candidate v{-INFINITY, 0, kBeamMost};
        each([&](const Candidate &c) {
            if (last.before(c) && c.before(v)) v = c;
        });
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            Candidate y;
            y.score = __shfl_xor(v.score, o, 64);
            y.what = __shfl_xor(v.what, o, 64);
            y.beam = __shfl_xor(v.beam, o, 64);
            if (y.before(v)) v = y;
        }
        __syncthreads();
        if (lane == 0) list[w] = v;
        __syncthreads();
        for (int i = 0; i < kMergeWaves; ++i)
            if (list[i].before(v)) v = list[i];
        last = v;
        if (t == 0) {
            if (v.beam < kBeamMost) put(k, v);
            else none(k);
        }
    }
}

// Parts of 8192 logits, of 2048 where those would be fewer than 128 workgroups.  Rows of 128256, us of both kernels with small and large parts: 4 rows 10.5, 11.1; 16 rows 20.1, 14.0; 32 rows
// 25.5, 16.2 -- the merge reads what the parts leave.  Parts of 4096: 460 rows 76.8 + 10.9 for 66.3 + 7.7.  All float32; bfloat16 and other vocabularies were not timed for this choice.
constexpr int kBeamFew = 8, kBeamMany = 32;
int beam_parts(int vocab, int per) { return (int)(((int64_t)vocab + kBeamThreads * per - 1) / (kBeamThreads * per)); }
int beam_per(int G, int W, int vocab) { return (int64_t)G * W * beam_parts(vocab, kBeamMany) >= 128 ? kBeamMany : kBeamFew; }

// ---- children ------------------------------------------------------------------------------------------------------------------
// Bound by their chains, not by their bytes: lengths and parents, the column's ids, what the parts have freed; then the ids of the fresh blocks (one group of 8 beams, 2048 columns, 4.6 + 6.1 us;
// 64 groups, 1000 columns, 5.1 + 8.8 us).  Over 16 beams by the comparisons of a column's thread, on few CUs (a group of 24, 4096 columns, 32 workgroups, 14.4 + 13.8 us; of 64 50.9 + 27.1).
// Every workgroup of the second launch adds up the counts of all parts, which counts from thousands of parts on: 31264 of them (32 groups of 2, 125000 columns) 28 + 1295 us.  Two launches over parts of 128 columns of a group's tables, a thread to a column.  k_fork_count finds the blocks that no child holds: in a column, of the old sequences that nobody
// continues, the ids that none of the continued ones names.  k_fork_write adds up the parts before its own, enters the freed ids, and writes the children's tables.
struct ForkParts {
    int32_t *freed_n;  // [G * parts]
    int32_t *fresh_n;  // [G]
    int32_t *freed;    // [G * parts][W * kForkCols]: ids by column and sequence
    int parts;
};

struct ForkGroup {  // in LDS: a group's sequences
    int len[kBeamMost], nb[kBeamMost], parent[kBeamMost], fresh[kBeamMost];  // old length and blocks; of a child: its parent, 1 where it needs a block
    uint64_t kept;                                                             // parents
    int shared, n_fresh;
};

// The old ids of this thread's column, of all sequences as they stand: read whether they are in use or not, so that they are on their way beside the lengths.  M sequences at most are held
// in registers, any number in LDS (M = 0).  Up to 16 are compared there (64 groups of 8 sequences, 1000 columns: the count takes 5 us, one by one from LDS 9.8), more in eights from LDS (a group of
// 24, 4096 columns: 14 us, one by one 33).
template <int M>
struct ForkColumn {
    int32_t v[M ? M : 1];
    __device__ __forceinline__ void load(const ForkArgs &a, int g, int c, int32_t *tile) {
        const int32_t *from = a.bt + (size_t)g * a.W * a.max_blocks + c;
        if constexpr (M > 0) {
#pragma unroll
            for (int i = 0; i < M; ++i) v[i] = -1;
            if (c >= a.max_blocks) return;
#pragma unroll
            for (int i = 0; i < M; ++i)
                if (i < a.W) v[i] = from[(size_t)i * a.max_blocks];
            return;
        }
        if (c >= a.max_blocks) return;
        int i = 0;
        for (; i + 16 <= a.W; i += 16) {
            int32_t x[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) x[k] = from[(size_t)(i + k) * a.max_blocks];
#pragma unroll
            for (int k = 0; k < 16; ++k) tile[(i + k) * kForkCols + threadIdx.x] = x[k];
        }
        for (; i < a.W; ++i) tile[i * kForkCols + threadIdx.x] = from[(size_t)i * a.max_blocks];
    }
    __device__ __forceinline__ void to_tile(const ForkArgs &a, int32_t *tile) const {
        if constexpr (M > 0) {
#pragma unroll
            for (int i = 0; i < M; ++i)
                if (i < a.W) tile[i * kForkCols + threadIdx.x] = v[i];
        }
    }
    // Which are freed: no sequence with children has the block in this column, and no earlier one of those without.
    __device__ __forceinline__ uint64_t freed(const ForkArgs &a, int c, const ForkGroup &f, int32_t *tile) const {
        const auto block = [&](int i, int32_t id) { return c < f.nb[i] && id >= 0 && id < a.num_blocks ? id : -1; };  // -1: none
        const uint64_t kept = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(f.kept >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)f.kept);
        uint64_t out = 0;
        if constexpr (M > 0 && M <= 16) {
            int32_t u[M];
#pragma unroll
            for (int i = 0; i < M; ++i) u[i] = i < a.W ? block(i, v[i]) : -1;
#pragma unroll
            for (int i = 0; i < M; ++i) {
                if (i >= a.W || kept >> i & 1) continue;
                bool held = u[i] < 0;
#pragma unroll
                for (int j = 0; j < M; ++j)
                    if (j < i || (j > i && kept >> j & 1)) held |= u[j] == u[i];
                if (!held) out |= 1ull << i;
            }
            return c < f.shared ? 0 : out;
        }
        // Eight sequences at a time against all others, eight of those at a time: each is read once for the eight.
        int32_t *const mine = tile + threadIdx.x;
        if constexpr (M > 0) {
#pragma unroll
            for (int i = 0; i < M; ++i)
                if (i < a.W) mine[i * kForkCols] = block(i, v[i]);
        } else {
#pragma unroll 8
            for (int i = 0; i < a.W; ++i) mine[i * kForkCols] = block(i, mine[i * kForkCols]);
        }
        const auto eight = [&](int32_t (&x)[8], int i0) {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = mine[min(i0 + k, a.W - 1) * kForkCols];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = i0 + k < a.W ? x[k] : -1;
        };
        for (int i0 = 0; i0 < a.W; i0 += 8) {
            if ((kept >> i0 & 255) == 255) continue;
            int32_t u[8];
            bool held[8];
            eight(u, i0);
#pragma unroll
            for (int k = 0; k < 8; ++k) held[k] = u[k] < 0 || (kept >> (i0 + k) & 1);
            const auto against = [&](int32_t x, int from) {  // the sequences from i0 + from on
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k >= from) held[k] |= x == u[k];
            };
            int32_t x[8];
            for (int j0 = 0; j0 < i0; j0 += 8) {
                eight(x, j0);
#pragma unroll
                for (int j = 0; j < 8; ++j) against(x[j], 0);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (kept >> (i0 + j) & 1) against(u[j], 0);  // itself too: it is not freed in any case
                else against(u[j], j + 1);
            }
            for (int j0 = i0 + 8; j0 < a.W; j0 += 8) {
                if ((kept >> j0 & 255) == 0) continue;
                eight(x, j0);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (kept >> (j0 + j) & 1) against(x[j], 0);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (!held[k]) out |= 1ull << (i0 + k);
        }
        return c < f.shared ? 0 : out;
    }
};

struct ForkSequence { int len, parent, shared; };  // what the arrays hold for this thread's
__device__ __forceinline__ ForkSequence fork_sequence(const ForkArgs &a, int g) {
    const int i = threadIdx.x;
    return i < a.W ? ForkSequence{a.kv_lens[g * a.W + i], a.parents[g * a.W + i], a.shared ? a.shared[g] : 0} : ForkSequence{0, -1, 0};
}

__device__ __forceinline__ void fork_group(const ForkArgs &a, const ForkSequence &mine, ForkGroup &f) {  // by the first wave; a barrier follows
    const int i = threadIdx.x;
    if (i >= 64) return;
    const int64_t room = (int64_t)a.max_blocks * a.Bk;
    const int n = (int)min((int64_t)max(mine.len, 0), room), parent = mine.parent >= 0 && mine.parent < a.W ? mine.parent : -1, shared = __builtin_amdgcn_readfirstlane(max(mine.shared, 0));
    f.len[i] = n;
    f.nb[i] = n / a.Bk + (n % a.Bk != 0);
    f.parent[i] = parent;
    bool first = parent >= 0;
    uint64_t kept = 0;
    for (int j = 0; j < a.W; ++j) {
        const int q = __builtin_amdgcn_readlane(parent, j);
        if (j < i && q == parent) first = false;
        if (q >= 0) kept |= 1ull << q;
    }
    const int plen = __shfl(n, max(parent, 0), 64);
    const bool fresh = parent >= 0 && plen % a.Bk != 0 && (!first || plen / a.Bk < shared);
    f.fresh[i] = fresh;
    const int n_fresh = __popcll(__ballot(fresh));
    if (i == 0) {
        f.kept = kept;
        f.shared = shared;
        f.n_fresh = n_fresh;
    }
}

// Inclusive sum over the wave.
__device__ __forceinline__ int wave_scan(int x) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if ((int)(threadIdx.x & 63) >= o) x += y;
    }
    return x;
}
constexpr int kForkWaves = kForkCols / 64;

template <int M>
__global__ void __launch_bounds__(kForkCols) k_fork_count(ForkArgs a, ForkParts p) {
    extern __shared__ int32_t tile[];  // [W][kForkCols], more than 16
    __shared__ ForkGroup f;
    __shared__ int wsum[kForkWaves];
    const int g = blockIdx.y, part = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6, c = part * kForkCols + t;
    ForkColumn<M> col;
    const ForkSequence seq = fork_sequence(a, g);
    col.load(a, g, c, tile);
    fork_group(a, seq, f);
    __syncthreads();
    const uint64_t freed = col.freed(a, c, f, tile);
    const int n = __popcll(freed), x = wave_scan(n);
    if (lane == 63) wsum[w] = x;
    __syncthreads();
    int at = x - n, all = 0;
    for (int i = 0; i < kForkWaves; ++i) {
        if (i < w) at += wsum[i];
        all += wsum[i];
    }
    int32_t *out = p.freed + ((size_t)g * p.parts + part) * a.W * kForkCols;
    if constexpr (M > 0 && M <= 16) {
#pragma unroll
        for (int i = 0; i < M; ++i)
            if (freed >> i & 1) out[at++] = col.v[i];
    } else {
        for (uint64_t left = freed; left; left &= left - 1) out[at++] = tile[(__ffsll((unsigned long long)left) - 1) * kForkCols + t];
    }
    if (t == 0) {
        p.freed_n[(size_t)g * p.parts + part] = all;
        if (part == 0) p.fresh_n[g] = f.n_fresh;
    }
}

template <int M>
__global__ void __launch_bounds__(kForkCols) k_fork_write(ForkArgs a, ForkParts p) {
    extern __shared__ int32_t tile[];  // [W][kForkCols]
    __shared__ ForkGroup f;
    __shared__ int fresh_id[kBeamMost], fresh_at[kBeamMost], red[4][kForkWaves];
    __shared__ int64_t fresh_from[kBeamMost];  // where a child's id stands in the parts' lists
    const int g = blockIdx.y, part = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6, c = part * kForkCols + t;
    const int n_parts = a.G * p.parts, me = g * p.parts + part;
    // Every read that waits for no other comes first: the parts' lists and counts are another launch's, and each round of reads is a microsecond.
    const ForkSequence seq = fork_sequence(a, g);
    const int used = *a.free_used, n_mine = p.freed_n[me];
    const int32_t *mine = p.freed + (size_t)me * a.W * kForkCols;
    const int first_mine = mine[t];  // of no use from n_mine on
    int n_fresh = t < a.G ? p.fresh_n[t] : 0;
    ForkColumn<M> col;
    col.load(a, g, c, tile);
    // sums over the parts and groups before this one, and over all; a thread takes a run of parts
    constexpr int RUN = 8;
    int sum[4] = {0, 0, 0, 0}, n[RUN];
    const int run = (n_parts + kForkCols - 1) / kForkCols, run0 = min(t * run, n_parts), run1 = min(run0 + run, n_parts);
    for (int i0 = run0; i0 < run1; i0 += RUN) {
#pragma unroll
        for (int k = 0; k < RUN; ++k) n[k] = i0 + k < run1 ? p.freed_n[i0 + k] : 0;
#pragma unroll
        for (int k = 0; k < RUN; ++k) {
            sum[1] += n[k];
            if (i0 + k < me) sum[0] += n[k];
        }
    }
    for (int i = t; i < a.G; i += kForkCols) {
        if (i != t) n_fresh = p.fresh_n[i];
        sum[3] += n_fresh;
        if (i < g) sum[2] += n_fresh;
    }
    fork_group(a, seq, f);
    col.to_tile(a, tile);
    const int run_n = sum[1];
    int run_at = wave_scan(run_n) - run_n;  // freed ids before this thread's parts; the waves before are added below
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum[k] += __shfl_xor(sum[k], o, 64);
        if (lane == 0) red[k][w] = sum[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        sum[k] = red[k][0];
        for (int i = 1; i < kForkWaves; ++i) sum[k] += red[k][i];
    }
    for (int i = 0; i < w; ++i) run_at += red[1][i];
    const int before = sum[0], all = sum[1], fresh_before = sum[2], fresh_all = sum[3];
    const int head = min(max(used, 0), a.n_free), low = head - all, start = max(low, 0);  // freed id j stands at low + j
    for (int j = t; j < n_mine; j += kForkCols)
        if (low + before + j >= 0) a.free_ids[low + before + j] = j == t ? first_mine : mine[j];
    // Fresh ids of the group's children: entries start + fresh_before .. of the list.  Those before the head are freed ids of this call: from the parts' lists, since another workgroup
    // may not have entered them yet.
    if (t < 64) {
        const bool need = t < a.W && f.fresh[t];
        const int64_t at = (int64_t)start + fresh_before + __popcll(__ballot(need) & ((1ull << t) - 1));
        fresh_at[t] = need ? (at < a.n_free ? (int)at : -1) : -2;
        fresh_id[t] = -1;
        fresh_from[t] = -1;
    }
    __syncthreads();
    if (f.n_fresh) {
        const int want = start + fresh_before - low;  // the first of them among all freed ids
        if (run_n > 0 && run_at < want + f.n_fresh && run_at + run_n > want) {  // 0: the thread may have no parts, and n nothing
            const auto find = [&](int i, int count) {
                for (int j = 0; j < a.W && run_at < want + f.n_fresh && run_at + count > want; ++j) {
                    const int k = fresh_at[j] - low - run_at;
                    if (fresh_at[j] >= 0 && fresh_at[j] < head && k >= 0 && k < count) fresh_from[j] = (int64_t)i * a.W * kForkCols + k;
                }
                run_at += count;
            };
            if (run <= RUN) {
#pragma unroll
                for (int k = 0; k < RUN; ++k)
                    if (n[k]) find(run0 + k, n[k]);
            } else {
                for (int i = run0; i < run1; ++i) find(i, p.freed_n[i]);
            }
        }
        __syncthreads();
        if (t < a.W && fresh_at[t] >= head) fresh_id[t] = a.free_ids[fresh_at[t]];
        else if (t < a.W && fresh_from[t] >= 0) fresh_id[t] = p.freed[fresh_from[t]];
        __syncthreads();
    }
    for (int i0 = 0; i0 < a.W; i0 += 8) {  // eight children at a time, for the chains of reads from LDS
        int q[8], at[8], id[8], nb[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = min(i0 + k, a.W - 1);
            q[k] = f.parent[i], at[k] = fresh_at[i], id[k] = fresh_id[i];
            if (i0 + k >= a.W || at[k] == -1) q[k] = -1;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int last = f.nb[max(q[k], 0)] - 1, old = tile[max(q[k], 0) * kForkCols + t];
            nb[k] = q[k] < 0 ? 0 : last + 1;
            if (at[k] < 0 || c != last) {
                id[k] = old;
            } else if (q[k] >= 0) {  // the block that is not full
                if (id[k] < 0 || id[k] >= a.num_blocks) id[k] = -1;
                const bool copy = id[k] >= 0 && old >= 0 && old < a.num_blocks;
                a.copy_src[g * a.W + i0 + k] = copy ? old : -1;
                a.copy_dst[g * a.W + i0 + k] = copy ? id[k] : -1;
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (c < nb[k]) a.new_bt[((size_t)g * a.W + i0 + k) * a.max_blocks + c] = id[k];
    }
    if (part == 0 && t < a.W) {
        const int q = f.parent[t];
        a.new_lens[g * a.W + t] = q < 0 || fresh_at[t] == -1 ? 0 : f.len[q];
        if (fresh_at[t] < 0) a.copy_src[g * a.W + t] = a.copy_dst[g * a.W + t] = -1;
    }
    if (me == 0 && t == 0) {
        const int64_t end = (int64_t)start + fresh_all;
        a.counts[0] = (int)min(end, (int64_t)a.n_free);
        a.counts[1] = (int)max(end - a.n_free, (int64_t)0);
        a.counts[2] = all;
    }
}

// ---- copies of blocks --------------------------------------------------------------------------------------------------------
constexpr int kCopyArrays = 64, kCopyPiece = 16384, kCopyThreads = 256;
template <int N>  // in the kernel's arguments: 8 for a few, which the host writes half a microsecond faster, or 64
struct CopyArrays {
    uint32_t *at[N];
    int64_t bytes[N];
};
// A workgroup to a piece of 16 KB of a block in one array, 16 bytes a lane where the array's blocks begin at multiples of them.  grid: pieces, copies, arrays.  Bound by HBM where there is
// much to copy: 307 blocks of 64 KB in 8 pools, 322 MB, 55 us, 5.9 TB/s read and written.
template <int N>
__global__ void __launch_bounds__(kCopyThreads) k_copy_blocks(CopyArrays<N> a, const int32_t *src, const int32_t *dst, int num_blocks) {
    char *const p = (char *)a.at[blockIdx.z];
    const int64_t bytes = a.bytes[blockIdx.z], first = (int64_t)blockIdx.x * kCopyPiece;
    const int s = src[blockIdx.y], d = dst[blockIdx.y];
    if (s < 0 || d < 0 || s >= num_blocks || d >= num_blocks || s == d || first >= bytes) return;
    const char *from = p + s * bytes + first + threadIdx.x * 16;
    char *to = p + d * bytes + first + threadIdx.x * 16;
    const int n = (int)min((int64_t)kCopyPiece, bytes - first);
    const bool wide = ((uintptr_t)p | bytes) % 16 == 0;
    if (wide && n == kCopyPiece) {
        const uint4 v0 = *(const uint4 *)from, v1 = *(const uint4 *)(from + 4096), v2 = *(const uint4 *)(from + 8192), v3 = *(const uint4 *)(from + 12288);
        *(uint4 *)to = v0;
        *(uint4 *)(to + 4096) = v1;
        *(uint4 *)(to + 8192) = v2;
        *(uint4 *)(to + 12288) = v3;
    } else if (wide) {
        for (int k = threadIdx.x * 16; k < n; k += kCopyThreads * 16, from += kCopyThreads * 16, to += kCopyThreads * 16) *(uint4 *)to = *(const uint4 *)from;
    } else {
        from -= threadIdx.x * 12;
        to -= threadIdx.x * 12;
        for (int k = threadIdx.x * 4; k < n; k += kCopyThreads * 4, from += kCopyThreads * 4, to += kCopyThreads * 4) *(uint32_t *)to = *(const uint32_t *)from;
    }
}

// ---- attention over a shared prefix, any shape -------------------------------------------------------------------------------------
// A workgroup to a query head of a sequence; a thread to a position for the scores, to a channel for the sum of the values.  Running maximum and sum in float32, rounds
// of kChunk positions.  Each sequence reads its own table from the first column on: right for every block and head size, and slow.
constexpr int kChunk = 512;
template <typename T, typename KT>
__global__ void __launch_bounds__(256) k_prefix_attn_generic(PrefixAttnArgs a, int Hq, int Hkv, int D, int Bk, float scale, float k_scale, float v_scale) {
    __shared__ float qs[256], sc[kChunk], red[16];
    __shared__ int64_t where[kChunk];  // a position's element of channel 0 of the values, -1: masked
    const int s = blockIdx.y, h = blockIdx.x, c = h / (Hq / Hkv);
    bool grouped = false;
    for (int g = threadIdx.x; g < a.G; g += 256) grouped |= a.group_start[g] <= s && s < a.group_start[g + 1];
    if (!__syncthreads_or(grouped)) return;
    const int row0 = min(max(a.row_start[s], 0), a.R), row1 = min(max(a.row_start[s + 1], row0), a.R);
    const int64_t n = min((int64_t)max(a.kv_lens[s], 0), (int64_t)a.max_blocks * Bk);
    const int32_t *bt = a.bt + (size_t)s * a.max_blocks;
    const KT *pool = (const KT *)a.pool + (size_t)c * 2 * Bk * D;
    const size_t blk_stride = (size_t)Hkv * 2 * Bk * D;
    for (int row = row0; row < row1; ++row) {
        const T *q = (const T *)a.q + ((size_t)row * Hq + h) * D;
        __syncthreads();
        for (int i = threadIdx.x; i < D; i += 256) qs[i] = Elem<T>::ld(q + i);
        float m = -INFINITY, l = 0.f, acc = 0.f;
        for (int64_t t0 = 0; t0 < n; t0 += kChunk) {
            const int cnt = (int)min((int64_t)kChunk, n - t0);
            __syncthreads();
            float most = -INFINITY;
            for (int t = threadIdx.x; t < cnt; t += 256) {
                const int off = (int)((t0 + t) % Bk), id = bt[(t0 + t) / Bk];
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
            const float alpha = m == -INFINITY ? 1.f : __expf(m - m_new);  // before the first score there is nothing, or only NaN
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

}  // namespace

size_t beam_workspace(int G, int W, int vocab) {
    if (G == 0) return 256;
    return (size_t)G * W * beam_parts(vocab, beam_per(G, W, vocab)) * (16 + 8 * (size_t)W) + 256;
}

hipError_t launch_beam(const BeamArgs &a, void *workspace, hipStream_t st) {
    const int per = beam_per(a.G, a.W, a.vocab);
    BeamParts p;
    p.parts = beam_parts(a.vocab, per);
    p.sums = (double2 *)workspace;
    p.best = (uint64_t *)(p.sums + (size_t)a.G * a.W * p.parts);
    const dim3 grid(p.parts, a.G * a.W);
#define BEAM_PART(T)                                                                                                  \
    if (per == kBeamMany) hipLaunchKernelGGL((k_beam_part<T, kBeamMany>), grid, dim3(kBeamThreads), 0, st, a, p);     \
    else hipLaunchKernelGGL((k_beam_part<T, kBeamFew>), grid, dim3(kBeamThreads), 0, st, a, p)
    if (a.bf16) { BEAM_PART(bf16_t); }
    else { BEAM_PART(float); }
#undef BEAM_PART
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_beam_merge, dim3(a.G), dim3(kMergeThreads), 0, st, a, p);
    return hipGetLastError();
}

static int fork_parts(int max_blocks) { return std::max(1, (max_blocks + kForkCols - 1) / kForkCols); }
size_t fork_workspace(int G, int W, int max_blocks) {
    const size_t parts = (size_t)G * fork_parts(max_blocks);
    return (parts * W * kForkCols + parts + G) * 4 + 256;
}

hipError_t launch_fork(const ForkArgs &a, void *workspace, hipStream_t st) {
    ForkParts p;
    p.parts = fork_parts(a.max_blocks);
    p.freed = (int32_t *)workspace;
    p.freed_n = p.freed + (size_t)a.G * p.parts * a.W * kForkCols;
    p.fresh_n = p.freed_n + (size_t)a.G * p.parts;
    const dim3 grid(p.parts, a.G);
    const size_t lds = (size_t)a.W * kForkCols * 4;
    if (a.W <= 8) hipLaunchKernelGGL(k_fork_count<8>, grid, dim3(kForkCols), 0, st, a, p);
    else if (a.W <= 16) hipLaunchKernelGGL(k_fork_count<16>, grid, dim3(kForkCols), 0, st, a, p);
    else if (a.W <= 32) hipLaunchKernelGGL(k_fork_count<32>, grid, dim3(kForkCols), lds, st, a, p);
    else hipLaunchKernelGGL(k_fork_count<0>, grid, dim3(kForkCols), lds, st, a, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.W <= 8) hipLaunchKernelGGL(k_fork_write<8>, grid, dim3(kForkCols), lds, st, a, p);
    else if (a.W <= 16) hipLaunchKernelGGL(k_fork_write<16>, grid, dim3(kForkCols), lds, st, a, p);
    else if (a.W <= 32) hipLaunchKernelGGL(k_fork_write<32>, grid, dim3(kForkCols), lds, st, a, p);
    else hipLaunchKernelGGL(k_fork_write<0>, grid, dim3(kForkCols), lds, st, a, p);
    return hipGetLastError();
}

template <int N>
static hipError_t copy_launches(void *const *arrays, const int64_t *block_bytes, int cnt, const int32_t *src, const int32_t *dst, int n, int num_blocks, hipStream_t st) {
    CopyArrays<N> c{};
    int64_t most = 4;
    for (int i = 0; i < cnt; ++i) {
        c.at[i] = (uint32_t *)arrays[i];
        c.bytes[i] = block_bytes[i];
        most = std::max(most, c.bytes[i]);
    }
    const unsigned pieces = (unsigned)((most + kCopyPiece - 1) / kCopyPiece);  // at most 2^16
    for (int e = 0; e < n; e += 65535) {
        hipLaunchKernelGGL(k_copy_blocks<N>, dim3(pieces, std::min(65535, n - e), cnt), dim3(kCopyThreads), 0, st, c, src + e, dst + e, num_blocks);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

hipError_t launch_copy_blocks(void *const *arrays, const int64_t *block_bytes, int n_arrays, const int32_t *src, const int32_t *dst, int n, int num_blocks, hipStream_t st) {
    for (int i = 0; i < n_arrays; i += kCopyArrays) {
        const int cnt = std::min(kCopyArrays, n_arrays - i);
        const hipError_t e = cnt <= 8 ? copy_launches<8>(arrays + i, block_bytes + i, cnt, src, dst, n, num_blocks, st)
                                      : copy_launches<kCopyArrays>(arrays + i, block_bytes + i, cnt, src, dst, n, num_blocks, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_prefix_attn_generic(const Dims &dm, const PrefixAttnArgs &a, hipStream_t st) {
    const float scale = 1.f / sqrtf((float)dm.D);
    DISPATCH_TK(dm.bf16, dm.kv8, hipLaunchKernelGGL((k_prefix_attn_generic<T, KT>), dim3(dm.Hq, a.S), dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.D, dm.Bk, scale,
                                                    dm.k_scale, dm.v_scale));
    return hipGetLastError();
}

}  // namespace icarus
