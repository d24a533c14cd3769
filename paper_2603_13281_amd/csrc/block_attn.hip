// Attention of single-token rows over the blocks that were selected for their sequence and kv-head.
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

}  // namespace

hipError_t launch_block_attn_generic(const Dims &dm, const BlockAttnArgs &a, hipStream_t st) {
    const float scale = 1.f / sqrtf((float)dm.D);
    DISPATCH_TK(dm.bf16, dm.kv8, hipLaunchKernelGGL((k_block_attn_generic<T, KT>), dim3(dm.Hq, a.S), dim3(256), 0, st, a, dm.Hq, dm.Hkv, dm.D, dm.Bk, scale,
                                                    dm.k_scale, dm.v_scale));
    return hipGetLastError();
}

}  // namespace icarus
