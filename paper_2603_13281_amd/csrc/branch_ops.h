// Launch interface of the operators for sequences that branch (include/icarus_branches.h): icarus_api.hip checks, these launch.
#pragma once
#include "kernels.h"

namespace icarus {

constexpr int kBeamMost = 64;  // sequences of a group that is chosen from or forked: a bit each of 64, a lane each of a wave

struct BeamArgs {
    const void *logits; int bf16, vocab; int64_t ld; int R, G, W;
    const int32_t *row_start; const float *scores; const int32_t *done; int eos;
    int32_t *parents, *tokens; float *scores_out; int32_t *done_out;
};
size_t beam_workspace(int G, int W, int vocab);
hipError_t launch_beam(const BeamArgs &a, void *workspace, hipStream_t st);

struct ForkArgs {
    const int32_t *parents, *kv_lens, *bt; int max_blocks, Bk, num_blocks, G, W;
    const int32_t *shared; int32_t *free_ids; int n_free; const int32_t *free_used;
    int32_t *new_lens, *new_bt, *copy_src, *copy_dst, *counts;
};
constexpr int kForkCols = 128;  // columns of a part: a thread each
size_t fork_workspace(int G, int W, int max_blocks);
hipError_t launch_fork(const ForkArgs &a, void *workspace, hipStream_t st);

hipError_t launch_copy_blocks(void *const *arrays, const int64_t *block_bytes, int n_arrays, const int32_t *src, const int32_t *dst, int n, int num_blocks, hipStream_t st);

struct PrefixAttnArgs {
    const void *q, *pool; const int32_t *bt; int max_blocks, num_blocks, S;
    const int32_t *kv_lens; int R; const int32_t *row_start; int G; const int32_t *group_start, *prefix_lens;
    void *out;
};
bool prefix_attn_fast(const Dims &dm);
size_t prefix_attn_workspace(const Dims &dm, int S, int G, int R, int max_blocks);
hipError_t launch_prefix_attn(const Dims &dm, const PrefixAttnArgs &a, void *workspace, hipStream_t st);
hipError_t launch_prefix_attn_generic(const Dims &dm, const PrefixAttnArgs &a, hipStream_t st);

}  // namespace icarus
