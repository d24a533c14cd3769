// Launch interface of the operators with lengths on the device (include/icarus_blocks.h): icarus_api.hip checks, these launch.
#pragma once
#include "kernels.h"

namespace icarus {

struct ExtendArgs {
    const int32_t *ctx_lens, *new_lens, *streams;  // streams: null or [S]
    int32_t *bt; int max_blocks, Bk, num_blocks, S;
    int64_t max_position;
    const int32_t *free_ids, *free_used; int n_free, max_rows;
    int32_t *kv_lens, *row_start, *row_seq, *row_pos; int64_t *row_slot; int32_t *counts;
};
hipError_t launch_extend(const ExtendArgs &a, hipStream_t st);

struct AppendArgs {
    const void *qkv; int64_t ld; int R;
    const int32_t *row_pos; const int64_t *row_slot;
    void *q_out, *pool; int64_t n_slots;           // slots of the pool
    const void *q_norm, *k_norm;                   // read with Dims::qk_norm
    int first;                                     // row that the launch begins with
};
// generic, here and below: only the kernels for any shape
hipError_t launch_append(const Dims &dm, bool generic, AppendArgs a, hipStream_t st);

struct BoundsArgs {
    const void *pool; const int32_t *bt; int max_blocks, num_blocks, S;
    const int32_t *from_lens, *to_lens; int max_new;
    int8_t *codes; float *scales;
};
hipError_t launch_bounds(const Dims &dm, bool generic, const BoundsArgs &a, hipStream_t st);

__host__ __device__ inline int key_pitch(int max_blocks) { return (max_blocks + 3) & ~3; }
struct SelectArgs {
    const void *q; const int8_t *codes; const float *scales;
    const int32_t *bt; int max_blocks, num_blocks, S;
    const int32_t *kv_lens, *row_start; int R, top_k, first, last;
    int32_t *blocks, *counts;
    float *scores;                                 // workspace [S, Hkv, key_pitch(max_blocks)], 16-byte aligned
};
hipError_t launch_select(const Dims &dm, bool generic, const SelectArgs &a, hipStream_t st);

struct BlockAttnArgs {
    const void *q, *pool; const int32_t *bt; int max_blocks, num_blocks, S;
    const int32_t *kv_lens, *row_start; int R, seq_rows;
    const int32_t *blocks, *counts; int max_selected;
    void *out;
};
// Shapes that block_attn_fast names.  Workspace: 16-byte aligned, block_attn_workspace bytes.
bool block_attn_fast(const Dims &dm);
size_t block_attn_workspace(const Dims &dm, int S, int R, int max_selected);
hipError_t launch_block_attn(const Dims &dm, const BlockAttnArgs &a, void *workspace, hipStream_t st);
hipError_t launch_block_attn_generic(const Dims &dm, const BlockAttnArgs &a, hipStream_t st);

}  // namespace icarus
