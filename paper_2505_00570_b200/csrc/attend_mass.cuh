// Decode attention that writes its scores down (declarations).
#pragma once
#include "attend.cuh"

namespace freqkv {

// Place t of a head in the partial results of attend_scores_kernel holds channel channel_of(t).
__host__ __device__ inline int channel_of(int t) { return (t & 7) * 16 + (t >> 3); }
// CTAs of the kernel that the chip holds at once.
int64_t attend_scores_resident(int sm_count);
// bf16, head_dim 128, g <= 8 query heads per KV head: sequences batch0 .. + batch_count, lens and tiles (of 16 rows a split) theirs.
cudaError_t launch_attend_scores(const freqkv_layout& l, const void* k, const void* v, int32_t layer, const void* q, int32_t g, int32_t batch0,
                                 int32_t batch_count, const int32_t* lens, const uint16_t* tiles, int32_t splits, const float2* table, float scale,
                                 float* partial, float* scores, int64_t score_rows, bool overlap, cudaStream_t stream);

}  // namespace freqkv
