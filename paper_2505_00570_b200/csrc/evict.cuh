// Eviction of the rows with the least accumulated attention weight (declarations).
#pragma once
#include "common.cuh"

namespace freqkv {

constexpr int EVICT_MAX_BATCH = 128;  // sequences per launch (lengths travel as kernel arguments)

// Of rows [0, lens[b]) of every (batch, layer, kv_head) keep the first `sink`, the last `recent` and the kept[b] - recent heaviest
// between; K, V and mass move together to rows [0, sink + kept[b]).  mass, mass_out: [batch, layers, kv_heads, capacity], may be
// equal; rows: [batch, layers, kv_heads, rows_stride] the kept rows' old indexes.
cudaError_t launch_evict(const CacheView& view, int32_t dtype, int32_t batch, int32_t capacity, const float* mass, float* mass_out,
                         int32_t* rows, int64_t rows_stride, const int32_t* lens, const int32_t* kept, int32_t sink, int32_t recent,
                         int sm_count, int32_t* launched, cudaStream_t stream);

}  // namespace freqkv
