// Attention weights of a chunk's queries, added up per cache row (declarations).
#pragma once
#include "common.cuh"

namespace freqkv {

// Work areas: turned keys and queries as two fp16 parts each; maximum and sum of every query, and what the SMs have of some.
size_t mass_key_bytes(const freqkv_layout& l);
size_t mass_query_bytes(const freqkv_layout& l, int32_t q_heads_per_kv, int32_t n_new, int sm_count);
// mass [batch, layers, kv_heads, capacity] += the weights of q [batch, kv_heads * g, n_new, 128] (bf16) over layer `layer` of k.
cudaError_t launch_attend_chunk_mass(const freqkv_layout& l, const void* k, int32_t layer, const void* q, float* mass, int32_t g, int32_t n_new,
                                     const int32_t* lens_host, const float2* table, float scale, void* key_scratch, void* query_scratch,
                                     int sm_count, int32_t* status, unsigned long long wait_limit_ns, const char** error,
                                     int32_t* kernels_launched, cudaStream_t stream);

}  // namespace freqkv
