// The cache in 8 bits: device-side view and the kernels that write and read it (declarations).
#pragma once
#include "common.cuh"

namespace freqkv {

constexpr int Q8_MAX_BATCH = 128;  // sequences per launch (lengths travel as kernel arguments)

struct Q8View {
    void* codes[2];   // K, V
    float* scales[2];  // dense [batch, layers, kv_heads, blocks]
    int64_t stride_batch, stride_layer, stride_head, stride_token;  // of the codes, in bytes
    int32_t layers, kv_heads, head_dim, blocks, block_tokens, kind;
};

// Rows from `src` (K, V of type `dtype`; element (b, l, h, t, c) at b*sb + l*sl + h*sh + t*st + c) become rows
// [begin[b], begin[b] + count[b]) of sequence b, b < batch (begin null: from row 0; count null: n_new rows); source row 0 goes to row begin[b].
struct Q8Source {
    const void* rows[2];
    int64_t stride_batch, stride_layer, stride_head, stride_token;  // elements
    int32_t dtype;
};
cudaError_t launch_quantize(const Q8View& cache, const Q8Source& src, int32_t batch, const int32_t* begin, const int32_t* count,
                            int32_t n_new, int32_t* launched, cudaStream_t stream);

// rows [0, lens[b]) of a bf16/fp32 cache <- code * scale.
cudaError_t launch_dequantize(const Q8View& cache, const CacheView& out, int32_t dtype, int32_t batch, const int32_t* lens,
                              int32_t* launched, cudaStream_t stream);

}  // namespace freqkv
