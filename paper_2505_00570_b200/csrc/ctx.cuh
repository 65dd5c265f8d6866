// The context behind the C ABI and what the files that implement it share (internal).
#pragma once

#include <map>
#include <string>
#include <tuple>
#include <utility>
#include <vector>

#include "attend.cuh"
#include "common.cuh"
#include "dctmm.cuh"
#include "fdct.cuh"
#include "gemm.cuh"

struct freqkv_ctx {
    int device = 0;
    int sm_count = 0;
    freqkv_variant forced = FREQKV_AUTO;
    std::map<std::tuple<int32_t, int32_t, int32_t>, freqkv::Basis> bases;  // (n_in, n_keep, first retained component)
    std::map<std::pair<int32_t, int32_t>, freqkv::FdctPlan> fdct_plans;
    // keys: (n_in, n_keep, family of factorisation asked for: 0 = the kernel's own choice)
    std::map<std::tuple<int32_t, int32_t, int32_t>, freqkv::DctmmPlan> dctmm_plans;
    std::map<std::tuple<int32_t, int32_t, int32_t>, bool> dctmm_fits;  // does a factorisation meet the kernel's limits
    int32_t fast_family = 0;
    size_t basis_bytes = 0;
    void* scratch = nullptr;
    size_t scratch_bytes = 0;
    int32_t* status_dev = nullptr;
    freqkv::GemmState gemm;
    std::string last_error;
    // Work areas (folded rows, far sums, staging, attention partials) are shared by all calls on this
    // context: a call on another stream than the previous one first waits for that one's work.
    cudaEvent_t work_done = nullptr;
    cudaStream_t work_stream = nullptr;
    bool work_recorded = false;
    // instrumentation
    bool timing = false;
    std::vector<std::pair<cudaEvent_t, cudaEvent_t>> pending, spare;
    int64_t kernels_launched = 0;
    // host-buffer entry point: device staging caches
    void* stage[2] = {nullptr, nullptr};
    size_t stage_bytes = 0;
    // decode attention: RoPE table of one base, partial results of the row splits
    float2* rope_table = nullptr;
    int32_t rope_rows = 0;
    double rope_base = 0.0;
    cudaEvent_t rope_made = nullptr;  // the table's making; rope_settled: it is known to be over
    bool rope_settled = false;
    void* attend_work = nullptr;  // attend_ticket_bytes of tickets, then the splits' partials
    size_t attend_work_bytes = 0;
    int32_t* attend_lens = nullptr;  // host: the last call's lengths; what else its split of the rows follows from; that split
    int32_t attend_lens_room = 0, attend_key[4] = {0, 0, 0, 0};
    freqkv::AttendPlan attend_last = {};
    bool attend_tickets_clear = false;  // zeroed on a stream that later calls are ordered behind
    void* prefill_keys = nullptr;     // rotated keys of one layer, fp16
    size_t prefill_keys_bytes = 0;
    void* prefill_queries = nullptr;  // rotated, scaled queries of one chunk, fp16
    size_t prefill_queries_bytes = 0;
    cudaStream_t pipe[3] = {nullptr, nullptr, nullptr};  // copy in, compress, copy out
    cudaEvent_t pipe_begin = nullptr, pipe_end = nullptr;
    std::vector<cudaEvent_t> pipe_events;                // per group: copied in, compressed
};

namespace freqkv {

struct DeviceGuard {
    int prev = -1;
    bool ok = true, changed = false;
    explicit DeviceGuard(int dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
        if (prev == dev) return;
        changed = true;
        if (cudaSetDevice(dev) != cudaSuccess) ok = false;
    }
    ~DeviceGuard()
    {
        if (changed) cudaSetDevice(prev);
    }
};

// Orders the calls that use the context's work areas: on entry the caller's stream waits for the
// previous such call if that one ran on a different stream; on exit the end of this call's work
// is recorded.  (Calls on one stream are ordered anyway and pay nothing.)
struct WorkOrder {
    freqkv_ctx* ctx;
    cudaStream_t stream;
    bool captured;  // a captured call enqueues nothing now, and its replays are the caller's to order
    WorkOrder(freqkv_ctx* c, cudaStream_t s);
    ~WorkOrder();
};

// Notes the failure for freqkv_last_error, clears the error state, gives the status to return.
freqkv_status cuda_fail(freqkv_ctx* ctx, cudaError_t e, const char* where);
bool is_capturing(cudaStream_t stream);
// The layout rules of freqkv_layout; K and V there, aligned and apart.
freqkv_status check_layout(const freqkv_layout* l);
freqkv_status check_tensors(const freqkv_layout& l, const void* k, const void* v);
int64_t span_elements(const freqkv_layout& l);
bool apart(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes);
CacheView make_view(const freqkv_layout& l, void* k, void* v, int32_t batch0, int32_t batch_count);
// The context's staging area, of `bytes` at least.
freqkv_status get_scratch(freqkv_ctx* ctx, size_t bytes, void** out);
// The context's cos/sin table of `rope_base`, of `capacity` rows at least; *table stays null when RoPE is off.
freqkv_status rope_table_for(freqkv_ctx* ctx, int32_t capacity, float rope_base, cudaStream_t stream, const float2** table);

// The split of the rows of a decode attention of `groups` (kv head, ...) groups a sequence; the work area of the call: tickets, the
// splits' partials of q_heads heads a sequence, `more` bytes for the caller (256-byte aligned).
AttendPlan attend_plan_for(freqkv_ctx* ctx, int32_t batch, int32_t groups, int64_t resident, int32_t overhead_rows, const int32_t* lens);
struct AttendWork {
    int32_t* tickets;
    float* partial;
    char* more;
};
freqkv_status attend_work_for(freqkv_ctx* ctx, const AttendPlan& plan, int32_t batch, int32_t q_heads, int32_t capacity, size_t more,
                              cudaStream_t stream, AttendWork* out);

// Makes the prefill attention's two scratch buffers at least so large.
freqkv_status prefill_scratch(freqkv_ctx* ctx, size_t key_bytes, size_t query_bytes);

#define FREQKV_CUDA(ctx, call)                                             \
    do {                                                                   \
        const cudaError_t e__ = (call);                                    \
        if (e__ != cudaSuccess) return cuda_fail((ctx), e__, #call);       \
    } while (0)

struct TransformTimer {
    freqkv_ctx* ctx;
    cudaStream_t stream;
    std::pair<cudaEvent_t, cudaEvent_t> ev{nullptr, nullptr};
    TransformTimer(freqkv_ctx* c, cudaStream_t s) : ctx(c), stream(s) { begin(); }
    TransformTimer(freqkv_ctx* c, cudaStream_t s, bool start_now) : ctx(c), stream(s)
    {
        if (start_now) begin();
    }
    void begin()
    {
        if (!ctx->timing) return;
        if (!ctx->spare.empty()) {
            ev = ctx->spare.back();
            ctx->spare.pop_back();
        } else if (cudaEventCreate(&ev.first) != cudaSuccess || cudaEventCreate(&ev.second) != cudaSuccess) {
            ev = {nullptr, nullptr};
            cudaGetLastError();
            return;
        }
        cudaEventRecord(ev.first, stream);
    }
    void end()
    {
        if (!ev.first) return;
        cudaEventRecord(ev.second, stream);
        ctx->pending.push_back(ev);
        ev = {nullptr, nullptr};
    }
    ~TransformTimer() { end(); }
};

}  // namespace freqkv
