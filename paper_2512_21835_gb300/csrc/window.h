// window.h -- what the windowed-serving operators share (window.cu, window_tc.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "internal.h"

namespace loip {

constexpr int kPageTokens = 64;

// Attention of query rows over the paged cache behind a window with sinks: the
// query at position p sees the cached positions j <= p with j > p - window or
// j < sinks.
struct WindowArgs {
    const void* q;  // [rows, Hq * d] fp32 or bf16
    void* o;        // same shape and type
    KvView kv;
    const int32_t* ctx_lens;    // single tokens: cached positions of each request
    const int32_t* row_starts;  // prompts: [n_prompts + 1]
    const int32_t* first_pos;   // prompts: [n_prompts] or null
    int rows, n_prompts;
    int Hq, Hkv, d;
    int window, sinks, max_ctx;
    void* scratch;
};

// Attention of single tokens (window_decode.cu).  The scratch starts with completion
// counters that a call leaves at zero; its size follows from the sizes alone.
uint64_t window_decode_scratch(int B, int Hq, int Hkv, int d, int window, int sinks, int max_ctx);
cudaError_t launch_window_decode(const WindowArgs& a, bool f32, cudaStream_t st);

// Attention of prompt rows (window_prefill.cu).
uint64_t window_prefill_scratch(int M, int n_prompts, int Hq, int Hkv, int d, int window, int sinks, int max_ctx);
cudaError_t launch_window_prefill(const WindowArgs& a, bool f32, cudaStream_t st);
cudaError_t window_prefill_error(int* code);  // first failure code of any launch (0 = none)

}  // namespace loip
