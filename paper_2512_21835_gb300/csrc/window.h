// window.h -- what the windowed-serving operators share (window.cu, window_decode.cu,
// window_prefill.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "internal.h"

namespace loip {

constexpr int kPageTokens = 64;

// A scratch starts with the completion counters of the single-token attention, zero between
// calls.  Every operator leaves them alone or at zero and puts its partial states behind
// them, so that one scratch serves calls of any shape and of both kinds.
constexpr int kMaxCounters = 16384;
constexpr uint64_t kCounterBytes = kMaxCounters * sizeof(unsigned);

// Programmatic dependent launch: a kernel of this family lets its successor in the stream
// be launched as soon as all its own blocks are, and reads or writes global memory only
// after pdl_wait, which returns when the predecessor is complete and its writes are
// visible.  What overlaps is the launch and the set-up of a block.  The read-only path
// (ld.global.nc, __ldg) is not used for anything that a predecessor may write: the kernel
// may have been resident while that was written.
#ifdef __CUDACC__
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename Args>
cudaError_t launch_pdl(void (*kernel)(Args), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, const Args& args) {
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = st;
    c.attrs = at;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, kernel, args);
}

// Two fp32 numbers as a pair of bf16, to the nearest.
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// An fp32 number is the exact sum of three bf16 planes.  Each of the first two is the largest
// below what is left (in size), cut off and not rounded: so something of the number's own sign
// is always left, no plane of a number is zero (down to 2^-100 or so), and the product with
// an infinity is that infinity, as it would be in one piece.  (Rounded planes gave inf - inf,
// planes of zero 0 x inf.)  v (1 - 2^-24) is the fp32 number below v.
//
// The pair's next plane: v becomes v - plane, exactly.
__device__ __forceinline__ uint32_t peel(float& lo, float& hi) {
    const uint32_t a = __float_as_uint(lo * 0x1.fffffep-1f), b = __float_as_uint(hi * 0x1.fffffep-1f);
    lo -= __uint_as_float(a & 0xffff0000u);
    hi -= __uint_as_float(b & 0xffff0000u);
    return __byte_perm(a, b, 0x7632u);
}
#endif

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

// Attention of single tokens (window_decode.cu).  The scratch's size follows from the sizes
// alone.
uint64_t window_decode_scratch(int B, int Hq, int Hkv, int d, int window, int sinks, int max_ctx);
cudaError_t launch_window_decode(const WindowArgs& a, bool f32, cudaStream_t st);

// Attention of prompt rows (window_prefill.cu).
uint64_t window_prefill_scratch(int M, int n_prompts, int Hq, int Hkv, int d, int window, int sinks, int max_ctx);
cudaError_t launch_window_prefill(const WindowArgs& a, bool f32, cudaStream_t st);
cudaError_t window_prefill_error(int* code);  // first failure code of any launch (0 = none)

}  // namespace loip
