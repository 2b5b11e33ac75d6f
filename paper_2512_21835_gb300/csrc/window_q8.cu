// window_q8.cu -- the attention behind a sliding window with sinks over the 8-bit cache: a warp
// per row and head, position by position.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "internal.h"
#include "window.h"
#include "window_walk.h"

namespace loip {
namespace {

constexpr int kWarps = 4;

template <int D, typename T>
__global__ void __launch_bounds__(kWarps * 32) window_walk_kernel(const __grid_constant__ WindowArgs a) {
    pdl_trigger();
    pdl_wait();
    const int64_t i = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    if (i >= (int64_t)a.rows * a.Hq) return;
    const int row = (int)(i / a.Hq), head = (int)(i % a.Hq);
    int req = row, pos;
    if (a.ctx_lens) {
        pos = min(a.ctx_lens[row], a.max_ctx) - 1;
    } else {
        for (req = 0; req < a.n_prompts && row >= a.row_starts[req + 1]; ++req) {}
        if (req == a.n_prompts || row < a.row_starts[req]) return;  // behind the last prompt
        pos = (a.first_pos ? a.first_pos[req] : 0) + row - a.row_starts[req];
    }
    walk_row<D, true, T>(a, req, head / (a.Hq / a.Hkv), pos, static_cast<const T*>(a.q) + i * D,
                         static_cast<T*>(a.o) + i * D);
}

cudaError_t launch(WindowArgs a, bool f32, cudaStream_t st) {
    a.window = a.window > 1 << 30 ? 1 << 30 : a.window;  // positions are below max_ctx <= 2^30
    a.sinks = a.sinks > 1 << 30 ? 1 << 30 : a.sinks;
    const int64_t blocks = ((int64_t)a.rows * a.Hq + kWarps - 1) / kWarps;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    const dim3 grid((unsigned)blocks);
    if (a.d == 128)
        return f32 ? launch_pdl(window_walk_kernel<128, float>, grid, kWarps * 32, 0, st, a)
                   : launch_pdl(window_walk_kernel<128, __nv_bfloat16>, grid, kWarps * 32, 0, st, a);
    return f32 ? launch_pdl(window_walk_kernel<64, float>, grid, kWarps * 32, 0, st, a)
               : launch_pdl(window_walk_kernel<64, __nv_bfloat16>, grid, kWarps * 32, 0, st, a);
}

}  // namespace

uint64_t window_prefill_q8_scratch(int M, int n_prompts, int Hq, int Hkv, int d, int window, int sinks, int max_ctx) {
    return window_prefill_scratch(M, n_prompts, Hq, Hkv, d, window, sinks, max_ctx);
}
cudaError_t launch_window_prefill_q8(const WindowArgs& a, bool f32, cudaStream_t st) { return launch(a, f32, st); }

}  // namespace loip
