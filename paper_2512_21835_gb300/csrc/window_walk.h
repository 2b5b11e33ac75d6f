// window_walk.h -- the attention of one row, position by position: what the prompt attentions
// fall back on where a tile holds values that are not finite and that not all its rows see.
#pragma once
#include "q8.h"
#include "window.h"

namespace loip {
namespace {

__device__ __forceinline__ float row_load(const float* p) { return *p; }
__device__ __forceinline__ float row_load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void row_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void row_store(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// One row by one warp, position by position: what is not seen is not touched.
template <int D, bool Q8, typename T>
__device__ __forceinline__ void walk_row(const WindowArgs& a, int req, int kvh, int pos, const T* q, T* out) {
    const int lane = threadIdx.x % 32;
    const char* layer = a.kv.base + (uint64_t)a.kv.layer * a.kv.layer_page_bytes;
    float qv[D / 32], o[D / 32], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        qv[i] = row_load(q + i * 32 + lane);
        o[i] = 0.f;
    }
    const float scale = 1.0f / sqrtf((float)D);
    const int last = min(pos, a.max_ctx - 1);
    for (int j = 0; j <= last; ++j) {
        if (j >= a.sinks && j <= pos - a.window) {  // to the window's first position
            j = pos - a.window;
            continue;
        }
        const char* page = layer + a.kv.page_offsets[(int64_t)req * a.kv.max_pages + j / kPageTokens];
        float k[D / 32], v[D / 32];
        if constexpr (Q8) {
            using G = q8::Granule<D>;
            const char* g = page + q8::granule_at<D>(kvh, j);
            auto element = [&](int is_v, int i) {
                const int t = j % q8::kGranule;
                return q8::value_of((uint8_t)g[G::piece(is_v, t, 2 * i + lane / 16) + lane % 16],
                                    q8::step_of((uint8_t)g[G::exponents(is_v, t) + i]));
            };
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                k[i] = element(0, i);
                v[i] = element(1, i);
            }
        } else {
            const __nv_bfloat16* at =
                reinterpret_cast<const __nv_bfloat16*>(page) + ((int64_t)kvh * kPageTokens + j % kPageTokens) * D;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                k[i] = __bfloat162float(at[i * 32 + lane]);
                v[i] = __bfloat162float(at[(int64_t)a.Hkv * kPageTokens * D + i * 32 + lane]);
            }
        }
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) s = fmaf(qv[i], k[i], s);
#pragma unroll
        for (int x = 16; x; x /= 2) s += __shfl_xor_sync(0xffffffffu, s, x);
        s *= scale;
        const float m_new = fmaxf(m, s), alpha = m == -INFINITY ? 0.f : expf(m - m_new);
        const float w = expf(s - (m_new == -INFINITY ? 0.f : m_new));  // a score of -inf: weight zero, the first one too
        l = l * alpha + w;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) o[i] = fmaf(w, v[i], o[i] * alpha);
        m = m_new;
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) row_store(out + i * 32 + lane, o[i] * inv);
}

}  // namespace
}  // namespace loip
