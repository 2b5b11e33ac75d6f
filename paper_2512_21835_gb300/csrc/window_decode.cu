// window_decode.cu -- attention of one new token per request over the paged
// cache, behind a sliding window with sinks.
//
// For each request and kv head the R <= 8 query heads of a group share every key
// and value, so the cache is read once per group and is all the traffic: 4 d bytes
// per visible position and kv head, against 4 R d flop.  At full memory bandwidth
// that is 27 TFLOP/s for eight heads (and three times that with the split operands
// below), too much for the fp32 pipe beside the conversions; the warp-wide bf16
// MMAs (m16n8k16) have it to spare, and their fragments can be loaded from global
// memory directly, so there is no shared-memory staging and no barrier in the loop.
//
// A tile is 16 consecutive positions (a quarter of a page), one warp's step:
//   S [R x 16] = Q K^T   A = Q rows, B = keys; the contraction index d is permuted so
//                        that a lane's B registers are 16 contiguous bytes of its key:
//                        lane 4 n + c holds, of key n, the elements 32 i + 8 c .. + 7
//   O [R x d] += P V     A = P straight from the accumulator layout of S; a lane
//                        loads 16 contiguous bytes of four value rows and pairs
//                        adjacent rows with byte permutes (columns of O permuted
//                        likewise: lane 4 n + c, register m: element 64 i + 8 n + m)
//
// Precision.  The MMA's 16 rows hold 8 heads twice.  An fp32 query is the exact sum
// of three bf16 planes: the first two go to rows 0-7 and 8-15 of one MMA, the third
// to rows 0-7 of another; the row pairs are added in fp32.  Weights likewise (two
// planes, 2^-17, for bf16 activations: the second plane's rows are there anyway).
//
// Masked positions are neither loaded nor multiplied: their key and value registers
// are zero, whatever the cache holds there.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "window.h"

namespace loip {
namespace {

constexpr int kTile = 16;   // positions per warp step
constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kMaxCounters = 16384;  // completion counters, at the start of the scratch

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// The pair's next plane: v becomes v - bf16(v), exactly.
__device__ __forceinline__ uint32_t peel(float& lo, float& hi) {
    const uint32_t p = pack(lo, hi);
    lo -= __uint_as_float(p << 16);
    hi -= __uint_as_float(p & 0xffff0000u);
    return p;
}
__device__ __forceinline__ uint4 load_row(const char* p, bool live) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (live)
        asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "l"(p));
    return v;
}

struct Plan {
    int heads;    // query heads per group
    int groups;   // groups per kv head
    int chunk;    // tiles per block
    int splits;   // blocks per (request, group)
};

struct DecodeArgs {
    WindowArgs a;
    Plan plan;
    unsigned* counters;
    float2* ml;     // [request][group][split][heads]: maximum (log2), sum
    float* part;    // [request][group][split][heads][d], not normalised
};

template <int D, typename T>
__global__ void __launch_bounds__(kThreads, 2) window_decode_kernel(const __grid_constant__ DecodeArgs p) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NQ = D / 32;  // 16-byte pieces of a key per lane
    constexpr int NV = D / 64;  // 16-byte pieces of a value row per lane
    __shared__ __align__(16) float sm_o[kWarps][8][D];
    __shared__ float sm_m[kWarps][8], sm_l[kWarps][8];
    __shared__ bool sm_last;
    const WindowArgs& a = p.a;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, n4 = lane / 4, c4 = lane % 4;
    const int b = blockIdx.x / p.plan.splits, split = blockIdx.x % p.plan.splits;
    const int kvh = blockIdx.y / p.plan.groups, G = a.Hq / a.Hkv;
    const int head0 = (blockIdx.y % p.plan.groups) * p.plan.heads;          // of the kv head's G
    const int heads = min(p.plan.heads, G - head0);
    const int ctx = max(0, min(a.ctx_lens[b], a.max_ctx));
    // visible tiles: those of the sinks, then those of the window (which may touch)
    const int win0 = a.window >= ctx ? 0 : ctx - a.window;                  // first position of the window
    const int tiles_end = (ctx + kTile - 1) / kTile;
    const int sink_tiles = min((int)(((int64_t)a.sinks + kTile - 1) / kTile), tiles_end);
    const int win_tile = a.window == 0 ? tiles_end : max(win0 / kTile, sink_tiles);
    const int tiles = sink_tiles + max(0, tiles_end - win_tile);
    const int active = max(1, (tiles + p.plan.chunk - 1) / p.plan.chunk);   // blocks with work
    if (split >= active) return;
    const int last = min(tiles, (split + 1) * p.plan.chunk);

    // queries: bf16 planes in the A layout, rows past the group's heads zero
    uint32_t qa[NQ][2][2], qb[F32 ? NQ : 1][2][2], qc[F32 ? NQ : 1][2][2];
    {
        const T* q = static_cast<const T*>(a.q) + ((int64_t)b * a.Hq + kvh * G + head0 + n4) * D + 8 * c4;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if constexpr (F32) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.f;
                if (n4 < heads) {
                    const float4 x = *reinterpret_cast<const float4*>(q + 32 * i);
                    const float4 y = *reinterpret_cast<const float4*>(q + 32 * i + 4);
                    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    qa[i][e / 2][e % 2] = peel(v[2 * e], v[2 * e + 1]);
                    qb[i][e / 2][e % 2] = peel(v[2 * e], v[2 * e + 1]);
                    qc[i][e / 2][e % 2] = pack(v[2 * e], v[2 * e + 1]);
                }
            } else {
                const uint4 x = n4 < heads ? *reinterpret_cast<const uint4*>(q + 32 * i) : make_uint4(0u, 0u, 0u, 0u);
                qa[i][0][0] = x.x; qa[i][0][1] = x.y; qa[i][1][0] = x.z; qa[i][1][1] = x.w;
            }
        }
    }

    const char* layer = a.kv.base + (uint64_t)a.kv.layer * a.kv.layer_page_bytes;
    const int64_t* table = a.kv.page_offsets + (int64_t)b * a.kv.max_pages;
    auto tile_at = [&](int i) { return i < sink_tiles ? i : i - sink_tiles + win_tile; };
    auto seen = [&](int j) { return j < ctx && (j >= win0 || j < a.sinks); };
    // the tile's first key of this kv head
    auto key_at = [&](int t) {
        return layer + __ldg(table + t / (kPageTokens / kTile)) +
               (uint32_t)((kvh * kPageTokens + (t % (kPageTokens / kTile)) * kTile) * D * 2);
    };
    const uint32_t v_off = (uint32_t)(a.Hkv * kPageTokens) * D * 2;

    float o[8 * NV][4];
#pragma unroll
    for (int i = 0; i < 8 * NV; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m = -INFINITY, l = 0.f;
    const float scale = 1.44269504088896f / sqrtf((float)D);  // scores in units of log 2

    uint4 k[2][NQ], v[4][NV];
    auto load_k = [&](int t, const char* at) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bool live = seen(t * kTile + 8 * j + n4);
#pragma unroll
            for (int i = 0; i < NQ; ++i) k[j][i] = load_row(at + ((8 * j + n4) * D + 32 * i + 8 * c4) * 2, live);
        }
    };
    int i = split * p.plan.chunk + warp;
    const char* at = nullptr;
    if (i < last) {
        at = key_at(tile_at(i));
        load_k(tile_at(i), at);
    }
    for (; i < last; i += kWarps) {
        const int t = tile_at(i);
        const char* at_next = i + kWarps < last ? key_at(tile_at(i + kWarps)) : nullptr;
#pragma unroll
        for (int r = 0; r < 4; ++r) {  // value rows 2 c4, 2 c4 + 1, 2 c4 + 8, 2 c4 + 9
            const int row = 2 * c4 + (r & 1) + 8 * (r >> 1);
            const bool live = seen(t * kTile + row);
#pragma unroll
            for (int x = 0; x < NV; ++x) v[r][x] = load_row(at + v_off + (row * D + 64 * x + 8 * n4) * 2, live);
        }
        // ---- scores
        float s[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
            if constexpr (F32) {  // the smallest plane first
#pragma unroll
                for (int x = 0; x < NQ; ++x) {
                    mma(s[j], qc[x][0][0], 0u, qc[x][0][1], 0u, k[j][x].x, k[j][x].y);
                    mma(s[j], qc[x][1][0], 0u, qc[x][1][1], 0u, k[j][x].z, k[j][x].w);
                }
            }
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                if constexpr (F32) {
                    mma(s[j], qa[x][0][0], qb[x][0][0], qa[x][0][1], qb[x][0][1], k[j][x].x, k[j][x].y);
                    mma(s[j], qa[x][1][0], qb[x][1][0], qa[x][1][1], qb[x][1][1], k[j][x].z, k[j][x].w);
                } else {
                    mma(s[j], qa[x][0][0], 0u, qa[x][0][1], 0u, k[j][x].x, k[j][x].y);
                    mma(s[j], qa[x][1][0], 0u, qa[x][1][1], 0u, k[j][x].z, k[j][x].w);
                }
            }
        }
        if (at_next) load_k(tile_at(i + kWarps), at_next);
        // ---- softmax: this lane has head n4, positions 8 j + 2 c4 + {0, 1}
        float w[2][2], mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                w[j][e] = seen(t * kTile + 8 * j + 2 * c4 + e) ? (s[j][e] + s[j][e + 2]) * scale : -INFINITY;
                mx = fmaxf(mx, w[j][e]);
            }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        if (__any_sync(0xffffffffu, mx > m)) {
            const float m_new = fmaxf(m, mx);
            const float alpha = m == -INFINITY ? 0.f : exp2f(m - m_new);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int x = 0; x < 8 * NV; ++x) {
                o[x][0] *= alpha; o[x][1] *= alpha; o[x][2] *= alpha; o[x][3] *= alpha;
            }
        }
        const float base = m == -INFINITY ? 0.f : m;  // nothing seen yet: every weight is zero
        uint32_t p0[2], p1[2], p2[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            w[j][0] = exp2f(w[j][0] - base);
            w[j][1] = exp2f(w[j][1] - base);
            l += w[j][0] + w[j][1];
            p0[j] = peel(w[j][0], w[j][1]);
            if constexpr (F32) {
                p1[j] = peel(w[j][0], w[j][1]);
                p2[j] = pack(w[j][0], w[j][1]);
            } else {
                p1[j] = pack(w[j][0], w[j][1]);
            }
        }
        // ---- values
#pragma unroll
        for (int x = 0; x < NV; ++x) {
            const uint32_t r0[4] = {v[0][x].x, v[0][x].y, v[0][x].z, v[0][x].w};
            const uint32_t r1[4] = {v[1][x].x, v[1][x].y, v[1][x].z, v[1][x].w};
            const uint32_t r2[4] = {v[2][x].x, v[2][x].y, v[2][x].z, v[2][x].w};
            const uint32_t r3[4] = {v[3][x].x, v[3][x].y, v[3][x].z, v[3][x].w};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t sel = e & 1 ? 0x7632u : 0x5410u;
                const uint32_t b0 = __byte_perm(r0[e / 2], r1[e / 2], sel), b1 = __byte_perm(r2[e / 2], r3[e / 2], sel);
                if constexpr (F32) mma(o[8 * x + e], p2[0], 0u, p2[1], 0u, b0, b1);
                mma(o[8 * x + e], p0[0], p1[0], p0[1], p1[1], b0, b1);
            }
        }
        at = at_next;
    }

    // ---- join the warps: head n4, elements 64 x + 8 (2 c4 + e) + y
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    if (c4 == 0) {
        sm_m[warp][n4] = m;
        sm_l[warp][n4] = l;
    }
#pragma unroll
    for (int x = 0; x < NV; ++x)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int y = 0; y < 8; y += 4) {
                float4 r;
                r.x = o[8 * x + y][e] + o[8 * x + y][e + 2];
                r.y = o[8 * x + y + 1][e] + o[8 * x + y + 1][e + 2];
                r.z = o[8 * x + y + 2][e] + o[8 * x + y + 2][e + 2];
                r.w = o[8 * x + y + 3][e] + o[8 * x + y + 3][e + 2];
                *reinterpret_cast<float4*>(&sm_o[warp][n4][64 * x + 8 * (2 * c4 + e) + y]) = r;
            }
    __syncthreads();
    const int64_t unit = (int64_t)b * gridDim.y + blockIdx.y;
    const int units = heads * (D / 4);  // four elements of a head each
    T* out = static_cast<T*>(a.o) + ((int64_t)b * a.Hq + kvh * G + head0) * D;
    auto put = [&](int u, float4 r, float inv) {
        r.x *= inv; r.y *= inv; r.z *= inv; r.w *= inv;
        if constexpr (F32)
            reinterpret_cast<float4*>(out)[u] = r;
        else
            reinterpret_cast<uint2*>(out)[u] = make_uint2(pack(r.x, r.y), pack(r.z, r.w));
    };
    for (int u = threadIdx.x; u < units; u += kThreads) {
        const int h = u / (D / 4);
        float mt = -INFINITY, lt = 0.f;
#pragma unroll
        for (int x = 0; x < kWarps; ++x) mt = fmaxf(mt, sm_m[x][h]);
        float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int x = 0; x < kWarps; ++x) {
            const float f = sm_m[x][h] == -INFINITY ? 0.f : exp2f(sm_m[x][h] - mt);
            const float4 y = *reinterpret_cast<const float4*>(&sm_o[x][h][4 * (u % (D / 4))]);
            lt = fmaf(f, sm_l[x][h], lt);
            r.x = fmaf(f, y.x, r.x); r.y = fmaf(f, y.y, r.y); r.z = fmaf(f, y.z, r.z); r.w = fmaf(f, y.w, r.w);
        }
        if (active == 1) {
            put(u, r, lt == 0.f ? 0.f : 1.0f / lt);
        } else {
            const int64_t at = (unit * p.plan.splits + split) * p.plan.heads + h;
            __stcg(reinterpret_cast<float4*>(p.part + at * D) + u % (D / 4), r);
            if (u % (D / 4) == 0) __stcg(p.ml + at, make_float2(mt, lt));
        }
    }
    if (active == 1) return;
    // ---- join the blocks: the last one to arrive sums all parts, in their order; the
    // counter wraps to zero with that arrival
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) sm_last = atomicInc(p.counters + unit, (unsigned)active - 1u) == (unsigned)active - 1u;
    __syncthreads();
    if (!sm_last) return;
    __threadfence();
    for (int u = threadIdx.x; u < units; u += kThreads) {
        const int h = u / (D / 4);
        const int64_t first = unit * p.plan.splits * p.plan.heads + h;
        float mt = -INFINITY, lt = 0.f;
#pragma unroll 8
        for (int x = 0; x < active; ++x) mt = fmaxf(mt, __ldcg(p.ml + first + (int64_t)x * p.plan.heads).x);
        float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int x = 0; x < active; ++x) {
            const int64_t at = first + (int64_t)x * p.plan.heads;
            const float2 ml = __ldcg(p.ml + at);
            const float4 y = __ldcg(reinterpret_cast<const float4*>(p.part + at * D) + u % (D / 4));
            const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - mt);
            lt = fmaf(f, ml.y, lt);
            r.x = fmaf(f, y.x, r.x); r.y = fmaf(f, y.y, r.y); r.z = fmaf(f, y.z, r.z); r.w = fmaf(f, y.w, r.w);
        }
        put(u, r, lt == 0.f ? 0.f : 1.0f / lt);
    }
}

// Blocks of `chunk` tiles.  Small problems take the smallest block (a tile per warp),
// so that they spread over the card; large ones take blocks long enough to hide their
// first loads and the join, short enough to leave no long tail.
Plan make_plan(int B, int Hq, int Hkv, int window, int sinks, int max_ctx) {
    Plan p{};
    const int G = Hq / Hkv;
    p.groups = (G + 7) / 8;
    p.heads = (G + p.groups - 1) / p.groups;
    const int64_t tiles = std::min<int64_t>(((int64_t)max_ctx + kTile - 1) / kTile,
                                            ((int64_t)window + kTile - 1) / kTile + 1 +
                                                ((int64_t)sinks + kTile - 1) / kTile);
    const int64_t units = (int64_t)B * Hkv * p.groups;
    int64_t chunk = (units * tiles / (152 * 16) + kWarps - 1) / kWarps * kWarps;
    chunk = std::min<int64_t>(std::max<int64_t>(chunk, kWarps), 64);
    if (units > kMaxCounters) chunk = tiles;
    p.chunk = (int)std::max<int64_t>(chunk, 1);
    p.splits = (int)std::max<int64_t>((tiles + p.chunk - 1) / p.chunk, 1);
    return p;
}

template <int D, typename T>
cudaError_t launch_t(const DecodeArgs& p, cudaStream_t st) {
    window_decode_kernel<D, T>
        <<<dim3((unsigned)p.a.rows * p.plan.splits, p.a.Hkv * p.plan.groups), kThreads, 0, st>>>(p);
    return cudaGetLastError();
}

}  // namespace

uint64_t window_decode_scratch(int B, int Hq, int Hkv, int d, int window, int sinks, int max_ctx) {
    const Plan p = make_plan(B, Hq, Hkv, window, sinks, max_ctx);
    uint64_t n = kMaxCounters * sizeof(unsigned);
    if (p.splits > 1) n += (uint64_t)B * Hkv * p.groups * p.splits * p.heads * (d + 2) * sizeof(float);
    return (n + 15) / 16 * 16;
}

cudaError_t launch_window_decode(const WindowArgs& a, bool f32, cudaStream_t st) {
    DecodeArgs p{};
    p.a = a;
    p.plan = make_plan(a.rows, a.Hq, a.Hkv, a.window, a.sinks, a.max_ctx);
    if ((int64_t)a.rows * p.plan.splits > 0x7fffffff) return cudaErrorInvalidValue;
    const int64_t parts = (int64_t)a.rows * a.Hkv * p.plan.groups * p.plan.splits * p.plan.heads;
    p.counters = static_cast<unsigned*>(a.scratch);
    p.part = reinterpret_cast<float*>(p.counters + kMaxCounters);
    p.ml = reinterpret_cast<float2*>(p.part + parts * a.d);
    if (a.d == 128) return f32 ? launch_t<128, float>(p, st) : launch_t<128, __nv_bfloat16>(p, st);
    return f32 ? launch_t<64, float>(p, st) : launch_t<64, __nv_bfloat16>(p, st);
}

}  // namespace loip
