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
// A tile is 16 consecutive positions (a quarter of a page), one warp's step.  The heads
// are the MMA's eight columns, the cache its sixteen rows:
//   S^T [16 x 8] = K Q^T     a lane's A registers are 16 contiguous bytes of two keys:
//                            lane 4 n + c holds, of keys n and n + 8, the elements
//                            32 i + 8 c .. + 7 (the contraction index d is permuted)
//   O^T [d x 8] += V^T P^T   a lane loads 16 contiguous bytes of four value rows and pairs
//                            adjacent rows with byte permutes (rows of O^T permuted
//                            likewise); P^T is S^T's accumulator, transposed 8 x 8
// With the heads as rows instead, half of every MMA and of O's registers were empty.
//
// Precision.  An fp32 query is the exact sum of three bf16 planes, and so are the
// weights of fp32 activations: three MMAs per product, a tile's product added to O in
// fp32 (the MMA's own sums truncate: 4e-6 over 150 tiles).  bf16 activations: one MMA for
// the scores, two planes of the weights (2^-16; the second costs 1%).
//
// Measured (GB300, in a graph): 64 requests behind a 4096-token window, 64 heads of 128: 175
// us, 6.0 TB/s (fp32 183, 5.7 TB/s; heads of 64 95, 5.5 TB/s); 4 requests of up to 131072
// tokens, 32 heads: 254 us, 6.2 TB/s (fp32 276), bound by memory; 8 fp32 requests of up to
// 1028: 13.3 us, one request of 1088: 6.2 us (a chain of latencies: length, page table, keys,
// join).
//
// Masked positions are neither loaded nor multiplied: their key and value registers
// are zero, whatever the cache holds there.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "q8.h"
#include "window.h"

namespace loip {
namespace {

constexpr int kTile = 16;   // positions per warp step
constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kResident = 3;  // blocks per SM that the registers are held to

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same onto zero.
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// 8 x 8 transpose over the warp: lane 4 n + c gives elements (n, 2 c), (n, 2 c + 1) and
// gets (2 c, n), (2 c + 1, n).
__device__ __forceinline__ uint32_t transpose(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// (Not the read-only path: the kernel before this one may have written the row, see pdl_wait.)
__device__ __forceinline__ uint4 load_row(const char* p, bool live) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (live)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
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

// The tiles that a request's token sees: those of the sinks, then those of the window (which may
// touch), as a list without a gap.
struct Tiles {
    int ctx, win0, sinks;  // cached positions, first position of the window
    int sink_tiles, win_tile, n;
    __device__ __forceinline__ Tiles(const WindowArgs& a, int b) {
        ctx = max(0, min(a.ctx_lens[b], a.max_ctx));
        win0 = a.window >= ctx ? 0 : ctx - a.window;
        sinks = a.sinks;
        const int end = (ctx + kTile - 1) / kTile;
        sink_tiles = min((int)(((int64_t)a.sinks + kTile - 1) / kTile), end);
        win_tile = a.window == 0 ? end : max(win0 / kTile, sink_tiles);
        n = sink_tiles + max(0, end - win_tile);
    }
    __device__ __forceinline__ int at(int i) const { return i < sink_tiles ? i : i - sink_tiles + win_tile; }
    __device__ __forceinline__ bool seen(int j) const { return j < ctx && (j >= win0 || j < sinks); }
};

// The running softmax over a tile: a lane has the scores of positions n4 (s[0], s[1]) and n4 + 8
// (s[2], s[3]) and heads 2 c4 + {0, 1}; O is rescaled where a maximum has grown.  pb: the planes of
// P^T in the MMA's B layout; the last one is rounded (exact if it is the third).  FAST: weights below
// 2^-126 are zero.
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <bool FAST, int PV, int NO>
__device__ __forceinline__ void soften(const float (&s)[4], bool see0, bool see1, float scale, float (&m)[2], float (&l)[2],
                                       float (&o)[NO][4], uint32_t (&pb)[PV][2]) {
    auto power = [](float x) { return FAST ? ex2(x) : exp2f(x); };
    float w[4], mx[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] = see0 ? s[h] * scale : -INFINITY;
        w[2 + h] = see1 ? s[2 + h] * scale : -INFINITY;
        mx[h] = fmaxf(w[h], w[2 + h]);
#pragma unroll
        for (int x = 4; x < 32; x *= 2) mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], x));
    }
    if (__any_sync(0xffffffffu, mx[0] > m[0] || mx[1] > m[1])) {
        float alpha[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float m_new = fmaxf(m[h], mx[h]);
            alpha[h] = m[h] == -INFINITY ? 0.f : power(m[h] - m_new);
            m[h] = m_new;
            l[h] *= alpha[h];
        }
#pragma unroll
        for (int x = 0; x < NO; ++x) {
            o[x][0] *= alpha[0]; o[x][1] *= alpha[1]; o[x][2] *= alpha[0]; o[x][3] *= alpha[1];
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float base = m[h] == -INFINITY ? 0.f : m[h];  // nothing seen yet: every weight is zero
        w[h] = power(w[h] - base);
        w[2 + h] = power(w[2 + h] - base);
        l[h] += w[h] + w[2 + h];
    }
#pragma unroll
    for (int pl = 0; pl < PV; ++pl)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            pb[pl][j] = transpose(pl < PV - 1 ? peel(w[2 * j], w[2 * j + 1]) : pack(w[2 * j], w[2 * j + 1]));
}

// O^T += V^T P^T of a tile, 16 of its rows; smallest plane first.  The MMA's sums truncate, so that
// fp32 rows add a tile's product to O in fp32.
template <bool F32, int PV>
__device__ __forceinline__ void add_values(float (&o)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                           const uint32_t (&pb)[PV][2]) {
    if constexpr (F32) {
        float y[4];
        mma_first(y, a0, a1, a2, a3, pb[PV - 1][0], pb[PV - 1][1]);
#pragma unroll
        for (int pl = PV - 2; pl >= 0; --pl) mma(y, a0, a1, a2, a3, pb[pl][0], pb[pl][1]);
#pragma unroll
        for (int h = 0; h < 4; ++h) o[h] += y[h];
    } else {
#pragma unroll
        for (int pl = PV - 1; pl >= 0; --pl) mma(o, a0, a1, a2, a3, pb[pl][0], pb[pl][1]);
    }
}

// What the warps of a block share at the end: maxima, sums, and where their O lie ([8][D], a
// warp's `pitch` floats behind the last one's).
struct Shared {
    float m[kWarps][8], l[kWarps][8];
    bool last;
};

// The end of a unit of the 8-bit cache, or of a part of it: sums of the block's warps, and of the unit's
// `active` blocks in the last one to arrive.  head: the first of the group's `heads` query heads; slot:
// where this block's part goes; slot_of(x): where the unit's part x is.  (The bf16 cache's kernel has an end
// of its own: with this one 8 requests of up to 1028 took 13.6 us instead of 13.3, 4 of up to 3000 13.8
// instead of 13.5.)
template <int D, typename T, typename SlotOf>
__device__ __forceinline__ void join(const DecodeArgs& p, Shared& sh, const float* sm_o, int pitch, const float (&m)[2],
                                     float (&l)[2], int b, int head, int heads, int active, unsigned* counter, int64_t slot,
                                     SlotOf&& slot_of) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, n4 = lane / 4, c4 = lane % 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int x = 4; x < 32; x *= 2) l[h] += __shfl_xor_sync(0xffffffffu, l[h], x);
        if (n4 == 0) {
            sh.m[warp][2 * c4 + h] = m[h];
            sh.l[warp][2 * c4 + h] = l[h];
        }
    }
    __syncthreads();
    const int units = heads * (D / 4);  // four elements of a head each
    T* out = static_cast<T*>(p.a.o) + ((int64_t)b * p.a.Hq + head) * D;
    auto put = [&](int u, float4 r, float inv) {
        r.x *= inv; r.y *= inv; r.z *= inv; r.w *= inv;
        if constexpr (sizeof(T) == 4)
            reinterpret_cast<float4*>(out)[u] = r;
        else
            reinterpret_cast<uint2*>(out)[u] = make_uint2(pack(r.x, r.y), pack(r.z, r.w));
    };
    for (int u = threadIdx.x; u < units; u += kThreads) {
        const int h = u / (D / 4);
        float mt = -INFINITY, lt = 0.f;
#pragma unroll
        for (int x = 0; x < kWarps; ++x) mt = fmaxf(mt, sh.m[x][h]);
        float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int x = 0; x < kWarps; ++x) {
            const float f = sh.m[x][h] == -INFINITY ? 0.f : exp2f(sh.m[x][h] - mt);
            const float4 y = *reinterpret_cast<const float4*>(sm_o + x * pitch + h * D + 4 * (u % (D / 4)));
            lt = fmaf(f, sh.l[x][h], lt);
            r.x = fmaf(f, y.x, r.x); r.y = fmaf(f, y.y, r.y); r.z = fmaf(f, y.z, r.z); r.w = fmaf(f, y.w, r.w);
        }
        if (active == 1) {
            put(u, r, lt == 0.f ? 0.f : 1.0f / lt);
        } else {
            const int64_t at = slot * p.plan.heads + h;
            __stcg(reinterpret_cast<float4*>(p.part + at * D) + u % (D / 4), r);
            if (u % (D / 4) == 0) __stcg(p.ml + at, make_float2(mt, lt));
        }
    }
    if (active == 1) return;
    // ---- join the blocks: the last one to arrive sums all parts, in their order; the
    // counter wraps to zero with that arrival
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) sh.last = atomicInc(counter, (unsigned)active - 1u) == (unsigned)active - 1u;
    __syncthreads();
    if (!sh.last) return;
    __threadfence();
    // `N` units at a time, so many parts' loads in flight together.
    auto gather = [&](auto n_units, auto n_parts) {
        constexpr int N = decltype(n_units)::value, BATCH = decltype(n_parts)::value;
        for (int u0 = threadIdx.x; u0 < units; u0 += N * kThreads) {
            float mt[N], lt[N];
            float4 r[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                mt[k] = -INFINITY;
                lt[k] = 0.f;
                r[k] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
            for (int x0 = 0; x0 < active; x0 += BATCH) {
                float2 ml[N][BATCH];
                float4 y[N][BATCH];
#pragma unroll
                for (int x = 0; x < BATCH; ++x) {
                    const int64_t first = slot_of(min(x0 + x, active - 1)) * p.plan.heads;
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const int u = min(u0 + k * kThreads, units - 1);
                        const int64_t at = first + u / (D / 4);
                        ml[k][x] = __ldcg(p.ml + at);
                        y[k][x] = __ldcg(reinterpret_cast<const float4*>(p.part + at * D) + u % (D / 4));
                    }
                }
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    float mb = mt[k];
#pragma unroll
                    for (int x = 0; x < BATCH; ++x) mb = fmaxf(mb, ml[k][x].x);
                    const float keep = mt[k] == -INFINITY ? 0.f : exp2f(mt[k] - mb);
                    mt[k] = mb;
                    lt[k] *= keep;
                    r[k].x *= keep; r[k].y *= keep; r[k].z *= keep; r[k].w *= keep;
#pragma unroll
                    for (int x = 0; x < BATCH; ++x) {
                        const float f = x0 + x < active && ml[k][x].x != -INFINITY ? exp2f(ml[k][x].x - mt[k]) : 0.f;
                        lt[k] = fmaf(f, ml[k][x].y, lt[k]);
                        r[k].x = fmaf(f, y[k][x].x, r[k].x); r[k].y = fmaf(f, y[k][x].y, r[k].y);
                        r[k].z = fmaf(f, y[k][x].z, r[k].z); r[k].w = fmaf(f, y[k][x].w, r[k].w);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (u0 + k * kThreads < units) put(u0 + k * kThreads, r[k], lt[k] == 0.f ? 0.f : 1.0f / lt[k]);
        }
    };
    using std::integral_constant;
    if (units > kThreads)
        gather(integral_constant<int, 2>{}, integral_constant<int, 9>{});
    else
        gather(integral_constant<int, 1>{}, integral_constant<int, 12>{});
}

// Queries into shared memory, the same for every warp: bf16 planes in the MMA's B layout, of which a
// lane holds eight elements of head n4 in piece x, `step` elements from one piece to the next.
// Columns past the group's heads are zero.
template <int NQ, int PL, typename T>
__device__ __forceinline__ void load_queries(uint4 (&sm_q)[NQ][PL][32], const T* q, int step, bool live) {
    const int lane = threadIdx.x % 32;
    for (int x = threadIdx.x / 32; x < NQ; x += kWarps) {
        if constexpr (PL == 3) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
            if (live) {
                const float4 y = *reinterpret_cast<const float4*>(q + step * x);
                const float4 z = *reinterpret_cast<const float4*>(q + step * x + 4);
                v[0] = y.x; v[1] = y.y; v[2] = y.z; v[3] = y.w; v[4] = z.x; v[5] = z.y; v[6] = z.z; v[7] = z.w;
            }
#pragma unroll
            for (int pl = 0; pl < 3; ++pl) {
                uint32_t u[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    u[e] = pl < 2 ? peel(v[2 * e], v[2 * e + 1]) : pack(v[2 * e], v[2 * e + 1]);
                sm_q[x][pl][lane] = make_uint4(u[0], u[1], u[2], u[3]);
            }
        } else {
            sm_q[x][0][lane] = live ? *reinterpret_cast<const uint4*>(q + step * x) : make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

template <int D, typename T>
__global__ void __launch_bounds__(kThreads, kResident) window_decode_kernel(const __grid_constant__ DecodeArgs p) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NQ = D / 32;  // 16-byte pieces of a key per lane
    constexpr int NV = D / 64;  // 16-byte pieces of a value row per lane
    constexpr int PV = F32 ? 3 : 2;  // planes of the weights
    __shared__ __align__(16) float sm_o[kWarps][8][D];
    __shared__ Shared sh;
    __shared__ uint4 sm_q[NQ][F32 ? 3 : 1][32];
    const WindowArgs& a = p.a;
    pdl_wait();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, n4 = lane / 4, c4 = lane % 4;
    const int b = blockIdx.x / p.plan.splits, split = blockIdx.x % p.plan.splits;
    const int kvh = blockIdx.y / p.plan.groups, G = a.Hq / a.Hkv;
    const int head0 = (blockIdx.y % p.plan.groups) * p.plan.heads;          // of the kv head's G
    const int heads = min(p.plan.heads, G - head0);
    const Tiles seen(a, b);
    const int active = max(1, (seen.n + p.plan.chunk - 1) / p.plan.chunk);  // blocks with work
    if (split >= active) return;
    const int last = min(seen.n, (split + 1) * p.plan.chunk);

    load_queries(sm_q, static_cast<const T*>(a.q) + ((int64_t)b * a.Hq + kvh * G + head0 + n4) * D + 8 * c4, 32, n4 < heads);

    const char* layer = a.kv.base + (uint64_t)a.kv.layer * a.kv.layer_page_bytes;
    const int64_t* table = a.kv.page_offsets + (int64_t)b * a.kv.max_pages;
    // the tile's first key of this kv head
    auto key_at = [&](int t) {
        return layer + table[t / (kPageTokens / kTile)] +
               (uint32_t)((kvh * kPageTokens + (t % (kPageTokens / kTile)) * kTile) * D * 2);
    };
    const uint32_t v_off = (uint32_t)(a.Hkv * kPageTokens) * D * 2;

    float o[4 * NV][4];  // rows 64 x + 8 n4 + 2 e (+ 1) of O^T, heads 2 c4 and 2 c4 + 1
#pragma unroll
    for (int i = 0; i < 4 * NV; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};  // of heads 2 c4 and 2 c4 + 1
    const float scale = 1.44269504088896f / sqrtf((float)D);  // scores in units of log 2

    uint4 k[2][NQ], v[4][NV];
    auto load_k = [&](int t, const char* at) {  // keys n4 and n4 + 8
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bool live = seen.seen(t * kTile + 8 * j + n4);
#pragma unroll
            for (int x = 0; x < NQ; ++x) k[j][x] = load_row(at + ((8 * j + n4) * D + 32 * x + 8 * c4) * 2, live);
        }
    };
    int i = split * p.plan.chunk + warp;
    const char* at = nullptr;
    if (i < last) {
        at = key_at(seen.at(i));
        load_k(seen.at(i), at);
    }
    __syncthreads();  // the queries
    for (; i < last; i += kWarps) {
        const int t = seen.at(i);
        const char* at_next = i + kWarps < last ? key_at(seen.at(i + kWarps)) : nullptr;
#pragma unroll
        for (int r = 0; r < 4; ++r) {  // value rows 2 c4, 2 c4 + 1, 2 c4 + 8, 2 c4 + 9
            const int row = 2 * c4 + (r & 1) + 8 * (r >> 1);
            const bool live = seen.seen(t * kTile + row);
#pragma unroll
            for (int x = 0; x < NV; ++x) v[r][x] = load_row(at + v_off + (row * D + 64 * x + 8 * n4) * 2, live);
        }
        // ---- scores, in independent sums (a chain of MMAs waits for each result)
        float s[4];
        {
            constexpr int PL = F32 ? 3 : 1;
            float z[PL][2][4];
#pragma unroll
            for (int pl = 0; pl < PL; ++pl)
#pragma unroll
                for (int h = 0; h < 2; ++h) z[pl][h][0] = z[pl][h][1] = z[pl][h][2] = z[pl][h][3] = 0.f;
#pragma unroll
            for (int x = 0; x < NQ; ++x)
#pragma unroll
                for (int pl = 0; pl < PL; ++pl) {
                    const uint4 q = sm_q[x][pl][lane];
                    mma(z[pl][0], k[0][x].x, k[1][x].x, k[0][x].y, k[1][x].y, q.x, q.y);
                    mma(z[pl][1], k[0][x].z, k[1][x].z, k[0][x].w, k[1][x].w, q.z, q.w);
                }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[e] = z[0][0][e] + z[0][1][e];
                if constexpr (F32) s[e] += (z[1][0][e] + z[1][1][e]) + (z[2][0][e] + z[2][1][e]);
            }
        }
        if (at_next) load_k(seen.at(i + kWarps), at_next);
        // ---- softmax
        uint32_t pb[PV][2];
        soften<false>(s, seen.seen(t * kTile + n4), seen.seen(t * kTile + 8 + n4), scale, m, l, o, pb);
        // ---- values
#pragma unroll
        for (int x = 0; x < NV; ++x) {
            const uint32_t r0[4] = {v[0][x].x, v[0][x].y, v[0][x].z, v[0][x].w};
            const uint32_t r1[4] = {v[1][x].x, v[1][x].y, v[1][x].z, v[1][x].w};
            const uint32_t r2[4] = {v[2][x].x, v[2][x].y, v[2][x].z, v[2][x].w};
            const uint32_t r3[4] = {v[3][x].x, v[3][x].y, v[3][x].z, v[3][x].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t a0 = __byte_perm(r0[e], r1[e], 0x5410u), a1 = __byte_perm(r0[e], r1[e], 0x7632u);
                const uint32_t a2 = __byte_perm(r2[e], r3[e], 0x5410u), a3 = __byte_perm(r2[e], r3[e], 0x7632u);
                add_values<F32>(o[4 * x + e], a0, a1, a2, a3, pb);
            }
        }
        at = at_next;
    }

    // The next launch comes at this one's end.  Where it may come from the start, or from here, its waiting
    // blocks slow this one's (graph and stream, us, from the start, from here, and so: one request of 1088
    // 7.7 8.3, 6.5 7.4, 6.2 6.2; 16 of up to 2000, 20/4 heads of 64, 12.0 12.3, 11.8 12.0, 11.0 11.1; in turn
    // with an append all alike).
    // ---- join the warps: heads 2 c4 + h, elements 64 x + 8 n4 .. + 7
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int x = 4; x < 32; x *= 2) l[h] += __shfl_xor_sync(0xffffffffu, l[h], x);
        if (n4 == 0) {
            sh.m[warp][2 * c4 + h] = m[h];
            sh.l[warp][2 * c4 + h] = l[h];
        }
#pragma unroll
        for (int x = 0; x < NV; ++x)
#pragma unroll
            for (int e = 0; e < 4; e += 2)
                *reinterpret_cast<float4*>(&sm_o[warp][2 * c4 + h][64 * x + 8 * n4 + 2 * e]) = make_float4(
                    o[4 * x + e][h], o[4 * x + e][2 + h], o[4 * x + e + 1][h], o[4 * x + e + 1][2 + h]);
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
        for (int x = 0; x < kWarps; ++x) mt = fmaxf(mt, sh.m[x][h]);
        float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int x = 0; x < kWarps; ++x) {
            const float f = sh.m[x][h] == -INFINITY ? 0.f : exp2f(sh.m[x][h] - mt);
            const float4 y = *reinterpret_cast<const float4*>(&sm_o[x][h][4 * (u % (D / 4))]);
            lt = fmaf(f, sh.l[x][h], lt);
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
    if (threadIdx.x == 0) sh.last = atomicInc(p.counters + unit, (unsigned)active - 1u) == (unsigned)active - 1u;
    __syncthreads();
    if (!sh.last) return;
    __threadfence();
    for (int u = threadIdx.x; u < units; u += kThreads) {
        const int h = u / (D / 4);
        const int64_t first = unit * p.plan.splits * p.plan.heads + h;
        float mt = -INFINITY, lt = 0.f;
        float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int BATCH = 12;  // parts whose loads are in flight together
        for (int x0 = 0; x0 < active; x0 += BATCH) {
            float2 ml[BATCH];
            float4 y[BATCH];
#pragma unroll
            for (int x = 0; x < BATCH; ++x) {
                const int64_t at = first + (int64_t)min(x0 + x, active - 1) * p.plan.heads;
                ml[x] = __ldcg(p.ml + at);
                y[x] = __ldcg(reinterpret_cast<const float4*>(p.part + at * D) + u % (D / 4));
            }
            float mb = mt;
#pragma unroll
            for (int x = 0; x < BATCH; ++x) mb = fmaxf(mb, ml[x].x);
            const float keep = mt == -INFINITY ? 0.f : exp2f(mt - mb);
            mt = mb;
            lt *= keep;
            r.x *= keep; r.y *= keep; r.z *= keep; r.w *= keep;
#pragma unroll
            for (int x = 0; x < BATCH; ++x) {
                const float f = x0 + x < active && ml[x].x != -INFINITY ? exp2f(ml[x].x - mt) : 0.f;
                lt = fmaf(f, ml[x].y, lt);
                r.x = fmaf(f, y[x].x, r.x); r.y = fmaf(f, y[x].y, r.y);
                r.z = fmaf(f, y[x].z, r.z); r.w = fmaf(f, y[x].w, r.w);
            }
        }
        put(u, r, lt == 0.f ? 0.f : 1.0f / lt);
    }
}

// ---------------------------------------------------------------------------
// The 8-bit cache.
//
// 33 d bytes a tile instead of 64 d, so that the conversion to bf16 is what the memory's rate has to
// hide: three instructions for two elements, four where exponents are extreme (q8.h), some 500 a tile of
// d = 128 in all, where memory leaves a scheduler 730 issue slots a tile.  A tile is one contiguous
// granule: a warp copies its own tiles, kStages - 1 ahead, whole (the positions of a granule that are
// not seen lie in a page of the request all the same), and reads the MMAs' fragments from
// shared memory, 16 bytes a lane without bank conflicts:
//   S^T = K Q^T     lane (n4, c4) has, of keys n4 and n4 + 8, the d / 4 elements from d / 4 c4,
//                   which are of one block; four codes are a lane's A registers of one MMA
//   O^T += V^T P^T  the d / 8 elements from d / 8 n4 of values 2 c4 + {0, 1, 8, 9}; adjacent
//                   tokens are paired by the byte permute that spreads the codes
// Positions that are not seen have a scale of zero, so that whatever the cache holds there is zero.
//
// Where the work is.  A step is four tiles of a unit (request, kv head and group of heads), one a
// warp.  The blocks share the steps of all units equally, as one list in their order, whatever
// the lengths are: each adds them up, finds its share and goes through it unit by unit.  A unit that
// begins in one block and ends in a later one is joined by the last of its blocks to arrive.  (With a
// share cut per request, as above, 5 of 60001 to 131072 tokens took 323 us, 96 behind a window 204.)
//
// Measured (in a graph): 5 bf16 requests of 60001 to 131072 tokens, 32/8 heads of 128, 180 us, 5.6 TB/s;
// 96 of 1000 to 32768 behind 4096 + 64, 64/8 heads, 152 us, 5.3 TB/s (fp32 175); 8 fp32 ones of 128 to 4352
// 23.5 us; one of 640 7.2 us.  Bound by memory and by issue together (dram 67%, issue 55%, integer pipe 51%).
// The older blocks of an SM are done first, after 80% of the time; larger shares for them (70:67:62:57)
// evened that out and the call took as long.  Nor did a smaller share and the rest in chunks as blocks get
// to them (206 us for the five): each chunk's end costs a join and a pipeline that fills again.
// ---------------------------------------------------------------------------
constexpr int kStages = 3;
constexpr float kUnit8 = 0x1p64f;  // of elements as shifted_of makes them
static_assert(q8::kShift == 64, "");
constexpr int kResident8 = 4;  // blocks per SM (96 requests: 152 us; three with four stages 159, five with two 154)
constexpr int kPlaces8 = 152 * kResident8;

__device__ __forceinline__ void copy16(uint32_t to, const char* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

template <int D, typename T>
__global__ void __launch_bounds__(kThreads, kResident8) window_decode_q8_kernel(const __grid_constant__ DecodeArgs p) {
    using Gr = q8::Granule<D>;
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NK = D / 64;       // 16-byte pieces of a key per lane
    constexpr int NW = D / 32;       // words of four codes of a value row per lane
    constexpr int PL = F32 ? 3 : 1;  // planes of the queries
    constexpr int PV = F32 ? 3 : 2;  // planes of the weights
    extern __shared__ __align__(16) uint8_t ring[];  // [warp][stage][granule]; at a unit's end [warp][8][D] floats
    static_assert(8 * D * sizeof(float) <= kStages * Gr::BYTES, "the join goes through a warp's own part");
    __shared__ Shared sh;
    __shared__ uint4 sm_q[D / 32][PL][32];
    const WindowArgs& a = p.a;
    pdl_wait();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, n4 = lane / 4, c4 = lane % 4;
    const int units = a.Hkv * p.plan.groups, G = a.Hq / a.Hkv;  // units of a request
    // ---- this block's share
    auto steps_of = [&](int b) { return b < a.rows ? max(1, (Tiles(a, b).n + kWarps - 1) / kWarps) : 0; };
    const int first32 = steps_of(lane);
    int64_t total = first32;
    for (int b = 32 + lane; b < a.rows; b += 32) total += steps_of(b);
#pragma unroll
    for (int x = 16; x; x /= 2) total += __shfl_xor_sync(0xffffffffu, total, x);
    total *= units;
    const int64_t share = (total + gridDim.x - 1) / gridDim.x;
    int64_t at = share * blockIdx.x;
    const int64_t end = min(at + share, total);
    if (at >= end) return;
    int b = 0, unit, step;  // where the share begins
    int64_t unit_at;        // first step of that unit in the list
    {
        int64_t before = 0;
        for (;; b += 32) {
            const int mine = b == 0 ? first32 : steps_of(b + lane);
            int64_t sum = mine;
#pragma unroll
            for (int x = 1; x < 32; x *= 2) {
                const int64_t y = __shfl_up_sync(0xffffffffu, sum, x);
                if (lane >= x) sum += y;
            }
            const unsigned past = __ballot_sync(0xffffffffu, (before + sum) * units > at);
            if (past) {  // (at < total: in some round)
                const int src = __ffs(past) - 1;
                before += __shfl_sync(0xffffffffu, sum - mine, src);
                const int steps = __shfl_sync(0xffffffffu, mine, src);
                b += src;
                unit = (int)((at - before * units) / steps);
                unit_at = before * units + (int64_t)unit * steps;
                step = (int)(at - unit_at);
                break;
            }
            before += __shfl_sync(0xffffffffu, sum, 31);
        }
    }
    uint8_t* const mine = ring + warp * kStages * Gr::BYTES;
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(mine) + lane * 16;
    auto copy = [&](const char* from, int stage) {
        constexpr int PIECES = Gr::BYTES / 16;
#pragma unroll
        for (int x = 0; x < PIECES; x += 32)
            if (x + 32 <= PIECES || lane < PIECES - x) copy16(to + stage * Gr::BYTES + x * 16, from + x * 16);
    };
    const float scale = 1.44269504088896f / sqrtf((float)D);  // scores in units of log 2
    const char* layer = a.kv.base + (uint64_t)a.kv.layer * a.kv.layer_page_bytes;

#pragma unroll 1
    for (;;) {
        const Tiles seen(a, b);
        const int steps = max(1, (seen.n + kWarps - 1) / kWarps);
        const int kvh = unit / p.plan.groups, head0 = unit % p.plan.groups * p.plan.heads;  // of the kv head's G
        const int heads = min(p.plan.heads, G - head0);
        const int last = min((int64_t)seen.n, (end - unit_at) * kWarps);  // tiles
        const char* head = layer + (int64_t)kvh * 4 * Gr::BYTES + lane * 16;
        const int64_t* table = a.kv.page_offsets + (int64_t)b * a.kv.max_pages;
        auto granule = [&](int i) {  // of the list's tile i
            const int t = seen.at(i);
            return head + table[t / 4] + t % 4 * Gr::BYTES;
        };
        int i = step * kWarps + warp;
        {
            const char* from[kStages - 1];
#pragma unroll
            for (int x = 0; x < kStages - 1; ++x) from[x] = i + x * kWarps < last ? granule(i + x * kWarps) : nullptr;
#pragma unroll
            for (int x = 0; x < kStages - 1; ++x) {
                if (from[x]) copy(from[x], x);
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
        }
        load_queries(sm_q, static_cast<const T*>(a.q) + ((int64_t)b * a.Hq + kvh * G + head0 + n4) * D + D / 4 * c4, 8,
                     n4 < heads);
        const char* next = i + (kStages - 1) * kWarps < last ? granule(i + (kStages - 1) * kWarps) : nullptr;

        float o[D / 16][4];  // rows d / 8 n4 + 2 e (+ 1) of O^T, heads 2 c4 and 2 c4 + 1
#pragma unroll
        for (int e = 0; e < D / 16; ++e) o[e][0] = o[e][1] = o[e][2] = o[e][3] = 0.f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};  // of heads 2 c4 and 2 c4 + 1
        bool exact = false;  // O in units of its own, and not of kUnit8
        __syncthreads();  // the queries
#pragma unroll 1
        for (int stage = 0; i < last; i += kWarps, stage = stage + 1 == kStages ? 0 : stage + 1) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
            __syncwarp();  // every lane's part of the tile is here, and the tile before is read
            if (next) copy(next, stage == 0 ? kStages - 1 : stage - 1);
            asm volatile("cp.async.commit_group;" ::: "memory");
            const int ahead = i + kStages * kWarps;
            next = ahead < last ? granule(ahead) : nullptr;
            const uint8_t* g = mine + stage * Gr::BYTES;
            const int j0 = seen.at(i) * kTile;
            const bool all = j0 + kTile <= seen.ctx && (j0 >= seen.win0 || j0 + kTile <= seen.sinks);
            const bool see0 = all || seen.seen(j0 + n4), see1 = all || seen.seen(j0 + 8 + n4);
            // exponents: of keys n4 and n4 + 8, of values 2 c4 and 2 c4 + 1, and eight further on
            uint32_t ek, ev[2];
            {
                uint32_t E[3][2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    E[0][r] = g[Gr::exponents(0, 8 * r + n4) + c4 * (D / 64) / 2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) E[1 + j][r] = g[Gr::exponents(1, 2 * c4 + r + 8 * j) + n4 / 2 * (D / 64) / 2];
                }
                ek = E[0][0] + E[0][1] * 65536u;
                ev[0] = E[1][0] + E[1][1] * 65536u;
                ev[1] = E[2][0] + E[2][1] * 65536u;
            }
            uint32_t keep[2] = {~0u, ~0u};  // the values that are seen
            if (!all) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    keep[j] = (seen.seen(j0 + 2 * c4 + 8 * j) ? 0xffffu : 0u) |
                              (seen.seen(j0 + 2 * c4 + 1 + 8 * j) ? 0xffff0000u : 0u);
                    ev[j] = (ev[j] & keep[j]) | (0x00800080u & ~keep[j]);
                }
                const uint32_t mask = (see0 ? 0xffffu : 0u) | (see1 ? 0xffff0000u : 0u);
                ek = (ek & mask) | (0x00800080u & ~mask);
            }
            // An exponent of 96 to 159 is one whose shift is a test of bits.  A tile with another one takes O to
            // its own units, and from then on elements are made by two products.
            const uint32_t off = (ek - 0x00600060u) | (ev[0] - 0x00600060u) | (ev[1] - 0x00600060u);
            if (!exact && __any_sync(0xffffffffu, off & 0xffc0ffc0u)) {
                exact = true;
#pragma unroll
                for (int e = 0; e < D / 16; ++e)
#pragma unroll
                    for (int h = 0; h < 4; ++h) o[e][h] *= kUnit8;
            }
            auto tile = [&](auto exactly) {
                constexpr bool EXACT = decltype(exactly)::value;
                auto pair = [](uint32_t twice, uint32_t sc) {
                    return EXACT ? q8::pair_of(twice, sc) : q8::shifted_of(twice, sc);
                };
                // ---- scores, in independent sums (a chain of MMAs waits for each result)
                float s[4];
                {
                    uint32_t k[2][4 * NK];
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int x = 0; x < NK; ++x) {
                            const uint4 u = *reinterpret_cast<const uint4*>(g + Gr::piece(0, 8 * j + n4, NK * c4 + x));
                            k[j][4 * x] = u.x; k[j][4 * x + 1] = u.y; k[j][4 * x + 2] = u.z; k[j][4 * x + 3] = u.w;
                        }
                    const uint32_t both = EXACT ? q8::scale2(ek) : q8::shifted2(ek);
                    const uint32_t sc[2] = {see0 ? __byte_perm(both, 0u, 0x1010u) : 0u,
                                            see1 ? __byte_perm(both, 0u, 0x3232u) : 0u};
                    constexpr int SUMS = F32 ? 1 : 2;
                    float z[PL][SUMS][4];
#pragma unroll
                    for (int x = 0; x < 4 * NK; ++x) {
                        uint32_t A[2][2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            A[j][0] = pair(__byte_perm(k[j][x], 0u, 0x1100u), sc[j]);
                            A[j][1] = pair(__byte_perm(k[j][x], 0u, 0x3322u), sc[j]);
                        }
#pragma unroll
                        for (int pl = 0; pl < PL; ++pl) {
                            const uint4 q = sm_q[x / 2][pl][lane];
                            if (x < SUMS)
                                mma_first(z[pl][x], A[0][0], A[1][0], A[0][1], A[1][1], x % 2 ? q.z : q.x, x % 2 ? q.w : q.y);
                            else
                                mma(z[pl][x % SUMS], A[0][0], A[1][0], A[0][1], A[1][1], x % 2 ? q.z : q.x, x % 2 ? q.w : q.y);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (F32)
                            s[e] = z[0][0][e] + (z[1][0][e] + z[2][0][e]);
                        else
                            s[e] = z[0][0][e] + z[0][1][e];
                    }
                }
                uint32_t pb[PV][2];
                soften<true>(s, see0, see1, EXACT ? scale : scale * kUnit8, m, l, o, pb);
                // ---- values: rows 2 c4, 2 c4 + 1, 2 c4 + 8, 2 c4 + 9
                uint32_t sc[2];
                uint32_t v[4][NW];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint8_t* from = g + Gr::piece(1, 2 * c4 + r + 8 * j, D == 128 ? n4 : n4 / 2);
                        if constexpr (D == 128) {
                            const uint4 u = *reinterpret_cast<const uint4*>(from);
                            v[2 * j + r][0] = u.x; v[2 * j + r][1] = u.y; v[2 * j + r][2] = u.z; v[2 * j + r][3] = u.w;
                        } else {
                            const uint2 u = *reinterpret_cast<const uint2*>(from + n4 % 2 * 8);
                            v[2 * j + r][0] = u.x; v[2 * j + r][1] = u.y;
                        }
                    }
                    sc[j] = (EXACT ? q8::scale2(ev[j]) : q8::shifted2(ev[j])) & keep[j];
                }
#pragma unroll
                for (int e = 0; e < D / 16; ++e) {
                    uint32_t A[2][2];
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            A[j][r] = pair(
                                __byte_perm(v[2 * j][e / 2], v[2 * j + 1][e / 2], 0x4400u + 0x1111u * (e % 2 * 2 + r)), sc[j]);
                    add_values<F32>(o[e], A[0][0], A[0][1], A[1][0], A[1][1], pb);
                }
            };
            if (exact)
                tile(std::true_type{});
            else
                tile(std::false_type{});
        }
        pdl_trigger();  // (from the start one request of 640 took 9.2 us a call, so 7.2)
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();
        float* sm_o = reinterpret_cast<float*>(mine);
        const float unit_o = exact ? 1.f : kUnit8;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < D / 16; e += 2)
                *reinterpret_cast<float4*>(sm_o + (2 * c4 + h) * D + D / 8 * n4 + 2 * e) =
                    make_float4(o[e][h] * unit_o, o[e][2 + h] * unit_o, o[e + 1][h] * unit_o, o[e + 1][2 + h] * unit_o);
        // A block's part of a unit that began in an earlier block is its first, of one that ends in a
        // later block its second; a unit's counter is that of the block where it begins.
        const int64_t from = unit_at / share, active = (unit_at + steps - 1) / share - from + 1;
        join<D, T>(p, sh, reinterpret_cast<const float*>(ring), kStages * Gr::BYTES / 4, m, l, b, kvh * G + head0, heads,
                   (int)active, p.counters + from, 2 * (int64_t)blockIdx.x + (from == blockIdx.x),
                   [&](int x) { return 2 * (from + x) + (x == 0); });
        unit_at += steps;
        if (unit_at >= end) return;
        step = 0;
        if (++unit == units) {
            unit = 0;
            ++b;
        }
        __syncthreads();  // the join has read the ring and the queries are free
    }
}

constexpr int kPlaces = 152 * kResident;
constexpr int kMostTiles = 96;    // per block, without whole waves
constexpr int kWaveTiles = 384;   // per block with them, unless
constexpr int kWaveBlocks = 76;   // a request alone has that many blocks

int64_t visible_tiles(int window, int sinks, int max_ctx) {
    return std::min<int64_t>(((int64_t)max_ctx + kTile - 1) / kTile, ((int64_t)window + kTile - 1) / kTile + 1 +
                                                                         ((int64_t)sinks + kTile - 1) / kTile);
}

// Blocks of `chunk` tiles.  Where the (request, group) units, each split alike, fill four
// fifths of the places that the card has for blocks, or more, all blocks run at once: whole
// waves, few joins, down to a tile per warp (4 requests of up to 131072 tokens: 14 parts
// each, 251 us, 267 us with blocks of 48 tiles; 8 requests of up to 1028: 12.9 us, 20.7 us
// with blocks of 4; one of 1088 in 17 parts: 6.2 us).  But the lengths are on the device, and what is one wave of equal requests is a
// few blocks at work when one is long and the others are short.  So a wave's blocks have at
// most 384 tiles, or a request alone has blocks for half of the SMs (48 requests, one of
// 131072 tokens among 1000: 139 us, 2150 us unsplit; 8: 102 and 371 us; the price: 8 of 65536
// each 333 us, 312 in one wave, 57 of 16384 565 and 546 us; 48 of 4160 stay one wave, 123 us,
// 135 us with blocks of 88).
// Otherwise a unit's tiles are cut into equal blocks of at most 96 (32 requests of 4160
// positions: three blocks of 88 tiles, 87 us; one of 264, 102 us; five of 64 and a remainder,
// 93 us).
Plan make_plan(int B, int Hq, int Hkv, int window, int sinks, int max_ctx) {
    Plan p{};
    const int G = Hq / Hkv;
    p.groups = (G + 7) / 8;
    p.heads = (G + p.groups - 1) / p.groups;
    const int64_t tiles = visible_tiles(window, sinks, max_ctx), units = (int64_t)B * Hkv * p.groups;
    auto equal = [&](int64_t parts) { return ((tiles + parts - 1) / parts + kWarps - 1) / kWarps * kWarps; };
    int64_t chunk = equal((tiles + kMostTiles - 1) / kMostTiles);
    const int64_t splits = kPlaces / std::max<int64_t>(units, 1);
    if (5 * units * splits >= 4 * kPlaces &&
        (equal(splits) <= kWaveTiles || splits * Hkv * p.groups >= kWaveBlocks)) {
        chunk = equal(splits);
    } else if (units > kMaxCounters) {  // no counter for each: unsplit, and far more units than places
        chunk = tiles;
    }
    p.chunk = (int)std::max<int64_t>(chunk, 1);
    p.splits = (int)std::max<int64_t>((tiles + p.chunk - 1) / p.chunk, 1);
    return p;
}

// Blocks of a call over the 8-bit cache: no more than it has steps.
int blocks8(int B, int Hkv, int groups, int window, int sinks, int max_ctx) {
    const int64_t units = (int64_t)B * Hkv * groups;
    if (units >= kPlaces8) return kPlaces8;
    return (int)std::min<int64_t>(kPlaces8, units * ((visible_tiles(window, sinks, max_ctx) + kWarps - 1) / kWarps));
}

template <int D, typename T>
cudaError_t launch_t(const DecodeArgs& p, bool q8, cudaStream_t st) {
    const dim3 grid((unsigned)p.a.rows * p.plan.splits, p.a.Hkv * p.plan.groups);
    if (!q8) return launch_pdl(window_decode_kernel<D, T>, grid, kThreads, 0, st, p);
    constexpr int BYTES = kWarps * kStages * q8::Granule<D>::BYTES;
    const dim3 grid8(blocks8(p.a.rows, p.a.Hkv, p.plan.groups, p.a.window, p.a.sinks, p.a.max_ctx));
    static std::atomic<uint64_t> ready{0};
    const cudaError_t e = raise_smem_limit(window_decode_q8_kernel<D, T>, BYTES, ready);
    return e != cudaSuccess ? e : launch_pdl(window_decode_q8_kernel<D, T>, grid8, kThreads, BYTES, st, p);
}

cudaError_t launch_any(const WindowArgs& a, bool f32, bool q8, cudaStream_t st) {
    DecodeArgs p{};
    p.a = a;
    p.plan = make_plan(a.rows, a.Hq, a.Hkv, a.window, a.sinks, a.max_ctx);
    if ((int64_t)a.rows * p.plan.splits > 0x7fffffff) return cudaErrorInvalidValue;
    const int64_t parts = q8 ? 2 * blocks8(a.rows, a.Hkv, p.plan.groups, a.window, a.sinks, a.max_ctx)
                             : (int64_t)a.rows * a.Hkv * p.plan.groups * p.plan.splits;
    p.counters = static_cast<unsigned*>(a.scratch);
    p.part = reinterpret_cast<float*>(p.counters + kMaxCounters);
    p.ml = reinterpret_cast<float2*>(p.part + parts * p.plan.heads * a.d);
    if (a.d == 128) return f32 ? launch_t<128, float>(p, q8, st) : launch_t<128, __nv_bfloat16>(p, q8, st);
    return f32 ? launch_t<64, float>(p, q8, st) : launch_t<64, __nv_bfloat16>(p, q8, st);
}

}  // namespace

// Enough for every smaller call too: parts of the plans of up to B requests and of this visible
// length or less.  Blocks in one wave are at most the card's places, and a warp has a tile at
// least; otherwise parts are equal, and as many as blocks of kMostTiles.
uint64_t window_decode_scratch(int B, int Hq, int Hkv, int d, int window, int sinks, int max_ctx) {
    const Plan p = make_plan(B, Hq, Hkv, window, sinks, max_ctx);
    const int64_t tiles = visible_tiles(window, sinks, max_ctx), units = (int64_t)B * Hkv * p.groups;
    int64_t parts = 0;
    if (tiles > kWarps) parts = std::min<int64_t>(kPlaces, units * ((tiles + kWarps - 1) / kWarps));
    if (tiles > kMostTiles)
        parts = std::max(parts, std::min<int64_t>(units, kMaxCounters) * ((tiles + kMostTiles - 1) / kMostTiles));
    const uint64_t n = kCounterBytes + (uint64_t)parts * p.heads * (d + 2) * sizeof(float);
    return (n + 15) / 16 * 16;
}

cudaError_t launch_window_decode(const WindowArgs& a, bool f32, cudaStream_t st) { return launch_any(a, f32, false, st); }

// Two parts for each block; more blocks for more or longer requests.
uint64_t window_decode_q8_scratch(int B, int Hq, int Hkv, int d, int window, int sinks, int max_ctx) {
    const Plan p = make_plan(B, Hq, Hkv, window, sinks, max_ctx);
    const uint64_t blocks = blocks8(B, Hkv, p.groups, window, sinks, max_ctx);
    return (kCounterBytes + blocks * 2 * p.heads * (d + 2) * sizeof(float) + 15) / 16 * 16;
}
cudaError_t launch_window_decode_q8(const WindowArgs& a, bool f32, cudaStream_t st) { return launch_any(a, f32, true, st); }

}  // namespace loip
