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
// tokens, 32 heads: 251 us, 6.2 TB/s (fp32 276), bound by memory; 8 fp32 requests of up to
// 1028: 13.1 us, one request of 1088: 7.6 us (a chain of latencies: length, page table, keys,
// join).
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
constexpr int kResident = 3;  // blocks per SM that the registers are held to

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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

template <int D, typename T>
__global__ void __launch_bounds__(kThreads, kResident) window_decode_kernel(const __grid_constant__ DecodeArgs p) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NQ = D / 32;  // 16-byte pieces of a key per lane
    constexpr int NV = D / 64;  // 16-byte pieces of a value row per lane
    constexpr int PV = F32 ? 3 : 2;  // planes of the weights
    __shared__ __align__(16) float sm_o[kWarps][8][D];
    __shared__ float sm_m[kWarps][8], sm_l[kWarps][8];
    __shared__ bool sm_last;
    __shared__ uint4 sm_q[NQ][F32 ? 3 : 1][32];
    const WindowArgs& a = p.a;
    pdl_trigger();
    pdl_wait();
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

    // queries: bf16 planes in the B layout (a lane: head n4, elements 32 x + 8 c4 ..), columns past
    // the group's heads zero; the same for every warp, in shared memory
    {
        const T* q = static_cast<const T*>(a.q) + ((int64_t)b * a.Hq + kvh * G + head0 + n4) * D + 8 * c4;
        for (int x = warp; x < NQ; x += kWarps) {
            if constexpr (F32) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.f;
                if (n4 < heads) {
                    const float4 y = *reinterpret_cast<const float4*>(q + 32 * x);
                    const float4 z = *reinterpret_cast<const float4*>(q + 32 * x + 4);
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
                sm_q[x][0][lane] = n4 < heads ? *reinterpret_cast<const uint4*>(q + 32 * x) : make_uint4(0u, 0u, 0u, 0u);
            }
        }
    }

    const char* layer = a.kv.base + (uint64_t)a.kv.layer * a.kv.layer_page_bytes;
    const int64_t* table = a.kv.page_offsets + (int64_t)b * a.kv.max_pages;
    auto tile_at = [&](int i) { return i < sink_tiles ? i : i - sink_tiles + win_tile; };
    auto seen = [&](int j) { return j < ctx && (j >= win0 || j < a.sinks); };
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
            const bool live = seen(t * kTile + 8 * j + n4);
#pragma unroll
            for (int x = 0; x < NQ; ++x) k[j][x] = load_row(at + ((8 * j + n4) * D + 32 * x + 8 * c4) * 2, live);
        }
    };
    int i = split * p.plan.chunk + warp;
    const char* at = nullptr;
    if (i < last) {
        at = key_at(tile_at(i));
        load_k(tile_at(i), at);
    }
    __syncthreads();  // the queries
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
        if (at_next) load_k(tile_at(i + kWarps), at_next);
        // ---- softmax: this lane has positions n4 (s[0], s[1]) and n4 + 8 (s[2], s[3]), heads 2 c4 + {0, 1}
        const bool see0 = seen(t * kTile + n4), see1 = seen(t * kTile + 8 + n4);
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
                alpha[h] = m[h] == -INFINITY ? 0.f : exp2f(m[h] - m_new);
                m[h] = m_new;
                l[h] *= alpha[h];
            }
#pragma unroll
            for (int x = 0; x < 4 * NV; ++x) {
                o[x][0] *= alpha[0]; o[x][1] *= alpha[1]; o[x][2] *= alpha[0]; o[x][3] *= alpha[1];
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float base = m[h] == -INFINITY ? 0.f : m[h];  // nothing seen yet: every weight is zero
            w[h] = exp2f(w[h] - base);
            w[2 + h] = exp2f(w[2 + h] - base);
            l[h] += w[h] + w[2 + h];
        }
        uint32_t pb[PV][2];  // planes of P^T in the B layout; the last one is rounded (exact if it is the third)
#pragma unroll
        for (int pl = 0; pl < PV; ++pl)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                pb[pl][j] = transpose(pl < PV - 1 ? peel(w[2 * j], w[2 * j + 1]) : pack(w[2 * j], w[2 * j + 1]));
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
                // smallest plane first; the MMA's sums truncate, so that fp32 rows add a tile's product
                // to O in fp32
                float y[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) y[h] = F32 ? 0.f : o[4 * x + e][h];
#pragma unroll
                for (int pl = PV - 1; pl >= 0; --pl) mma(y, a0, a1, a2, a3, pb[pl][0], pb[pl][1]);
#pragma unroll
                for (int h = 0; h < 4; ++h) o[4 * x + e][h] = F32 ? o[4 * x + e][h] + y[h] : y[h];
            }
        }
        at = at_next;
    }

    // ---- join the warps: heads 2 c4 + h, elements 64 x + 8 n4 .. + 7
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int x = 4; x < 32; x *= 2) l[h] += __shfl_xor_sync(0xffffffffu, l[h], x);
        if (n4 == 0) {
            sm_m[warp][2 * c4 + h] = m[h];
            sm_l[warp][2 * c4 + h] = l[h];
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
// with blocks of 4; one of 1088 in 17 parts: 6.7 us a call and 7.6 in a graph, in nine parts
// 6.7 and 6.9).  But the lengths are on the device, and what is one wave of equal requests is a
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

template <int D, typename T>
cudaError_t launch_t(const DecodeArgs& p, cudaStream_t st) {
    return launch_pdl(window_decode_kernel<D, T>,
                      dim3((unsigned)p.a.rows * p.plan.splits, p.a.Hkv * p.plan.groups), kThreads, 0, st, p);
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
