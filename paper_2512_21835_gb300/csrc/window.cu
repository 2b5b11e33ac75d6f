// window.cu -- windowed serving over the paged cache, in bf16 or in 8 bits: the append of
// new tokens (norm of queries and keys for each head, position rotation, keys and values
// into their pages), rows of the 8-bit cache read back, and the entries of the attention
// behind a sliding window with sinks.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/loip.h"
#include "internal.h"
#include "q8.h"
#include "window.h"

namespace loip {
namespace {

// ---------------------------------------------------------------------------
// Append.
//
// y = x / sqrt(mean(x^2) + eps) * g for each query and key head (optional), then
// (y_i, y_{i + d/2}) turns by position * theta^(-2i/d).
//
// The angle is kept in turns, as a 64-bit fixed-point fraction: turn_i =
// theta^(-2i/d) / (2 pi), and position * turn_i modulo 2^64 is the fraction of a
// turn itself -- one integer product, with nothing to be reduced modulo 2 pi.
// turn_i is made in fp64 and is off by less than 2^-54 of a turn, the angle by less
// than position * 2^-54.  Its top 32 bits, as a signed number, are an angle in
// [-pi, pi) for sincospif.
// ---------------------------------------------------------------------------
struct RopeTurns {
    uint64_t turn[64];
};

// The table of a base and head size; the thread's last one is kept (64 powers take longer
// than the launch).
const RopeTurns& rope_turns(float theta, int d) {
    thread_local RopeTurns r;
    thread_local float of_theta = -1.f;
    thread_local int of_d = 0;
    if (theta != of_theta || d != of_d) {
        for (int i = 0; i < d / 2; ++i)  // below 1 / (2 pi) of 2^64, so the conversion is in range
            r.turn[i] = theta == 0.f ? 0 : (uint64_t)ldexp(pow((double)theta, -2.0 * i / d) * 0.15915494309189535, 64);
        of_theta = theta;
        of_d = d;
    }
    return r;
}

struct AppendArgs {
    const void* qkv;
    int64_t row_stride;
    const __nv_bfloat16 *g_q, *g_k;
    float eps;
    const int32_t *positions, *row_req;
    int rows, n_req, Hq, Hkv;
    int heads;  // per block
    void* q_out;
    KvView kv;
    RopeTurns rope;
};

// Eight elements as they lie in memory, and their values.
template <typename T>
struct Raw8 {
    uint4 u[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) u[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        if constexpr (sizeof(T) == 4) {
            v[0] = __uint_as_float(u[0].x); v[1] = __uint_as_float(u[0].y); v[2] = __uint_as_float(u[0].z);
            v[3] = __uint_as_float(u[0].w); v[4] = __uint_as_float(u[1].x); v[5] = __uint_as_float(u[1].y);
            v[6] = __uint_as_float(u[1].z); v[7] = __uint_as_float(u[1].w);
        } else {
            const uint32_t w[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
};
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}

// A block takes a group of heads of one token; D / 16 lanes per head, each holding the
// elements 8l .. 8l + 7 of the head and their partners D / 2 further on.  Bound by memory:
// short blocks with all their loads issued at once, the gains' among them, and as many of
// them per SM as the registers can be held to (bf16: 32, which costs 16 bytes of spills, 2.5
// stores and half a load per warp).  8191 fp32 tokens of 120 heads of 128: 121 us, 6.9 TB/s;
// 1999 bf16 tokens of 80 heads, with norms: 15.2 us, 5.4 TB/s (each before
// the bank conflicts went: eight blocks per SM 18.3, six 20.7, two tokens per block 19.9,
// one wave of blocks that walk over the tokens with the next one's loads in flight 28.7).
//
// The next launch may come from the start for fp32 rows into the bf16 cache, and once the loads are done for the others
// (in a graph, late and early: 76 fp32 rows of 48 heads 2.57 and 2.20 us, 304 4.49 and 3.73; 304 bf16 ones 2.69 and
// 3.10; 1 to 40 rows and 512 and more alike).
//
// Q8: keys and values go to the 8-bit cache (q8.h); the four lanes that hold a block's 32 elements find its
// exponent with two shuffles.  8191 fp32 tokens of 120 heads of 128: 119 us, 6.4 TB/s.
template <int D, typename T, bool Q8>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 8 : 6) qk_append_kernel(const __grid_constant__ AppendArgs p) {
    constexpr int LANES = D / 16;
    __shared__ float4 turn[4][LANES];  // cos, sin of elements 8l + 2k and 8l + 2k + 1 at [k][l]: no bank conflicts
    constexpr bool EARLY = !Q8 && sizeof(T) == 4;
    if (EARLY) pdl_trigger();
    pdl_wait();
    const int t = blockIdx.x, l = threadIdx.x % LANES, head = blockIdx.y * p.heads + threadIdx.x / LANES;
    const bool live = head < min(p.Hq + 2 * p.Hkv, (int)(blockIdx.y + 1) * p.heads);
    const bool is_q = head < p.Hq, is_v = head >= p.Hq + p.Hkv;
    const int pos = p.positions[t], req = p.row_req ? p.row_req[t] : t;
    Raw8<T> ra, rb;
    Raw8<__nv_bfloat16> ga, gb;
    if (live) {
        const T* x = static_cast<const T*>(p.qkv) + (int64_t)t * p.row_stride + head * D + 8 * l;
        ra.load(x);
        rb.load(x + D / 2);
        if (p.g_q && !is_v) {
            const __nv_bfloat16* g = (is_q ? p.g_q : p.g_k) + 8 * l;
            ga.load(g);
            gb.load(g + D / 2);
        }
    }
    const bool padding = pos < 0 || pos / kPageTokens >= p.kv.max_pages || req < 0 || req >= p.n_req;
    int64_t page = 0;
    if (live && !is_q && !padding) page = p.kv.page_offsets[(int64_t)req * p.kv.max_pages + pos / kPageTokens];
    if (threadIdx.x < D / 2) {
        const int32_t turns = (int32_t)((uint64_t)pos * p.rope.turn[threadIdx.x] >> 32);
        float s, c;
        sincospif((float)turns * 0x1p-31f, &s, &c);
        reinterpret_cast<float2*>(&turn[threadIdx.x % 8 / 2][threadIdx.x / 8])[threadIdx.x % 2] = make_float2(c, s);
    }
    __syncthreads();
    if (!EARLY) pdl_trigger();
    float a[8], b[8];
    if (live) {
        ra.values(a);
        rb.values(b);
    }
    if (p.g_q) {  // the sum is fp32, over a head's lanes
        float ss = 0.f;
        if (live) {
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(a[i], a[i], fmaf(b[i], b[i], ss));
        }
#pragma unroll
        for (int m = 1; m < LANES; m *= 2) ss += __shfl_xor_sync(0xffffffffu, ss, m);
        if (live && !is_v) {
            const float r = 1.0f / sqrtf(ss * (1.0f / D) + p.eps);
            float g[8];
            ga.values(g);
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] *= r * g[i];
            gb.values(g);
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] *= r * g[i];
        }
    }
    if (!live) return;
    if (!is_v && p.rope.turn[0]) {  // (theta 0: no rotation, and no 0 x inf)
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float4 cs = turn[i / 2][l];
            const float x = a[i], y = b[i], z = a[i + 1], w = b[i + 1];
            a[i] = x * cs.x - y * cs.y;
            b[i] = y * cs.x + x * cs.y;
            a[i + 1] = z * cs.z - w * cs.w;
            b[i + 1] = w * cs.z + z * cs.w;
        }
    }
    if (is_q) {
        T* o = static_cast<T*>(p.q_out) + ((int64_t)t * p.Hq + head) * D + 8 * l;
        if (padding) {
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = b[i] = 0.f;
        }
        store8(o, a);
        store8(o + D / 2, b);
    } else if (padding) {
        return;
    } else if constexpr (Q8) {
        const unsigned four = 15u << (threadIdx.x % 32 / 4 * 4);
        auto most_of = [&](const float (&v)[8]) {  // as bits, so that a NaN is the largest
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
            most = max(most, __shfl_xor_sync(four, most, 1));
            return max(most, __shfl_xor_sync(four, most, 2));
        };
        using G = q8::Granule<D>;
        const int token = pos % q8::kGranule, c = l / 2;
        char* o = p.kv.base + page + (uint64_t)p.kv.layer * p.kv.layer_page_bytes +
                  q8::granule_at<D>(head - p.Hq - (is_v ? p.Hkv : 0), pos);
        auto put = [&](const float (&v)[8], int half) {
            const uint32_t E = q8::exponent_of(most_of(v));
            uint2 u = make_uint2(0u, 0u);
            if (E != 255u) {
                const float inv = q8::inverse_step(E);
                u.x = q8::codes_of(v[0], v[1], v[2], v[3], inv);
                u.y = q8::codes_of(v[4], v[5], v[6], v[7], inv);
            }
            *reinterpret_cast<uint2*>(o + G::piece(is_v, token, half * (D / 32) + c) + l % 2 * 8) = u;
            if (l % 4 == 0) o[G::exponents(is_v, token) + half * (D / 64) + l / 4] = (char)E;
        };
        put(a, 0);
        put(b, 1);
    } else {
        // keys, then values, of the layer: [Hkv][64][D] each
        __nv_bfloat16* o =
            reinterpret_cast<__nv_bfloat16*>(p.kv.base + page + (uint64_t)p.kv.layer * p.kv.layer_page_bytes) +
            ((int64_t)(head - p.Hq) * kPageTokens + pos % kPageTokens) * D + 8 * l;
        store8(o, a);
        store8(o + D / 2, b);
    }
}

// Heads in equal groups of at most a block's 256 threads.
template <int D, typename T, bool Q8>
cudaError_t launch_append(AppendArgs& a, cudaStream_t st) {
    constexpr int LANES = D / 16, MOST = 256 / LANES;
    const int heads = a.Hq + 2 * a.Hkv, groups = (heads + MOST - 1) / MOST;
    a.heads = (heads + groups - 1) / groups;
    const unsigned threads = std::max((a.heads * LANES + 31) / 32 * 32, D / 2);
    return launch_pdl(qk_append_kernel<D, T, Q8>, dim3(a.rows, groups), threads, 0, st, a);
}

// ---------------------------------------------------------------------------
// Rows of the 8-bit cache as numbers.
// ---------------------------------------------------------------------------
struct ReadArgs {
    const int32_t *positions, *row_req;
    int rows, n_req, Hkv;
    KvView kv;
    void* out;  // [rows][keys, values][Hkv][d]
};

// 32 bytes in one store: whole sectors.
__device__ __forceinline__ void store32(void* p, const uint32_t (&u)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]),
                 "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
                 : "memory");
}

// A thread takes a piece (16 elements) of a key and of its value in R rows, `per_block` rows apart, and
// has all its loads in flight at once: bound by memory, with a chain of three latencies (position,
// page, codes) before it.  Four rows where that leaves eight blocks for each SM (100003 bf16 rows of 8
// heads of 128: 93 us, 6.7 TB/s; 8191 of 40: 40 us; with one 133 and 51), else one (1087 rows of 8
// heads: 2.7 us, with four 3.9).
template <int D, typename T, int R>
__global__ void __launch_bounds__(256) cache_read_kernel(const __grid_constant__ ReadArgs p, int per_block) {
    using G = q8::Granule<D>;
    pdl_wait();
    const int pieces = p.Hkv * G::PIECES, row = threadIdx.x / pieces, i = blockIdx.y * 256 + threadIdx.x - row * pieces;
    if (row >= per_block || i >= pieces) return;
    const int head = i / G::PIECES, c = i % G::PIECES;
    const int64_t t0 = (int64_t)blockIdx.x * per_block * R + row;
    int pos[R], req[R];
#pragma unroll
    for (int x = 0; x < R; ++x) {
        const int64_t t = t0 + x * per_block;
        pos[x] = t < p.rows ? p.positions[t] : -1;
        req[x] = t < p.rows && p.row_req ? p.row_req[t] : (int)t;
    }
    const char* g[R];
#pragma unroll
    for (int x = 0; x < R; ++x) {
        g[x] = nullptr;
        if (pos[x] >= 0 && pos[x] / kPageTokens < p.kv.max_pages && req[x] >= 0 && req[x] < p.n_req)
            g[x] = p.kv.base + p.kv.page_offsets[(int64_t)req[x] * p.kv.max_pages + pos[x] / kPageTokens] +
                   (uint64_t)p.kv.layer * p.kv.layer_page_bytes + q8::granule_at<D>(head, pos[x]);
    }
    uint4 u[R][2];
    uint32_t E[R][2];
#pragma unroll
    for (int x = 0; x < R; ++x)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            u[x][v] = make_uint4(0u, 0u, 0u, 0u);
            E[x][v] = 0u;
            if (g[x]) {
                u[x][v] = *reinterpret_cast<const uint4*>(g[x] + G::piece(v, pos[x] % q8::kGranule, c));
                E[x][v] = (uint8_t)g[x][G::exponents(v, pos[x] % q8::kGranule) + c / 2];
            }
        }
    pdl_trigger();
#pragma unroll
    for (int x = 0; x < R; ++x) {
        const int64_t t = t0 + x * per_block;
        if (t >= p.rows) return;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const uint32_t scale = q8::scale2(E[x][v] * 0x00010001u), w[4] = {u[x][v].x, u[x][v].y, u[x][v].z, u[x][v].w};
            uint32_t y[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[2 * e] = q8::pair_of(__byte_perm(w[e], 0u, 0x1100u), scale);
                y[2 * e + 1] = q8::pair_of(__byte_perm(w[e], 0u, 0x3322u), scale);
            }
            T* o = static_cast<T*>(p.out) + ((t * 2 + v) * pieces + i) * 16;
            if constexpr (sizeof(T) == 2) {
                store32(o, y);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t z[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        z[2 * e] = y[4 * h + e] << 16;
                        z[2 * e + 1] = y[4 * h + e] & 0xffff0000u;
                    }
                    store32(o + 8 * h, z);
                }
            }
        }
    }
}

template <int D, typename T>
cudaError_t launch_read(const ReadArgs& a, cudaStream_t st) {
    const int pieces = a.Hkv * (D / 16), per_block = std::max(1, 256 / pieces);
    auto grid = [&](int64_t rows) { return dim3((unsigned)((a.rows + rows - 1) / rows), (pieces + 255) / 256); };
    const dim3 four = grid(4 * (int64_t)per_block);
    if ((int64_t)four.x * four.y >= 8 * 152) return launch_pdl(cache_read_kernel<D, T, 4>, four, 256, 0, st, a, per_block);
    return launch_pdl(cache_read_kernel<D, T, 1>, grid(per_block), 256, 0, st, a, per_block);
}

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// What every call on the cache has in common; null if it is in order.
const char* cache_refusal(bool q8, int dtype, int rows, int Hq, int Hkv, int d, const void* kv_base,
                          const int64_t* page_offsets, int max_pages, int page_tokens, int layer, uint64_t layer_page_bytes) {
    if (dtype != LOIP_F32 && dtype != LOIP_BF16) return "dtype is LOIP_F32 or LOIP_BF16";
    if (rows < 0) return "a negative number of rows";
    if (Hkv < 1 || Hq < 1 || Hq % Hkv) return "the query heads are a multiple of the kv heads";
    if ((int64_t)Hq + 2 * (int64_t)Hkv > 65535) return "more heads than the kernels take";
    if (d != 64 && d != 128) return "the head size is 64 or 128";
    if (page_tokens != kPageTokens) return "pages hold 64 tokens";
    if (max_pages < 1 || layer < 0) return "no pages, or a negative layer";
    if (!kv_base || !aligned(kv_base, 16) || layer_page_bytes % 16) return "the cache is 16-byte aligned";
    if (!page_offsets || !aligned(page_offsets, 8)) return "the page table is an 8-byte aligned device array";
    if (q8 && layer_page_bytes < q8::layer_bytes(Hkv, d)) return "a layer's part of a page is Hkv * 132 * d bytes";
    return nullptr;
}

const char* window_refusal(const void* q, const void* o, int max_pages, int window, int sinks, int max_ctx,
                           const void* scratch, uint64_t scratch_bytes, uint64_t scratch_need) {
    if (!q || !o || !aligned(q, 16) || !aligned(o, 16)) return "queries and outputs are 16-byte aligned";
    if (window < 0 || sinks < 0) return "a negative window or number of sinks";
    if (max_ctx < 1 || max_ctx > 1 << 30 || (int64_t)max_pages * kPageTokens < max_ctx)
        return "max_ctx is 1 to max_pages * 64, and at most 2^30";
    if (!scratch || !aligned(scratch, 16) || scratch_bytes < scratch_need)
        return "the scratch is 16-byte aligned and as large as its size function says";
    return nullptr;
}

}  // namespace
}  // namespace loip

using namespace loip;

namespace {

int append(bool q8, const void* qkv, int32_t dtype, int64_t row_stride, int32_t T, int32_t Hq, int32_t Hkv, int32_t d,
           const uint16_t* g_q, const uint16_t* g_k, float eps, float theta, const int32_t* positions,
           const int32_t* row_req, int32_t n_req, void* q_out, void* kv_base, const int64_t* page_offsets,
           int32_t max_pages, int32_t page_tokens, int32_t layer, uint64_t layer_page_bytes, void* stream) {
    if (const char* why = cache_refusal(q8, dtype, T, Hq, Hkv, d, kv_base, page_offsets, max_pages, page_tokens, layer,
                                        layer_page_bytes))
        return kernel_refused(why);
    if (T == 0) return LOIP_OK;
    const int64_t width = (int64_t)(Hq + 2 * Hkv) * d;
    if (!qkv || !q_out || !aligned(qkv, 16) || !aligned(q_out, 16) || row_stride < width ||
        row_stride % (dtype == LOIP_F32 ? 4 : 8))
        return kernel_refused("the rows of qkv and q_out are 16-byte aligned and do not overlap");
    if (!positions || !aligned(positions, 4) || !aligned(row_req, 4) || n_req < 1)
        return kernel_refused("positions (and requests) are device int32 arrays, the page table has a row");
    if (!g_q != !g_k || !aligned(g_q, 16) || !aligned(g_k, 16))
        return kernel_refused("both gains or neither, 16-byte aligned");
    if (!(theta == 0.f || (theta >= 1.f && isfinite(theta))) || !(eps >= 0.f && isfinite(eps)))
        return kernel_refused("theta is 0 or at least 1, eps is not negative");
    AppendArgs a{};
    a.qkv = qkv;
    a.row_stride = row_stride;
    a.g_q = reinterpret_cast<const __nv_bfloat16*>(g_q);
    a.g_k = reinterpret_cast<const __nv_bfloat16*>(g_k);
    a.eps = eps;
    a.positions = positions;
    a.row_req = row_req;
    a.rows = T;
    a.n_req = n_req;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.q_out = q_out;
    a.kv = KvView{(char*)kv_base, page_offsets, max_pages, page_tokens, layer, layer_page_bytes};
    a.rope = rope_turns(theta, d);
    cudaStream_t st = (cudaStream_t)stream;
    auto go = [&](auto head, auto q8_cache) {
        constexpr int D = decltype(head)::value;
        constexpr bool Q8 = decltype(q8_cache)::value;
        return kernel_status(dtype == LOIP_F32 ? launch_append<D, float, Q8>(a, st)
                                               : launch_append<D, __nv_bfloat16, Q8>(a, st));
    };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    if (q8) return d == 128 ? go(D128{}, std::true_type{}) : go(D64{}, std::true_type{});
    return d == 128 ? go(D128{}, std::false_type{}) : go(D64{}, std::false_type{});
}

int attention(bool q8, const void* q, int32_t dtype, const void* kv_base, const int64_t* page_offsets,
              int32_t max_pages, const int32_t* ctx_lens, int32_t B, int32_t Hq, int32_t Hkv, int32_t d,
              int32_t page_tokens, int32_t layer, uint64_t layer_page_bytes, int32_t window, int32_t sinks,
              int32_t max_ctx, void* scratch, uint64_t scratch_bytes, void* o, void* stream) {
    if (const char* why = cache_refusal(q8, dtype, B, Hq, Hkv, d, kv_base, page_offsets, max_pages, page_tokens, layer,
                                        layer_page_bytes))
        return kernel_refused(why);
    if (B == 0) return LOIP_OK;
    const uint64_t need = q8 ? loip_k_window_attention_q8_scratch_bytes(B, Hq, Hkv, d, window, sinks, max_ctx)
                             : loip_k_window_attention_scratch_bytes(B, Hq, Hkv, d, window, sinks, max_ctx);
    if (const char* why = window_refusal(q, o, max_pages, window, sinks, max_ctx, scratch, scratch_bytes, need))
        return kernel_refused(why);
    if (!ctx_lens || !aligned(ctx_lens, 4)) return kernel_refused("ctx_lens is a device int32 array");
    WindowArgs a{};
    a.q = q;
    a.o = o;
    a.kv = KvView{(char*)kv_base, page_offsets, max_pages, page_tokens, layer, layer_page_bytes};
    a.ctx_lens = ctx_lens;
    a.rows = B;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.d = d;
    a.window = window;
    a.sinks = sinks;
    a.max_ctx = max_ctx;
    a.scratch = scratch;
    return kernel_status((q8 ? launch_window_decode_q8 : launch_window_decode)(a, dtype == LOIP_F32, (cudaStream_t)stream));
}

int prefill(bool q8, const void* q, int32_t dtype, const void* kv_base, const int64_t* page_offsets, int32_t max_pages,
            const int32_t* row_starts, const int32_t* first_pos, int32_t n_prompts, int32_t M, int32_t Hq, int32_t Hkv,
            int32_t d, int32_t page_tokens, int32_t layer, uint64_t layer_page_bytes, int32_t window, int32_t sinks,
            int32_t max_ctx, void* scratch, uint64_t scratch_bytes, void* o, void* stream) {
    if (const char* why = cache_refusal(q8, dtype, M, Hq, Hkv, d, kv_base, page_offsets, max_pages, page_tokens, layer,
                                        layer_page_bytes))
        return kernel_refused(why);
    if (M == 0) return LOIP_OK;
    if (n_prompts < 1) return kernel_refused("rows without a prompt");
    const uint64_t need = q8 ? loip_k_window_prefill_q8_scratch_bytes(M, n_prompts, Hq, Hkv, d, window, sinks, max_ctx)
                             : loip_k_window_prefill_scratch_bytes(M, n_prompts, Hq, Hkv, d, window, sinks, max_ctx);
    if (const char* why = window_refusal(q, o, max_pages, window, sinks, max_ctx, scratch, scratch_bytes, need))
        return kernel_refused(why);
    if (!row_starts || !aligned(row_starts, 4) || !aligned(first_pos, 4))
        return kernel_refused("row_starts (and first_pos) are device int32 arrays");
    WindowArgs a{};
    a.q = q;
    a.o = o;
    a.kv = KvView{(char*)kv_base, page_offsets, max_pages, page_tokens, layer, layer_page_bytes};
    a.row_starts = row_starts;
    a.first_pos = first_pos;
    a.n_prompts = n_prompts;
    a.rows = M;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.d = d;
    a.window = window;
    a.sinks = sinks;
    a.max_ctx = max_ctx;
    a.scratch = scratch;
    return kernel_status((q8 ? launch_window_prefill_q8 : launch_window_prefill)(a, dtype == LOIP_F32, (cudaStream_t)stream));
}

bool scratch_sizes(int rows, int Hq, int Hkv, int d, int window, int sinks, int max_ctx) {
    return rows >= 0 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && (d == 64 || d == 128) && window >= 0 && sinks >= 0 &&
           max_ctx >= 1;
}

}  // namespace

extern "C" int loip_k_qk_append(const void* qkv, int32_t dtype, int64_t row_stride, int32_t T, int32_t Hq, int32_t Hkv,
                                int32_t d, const uint16_t* g_q, const uint16_t* g_k, float eps, float theta,
                                const int32_t* positions, const int32_t* row_req, int32_t n_req, void* q_out,
                                void* kv_base, const int64_t* page_offsets, int32_t max_pages, int32_t page_tokens,
                                int32_t layer, uint64_t layer_page_bytes, void* stream) {
    return append(false, qkv, dtype, row_stride, T, Hq, Hkv, d, g_q, g_k, eps, theta, positions, row_req, n_req, q_out,
                  kv_base, page_offsets, max_pages, page_tokens, layer, layer_page_bytes, stream);
}

extern "C" uint64_t loip_k_window_attention_scratch_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t d,
                                                          int32_t window, int32_t sinks, int32_t max_ctx) {
    if (!scratch_sizes(B, Hq, Hkv, d, window, sinks, max_ctx)) return 0;
    return window_decode_scratch(B, Hq, Hkv, d, window, sinks, max_ctx);
}

extern "C" int loip_k_window_attention(const void* q, int32_t dtype, const void* kv_base, const int64_t* page_offsets,
                                       int32_t max_pages, const int32_t* ctx_lens, int32_t B, int32_t Hq, int32_t Hkv,
                                       int32_t d, int32_t page_tokens, int32_t layer, uint64_t layer_page_bytes,
                                       int32_t window, int32_t sinks, int32_t max_ctx, void* scratch,
                                       uint64_t scratch_bytes, void* o, void* stream) {
    return attention(false, q, dtype, kv_base, page_offsets, max_pages, ctx_lens, B, Hq, Hkv, d, page_tokens, layer,
                     layer_page_bytes, window, sinks, max_ctx, scratch, scratch_bytes, o, stream);
}

extern "C" uint64_t loip_k_window_prefill_scratch_bytes(int32_t M, int32_t n_prompts, int32_t Hq, int32_t Hkv,
                                                        int32_t d, int32_t window, int32_t sinks, int32_t max_ctx) {
    if (!scratch_sizes(M, Hq, Hkv, d, window, sinks, max_ctx) || n_prompts < 0) return 0;
    return window_prefill_scratch(M, n_prompts, Hq, Hkv, d, window, sinks, max_ctx);
}

extern "C" int loip_k_window_prefill(const void* q, int32_t dtype, const void* kv_base, const int64_t* page_offsets,
                                     int32_t max_pages, const int32_t* row_starts, const int32_t* first_pos,
                                     int32_t n_prompts, int32_t M, int32_t Hq, int32_t Hkv, int32_t d,
                                     int32_t page_tokens, int32_t layer, uint64_t layer_page_bytes, int32_t window,
                                     int32_t sinks, int32_t max_ctx, void* scratch, uint64_t scratch_bytes, void* o,
                                     void* stream) {
    return prefill(false, q, dtype, kv_base, page_offsets, max_pages, row_starts, first_pos, n_prompts, M, Hq, Hkv, d,
                   page_tokens, layer, layer_page_bytes, window, sinks, max_ctx, scratch, scratch_bytes, o, stream);
}

extern "C" int loip_k_qk_append_q8(const void* qkv, int32_t dtype, int64_t row_stride, int32_t T, int32_t Hq, int32_t Hkv,
                                   int32_t d, const uint16_t* g_q, const uint16_t* g_k, float eps, float theta,
                                   const int32_t* positions, const int32_t* row_req, int32_t n_req, void* q_out,
                                   void* kv_base, const int64_t* page_offsets, int32_t max_pages, int32_t page_tokens,
                                   int32_t layer, uint64_t layer_page_bytes, void* stream) {
    return append(true, qkv, dtype, row_stride, T, Hq, Hkv, d, g_q, g_k, eps, theta, positions, row_req, n_req, q_out,
                  kv_base, page_offsets, max_pages, page_tokens, layer, layer_page_bytes, stream);
}

extern "C" uint64_t loip_k_window_attention_q8_scratch_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t d,
                                                             int32_t window, int32_t sinks, int32_t max_ctx) {
    if (!scratch_sizes(B, Hq, Hkv, d, window, sinks, max_ctx)) return 0;
    return window_decode_q8_scratch(B, Hq, Hkv, d, window, sinks, max_ctx);
}

extern "C" int loip_k_window_attention_q8(const void* q, int32_t dtype, const void* kv_base, const int64_t* page_offsets,
                                          int32_t max_pages, const int32_t* ctx_lens, int32_t B, int32_t Hq, int32_t Hkv,
                                          int32_t d, int32_t page_tokens, int32_t layer, uint64_t layer_page_bytes,
                                          int32_t window, int32_t sinks, int32_t max_ctx, void* scratch,
                                          uint64_t scratch_bytes, void* o, void* stream) {
    return attention(true, q, dtype, kv_base, page_offsets, max_pages, ctx_lens, B, Hq, Hkv, d, page_tokens, layer,
                     layer_page_bytes, window, sinks, max_ctx, scratch, scratch_bytes, o, stream);
}

extern "C" uint64_t loip_k_window_prefill_q8_scratch_bytes(int32_t M, int32_t n_prompts, int32_t Hq, int32_t Hkv,
                                                           int32_t d, int32_t window, int32_t sinks, int32_t max_ctx) {
    if (!scratch_sizes(M, Hq, Hkv, d, window, sinks, max_ctx) || n_prompts < 0) return 0;
    return window_prefill_q8_scratch(M, n_prompts, Hq, Hkv, d, window, sinks, max_ctx);
}

extern "C" int loip_k_window_prefill_q8(const void* q, int32_t dtype, const void* kv_base, const int64_t* page_offsets,
                                        int32_t max_pages, const int32_t* row_starts, const int32_t* first_pos,
                                        int32_t n_prompts, int32_t M, int32_t Hq, int32_t Hkv, int32_t d,
                                        int32_t page_tokens, int32_t layer, uint64_t layer_page_bytes, int32_t window,
                                        int32_t sinks, int32_t max_ctx, void* scratch, uint64_t scratch_bytes, void* o,
                                        void* stream) {
    return prefill(true, q, dtype, kv_base, page_offsets, max_pages, row_starts, first_pos, n_prompts, M, Hq, Hkv, d,
                   page_tokens, layer, layer_page_bytes, window, sinks, max_ctx, scratch, scratch_bytes, o, stream);
}

extern "C" int loip_k_cache_read_q8(const void* kv_base, const int64_t* page_offsets, int32_t max_pages,
                                    const int32_t* positions, const int32_t* row_req, int32_t n_req, int32_t T,
                                    int32_t Hkv, int32_t d, int32_t page_tokens, int32_t layer,
                                    uint64_t layer_page_bytes, void* out, int32_t dtype, void* stream) {
    if (const char* why = cache_refusal(true, dtype, T, Hkv, Hkv, d, kv_base, page_offsets, max_pages, page_tokens,
                                        layer, layer_page_bytes))
        return kernel_refused(why);
    if (T == 0) return LOIP_OK;
    if (!out || !aligned(out, 32)) return kernel_refused("the rows that are read are 32-byte aligned");
    if (!positions || !aligned(positions, 4) || !aligned(row_req, 4) || n_req < 1)
        return kernel_refused("positions (and requests) are device int32 arrays, the page table has a row");
    const ReadArgs a{positions, row_req, T, n_req, Hkv,
                     KvView{(char*)kv_base, page_offsets, max_pages, page_tokens, layer, layer_page_bytes}, out};
    cudaStream_t st = (cudaStream_t)stream;
    if (d == 128)
        return kernel_status(dtype == LOIP_F32 ? launch_read<128, float>(a, st) : launch_read<128, __nv_bfloat16>(a, st));
    return kernel_status(dtype == LOIP_F32 ? launch_read<64, float>(a, st) : launch_read<64, __nv_bfloat16>(a, st));
}
