// window_prefill.cu -- attention of prompt rows over the paged cache, behind a
// sliding window with sinks, on the 5th-generation tensor cores.
//
// Rows.  The `heads` query heads that share a kv head are packed with consecutive
// positions into the 128 rows of an MMA tile (row = token * heads + head), so a
// tile spans 128 / heads positions: keys and values are read once for all heads,
// and a window costs little more than its own length.
//
// Keys.  The pages that some row of the block sees, those of the sinks and then
// those of the window, are a list without a gap; KT consecutive positions of it (one
// page or two) are a key tile.  Positions that no row of the block sees are not read:
// their rows in shared memory are zero-filled.
//
// Per key tile:  S = Q K^T -> tensor memory -> softmax in registers, one row per
// thread -> P back into tensor memory -> O += P V, V in its cache layout (the MMA
// takes B with d contiguous).  Two streams w = 0, 1 of this chain run in turn, so that
// the tensor core works for one while the other is in its softmax:
//   QT = 2: two row tiles over the same key tiles
//   QT = 1: one row tile, even and odd key tiles; the two partial softmax states are
//           joined at the end.  For fewer row tiles than the card has places.
//
// Precision.  bf16 rows: one MMA per product, weights rounded to bf16, O stays in
// tensor memory; it is rescaled only when a row's maximum has grown by 2^8 (weights
// are relative to an older maximum until then, exact in the end).  fp32 rows (NP = 3):
// queries and weights are exact sums of three bf16 planes, three MMAs per product,
// smallest plane first; the tensor core's sums truncate, so O of one key tile is
// drained and added in fp32 registers.
//
// A value that is not finite would spoil rows that do not see it (0 x inf).  In key
// tiles that not all rows see in full, the loader looks for such values, zeroes them
// and flags the block, whose rows are then walked one by one (walk_row).
//
// Roles (512 threads): warps 0-3 and 4-7 softmax of stream 0 and 1 (one row per
// thread), warps 8-11 load (cp.async, 128-byte swizzle), warp 12 issues the MMAs.
// Every wait is bounded (2 s); one that runs out records an error, the block stops,
// lets its copies and MMAs finish, frees its tensor memory and returns.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "internal.h"
#include "window.h"

namespace loip {

__device__ int g_window_error;  // first failure code of any launch (0 = none)

namespace {

constexpr int kThreads = 512;
constexpr int kSms = 152;
constexpr int kSoftRegs = 192, kOtherRegs = 64;  // 2 x 128 x 192 + 2 x 128 x 64 = 512 x 128

template <int D, int NP, int QT>
struct Cfg {
    static constexpr int KT = NP == 1 ? 128 : 64;      // keys per tile
    static constexpr int PPT = KT / kPageTokens;       // pages per tile
    static constexpr int SLABS = D / 64;               // 128-byte columns of a row
    static constexpr int Q_SLAB = 128 * 128;
    static constexpr int Q_PLANE = SLABS * Q_SLAB;
    static constexpr int Q_BYTES = QT * NP * Q_PLANE;  // [tile][plane][slab][row]
    static constexpr int KV_SLAB = KT * 128;
    static constexpr int SLOT = SLABS * KV_SLAB;       // one tile of keys or of values
    static constexpr int ROOM = 227 * 1024 - 1024 - 512 - Q_BYTES;
    static constexpr int SLOTS = ROOM / SLOT < 8 ? ROOM / SLOT : 8;
    static constexpr int LAG = 2;                      // tiles in flight behind the newest
    static constexpr int LEAD = QT == 2 ? 1 : 2;       // key tiles ahead of the values
    static constexpr int CTL = Q_BYTES + SLOTS * SLOT;
    static constexpr int BYTES = CTL + 512 + 1024;     // + alignment of the window
    static_assert(SLOTS >= LAG + 2, "the loader signals a tile LAG tiles late");
    static_assert(QT == 2 || SLOTS * SLOT >= 128 * D * 4, "the join goes through the ring");
    // tensor memory of stream w, from column 256 w
    static constexpr uint32_t S = 0, O = 128;
    static constexpr uint32_t P0 = NP == 1 ? 0 : 64, P1 = 0, P2 = 96;  // columns that S has been read from, or free
};

struct Ctl {  // control words behind the ring
    uint64_t full[8], empty[8], s_full[2], p_full[2], pv_done[2], q_full, end;
    uint32_t tmem;
    int abort, bad;
    int row0, tokens, req, pos0;
};
static_assert(sizeof(Ctl) <= 512, "");

struct PrefillArgs {
    WindowArgs a;
    int heads, groups;  // query heads per row tile, groups per kv head
    int tok;            // positions per row tile
    float scale;        // log2(e) / sqrt(d)
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t n) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(smem_u32(b)), "r"(parity)
        : "memory");
    return ok != 0;
}
// Waits for the phase of that parity; false if the block is to stop.  (Inlined: a call
// would take part in the register split.)
__device__ __forceinline__ bool bar_wait_slow(Ctl* c, uint64_t* b, uint32_t parity, int code) {
    const uint64_t t0 = now_ns();
    while (!bar_try(b, parity)) {
        if (*(volatile int*)&c->abort) return false;
        if (now_ns() - t0 > 2000000000ull) {
            *(volatile int*)&c->abort = 1;
            atomicCAS(&g_window_error, 0, code);
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool bar_wait(Ctl* c, uint64_t* b, uint32_t parity, int code) {
    return bar_try(b, parity) || bar_wait_slow(c, b, parity, code);
}
// The same for a whole warp, which leaves it converged.
__device__ __forceinline__ bool warp_wait(Ctl* c, uint64_t* b, uint32_t parity, int code) {
    return __all_sync(0xffffffffu, bar_wait(c, b, parity, code));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The MMA warp runs as a whole; its issuing instructions are predicated on the elected
// lane inside one asm block, so that addresses and descriptors stay warp-uniform.  Issued
// from a lane's own branch they took 130 cycles each, twice what an MMA of 128 columns
// takes the tensor core.
__device__ __forceinline__ void commit(uint64_t* b) {
    asm volatile(
        "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n"
        " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(smem_u32(b))
        : "memory");
}
// kind::f16, fp32 accumulator, bf16 A and B, M = 128, N = n; B with its N contiguous when `b_mn`
__host__ __device__ constexpr uint32_t idesc(int n, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(128 >> 4) << 24);
}
// Shared-memory operand with 128-byte rows and the 128-byte swizzle, 8-row groups 1024
// bytes apart; lbo: distance of the next 64 columns when the rows run along K (B of P V)
__device__ __forceinline__ uint64_t sdesc(uint32_t addr, uint32_t lbo) {
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// Four MMAs (64 of K): both operands in shared memory, 32 bytes a step along their rows;
__device__ __forceinline__ void mma_ss4(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t acc) {
    asm volatile(
        "{\n .reg .pred e, p, t;\n .reg .b64 a1, a2, a3, b1, b2, b3;\n"
        " elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n setp.eq.b32 t, %4, %4;\n"
        " add.s64 a1, %1, 2;\n add.s64 a2, %1, 4;\n add.s64 a3, %1, 6;\n"
        " add.s64 b1, %2, 2;\n add.s64 b2, %2, 4;\n add.s64 b3, %2, 6;\n"
        " @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
        " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a1, b1, %3, t;\n"
        " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a2, b2, %3, t;\n"
        " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a3, b3, %3, t;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(id), "r"(acc)
        : "memory");
}
// A in tensor memory, 8 columns a step; B 16 rows of 128 bytes a step.
__device__ __forceinline__ void mma_ts4(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t acc) {
    asm volatile(
        "{\n .reg .pred e, p, t;\n .reg .b32 a1, a2, a3;\n .reg .b64 b1, b2, b3;\n"
        " elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n setp.eq.b32 t, %4, %4;\n"
        " add.s32 a1, %1, 8;\n add.s32 a2, %1, 16;\n add.s32 a3, %1, 24;\n"
        " add.s64 b1, %2, 128;\n add.s64 b2, %2, 256;\n add.s64 b3, %2, 384;\n"
        " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
        " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, t;\n"
        " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %3, t;\n"
        " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %3, t;\n}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(id), "r"(acc)
        : "memory");
}
#define LOIP_R32(r, b) \
    "=r"(r[b]), "=r"(r[b + 1]), "=r"(r[b + 2]), "=r"(r[b + 3]), "=r"(r[b + 4]), "=r"(r[b + 5]), "=r"(r[b + 6]), \
        "=r"(r[b + 7]), "=r"(r[b + 8]), "=r"(r[b + 9]), "=r"(r[b + 10]), "=r"(r[b + 11]), "=r"(r[b + 12]), \
        "=r"(r[b + 13]), "=r"(r[b + 14]), "=r"(r[b + 15]), "=r"(r[b + 16]), "=r"(r[b + 17]), "=r"(r[b + 18]), \
        "=r"(r[b + 19]), "=r"(r[b + 20]), "=r"(r[b + 21]), "=r"(r[b + 22]), "=r"(r[b + 23]), "=r"(r[b + 24]), \
        "=r"(r[b + 25]), "=r"(r[b + 26]), "=r"(r[b + 27]), "=r"(r[b + 28]), "=r"(r[b + 29]), "=r"(r[b + 30]), \
        "=r"(r[b + 31])
// 32 columns of this warp's 32 rows; valid after tmem_landed
template <int B, int N>
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t (&r)[N]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,"
        "%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : LOIP_R32(r, B)
        : "r"(addr));
}
#undef LOIP_R32
// Waits for the loads; the registers are operands so that no use moves ahead of the wait.
template <int N>
__device__ __forceinline__ void tmem_landed(uint32_t (&r)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i])::"memory");
}
template <int B, int N>
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[N]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
            addr),
        "r"(r[B]), "r"(r[B + 1]), "r"(r[B + 2]), "r"(r[B + 3]), "r"(r[B + 4]), "r"(r[B + 5]), "r"(r[B + 6]),
        "r"(r[B + 7]), "r"(r[B + 8]), "r"(r[B + 9]), "r"(r[B + 10]), "r"(r[B + 11]), "r"(r[B + 12]), "r"(r[B + 13]),
        "r"(r[B + 14]), "r"(r[B + 15])
        : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t n) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float asf(uint32_t u) { return __uint_as_float(u); }
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// The pair's next plane: v becomes v - bf16(v), exactly.
__device__ __forceinline__ uint32_t peel(float& lo, float& hi) {
    const uint32_t p = pack(lo, hi);
    lo -= asf(p << 16);
    hi -= asf(p & 0xffff0000u);
    return p;
}
__device__ __forceinline__ uint64_t low_bits(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; }

__device__ __forceinline__ float row_load(const float* p) { return *p; }
__device__ __forceinline__ float row_load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void row_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void row_store(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// One row by one warp, position by position: what is not seen is not touched.
template <int D, typename T>
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
        const __nv_bfloat16* k =
            reinterpret_cast<const __nv_bfloat16*>(
                layer + a.kv.page_offsets[(int64_t)req * a.kv.max_pages + j / kPageTokens]) +
            ((int64_t)kvh * kPageTokens + j % kPageTokens) * D;
        const __nv_bfloat16* v = k + (int64_t)a.Hkv * kPageTokens * D;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) s = fmaf(qv[i], __bfloat162float(k[i * 32 + lane]), s);
#pragma unroll
        for (int x = 16; x; x /= 2) s += __shfl_xor_sync(0xffffffffu, s, x);
        s *= scale;
        const float m_new = fmaxf(m, s), alpha = m == -INFINITY ? 0.f : expf(m - m_new), w = expf(s - m_new);
        l = l * alpha + w;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) o[i] = fmaf(w, __bfloat162float(v[i * 32 + lane]), o[i] * alpha);
        m = m_new;
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) row_store(out + i * 32 + lane, o[i] * inv);
}

// The pages that rows at positions p0 .. p1 see: [0, sink) and [win, end), a list of n.
struct Pages {
    int sink, win, end, n, last;  // last: one past the last position that a row sees
    __device__ Pages(const WindowArgs& a, int p0, int p1) {
        last = max(0, min(p1 + 1, a.max_ctx));
        end = (last + kPageTokens - 1) / kPageTokens;
        sink = min((a.sinks + kPageTokens - 1) / kPageTokens, end);
        win = a.window == 0 ? end : max(max(0, p0 - a.window + 1) / kPageTokens, sink);
        win = min(win, end);
        n = sink + end - win;
    }
    __device__ int at(int v) const { return v < sink ? v : v - sink + win; }
};

template <int D, int NP, int QT, typename T>
__global__ void __launch_bounds__(kThreads, 1) window_prefill_kernel(const __grid_constant__ PrefillArgs p) {
    using C = Cfg<D, NP, QT>;
    constexpr int KT = C::KT;
    const WindowArgs& a = p.a;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    Ctl* c = reinterpret_cast<Ctl*>(sm + C::CTL);
    const uint32_t q_smem = smem_u32(sm), ring = q_smem + C::Q_BYTES;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;

    // ---- which rows: block units are kv heads (and groups of their heads) fastest, prompts
    // and row tiles from the last, whose rows see the most
    const int units = a.Hkv * p.groups;
    const int kvh = blockIdx.x % units / p.groups, head0 = blockIdx.x % units % p.groups * p.heads;
    const int G = a.Hq / a.Hkv, heads = min(p.heads, G - head0);
    if (warp == 0) {
        int left = blockIdx.x / units;  // row tiles from the end
        int row0 = 0, tokens = 0, req = 0, pos0 = 0;
        for (int top = a.n_prompts - 1; top >= 0; top -= 32) {
            const int i = top - lane;
            int lo = 0, hi = 0;
            if (i >= 0) {
                lo = min(max(a.row_starts[i], 0), a.rows);
                hi = min(max(a.row_starts[i + 1], lo), a.rows);
            }
            const int mine = (hi - lo + QT * p.tok - 1) / (QT * p.tok);
            int sum = mine;
#pragma unroll
            for (int x = 1; x < 32; x *= 2) {
                const int y = __shfl_up_sync(0xffffffffu, sum, x);
                if (lane >= x) sum += y;
            }
            const unsigned has = __ballot_sync(0xffffffffu, sum > left);
            if (has) {
                const int src = __ffs(has) - 1;
                if (lane == src) {
                    const int first = (sum - 1 - left) * QT * p.tok;  // `left - (sum - mine)` tiles from its end
                    row0 = lo + first;
                    tokens = min(QT * p.tok, hi - lo - first);
                    req = i;
                    pos0 = min(max(a.first_pos ? a.first_pos[i] : 0, -(1 << 30)), 1 << 30) + first;
                }
                row0 = __shfl_sync(0xffffffffu, row0, src);
                tokens = __shfl_sync(0xffffffffu, tokens, src);
                req = __shfl_sync(0xffffffffu, req, src);
                pos0 = __shfl_sync(0xffffffffu, pos0, src);
                break;
            }
            left -= __shfl_sync(0xffffffffu, sum, 31);
        }
        if (lane == 0) {
            c->row0 = row0;
            c->tokens = tokens;
            c->req = req;
            c->pos0 = pos0;
            c->abort = 0;
            c->bad = 0;
            for (int i = 0; i < C::SLOTS; ++i) {
                bar_init(&c->full[i], 128);
                bar_init(&c->empty[i], 1);
            }
            for (int w = 0; w < 2; ++w) {
                bar_init(&c->s_full[w], 1);
                bar_init(&c->p_full[w], 128);
                bar_init(&c->pv_done[w], 1);
            }
            bar_init(&c->q_full, 256);
            bar_init(&c->end, 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
    }
    __syncthreads();
    const int row0 = c->row0, tokens = c->tokens, req = c->req, pos0 = c->pos0;
    if (tokens == 0) return;  // the grid is an upper bound
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&c->tmem)),
                     "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = c->tmem;

    const int pos1 = pos0 + tokens - 1;
    const Pages pages(a, pos0, pos1);
    const int n = (pages.n + C::PPT - 1) / C::PPT;  // key tiles
    // the rows of stream w: its row tile's
    auto stream_pos = [&](int w) { return QT == 2 ? pos0 + w * p.tok : pos0; };
    auto stream_tokens = [&](int w) { return QT == 2 ? min(max(tokens - w * p.tok, 0), p.tok) : tokens; };
    // the key tiles that stream w computes: [0, sink) and [lo, hi)
    struct Takes {
        int sink, lo, hi;
        __device__ bool operator()(int t) const { return t < sink || (t >= lo && t < hi); }
    };
    auto takes_of = [&](int w) {
        Takes k{0, 0, 0};
        if (stream_tokens(w) > 0) {
            const Pages mine(a, stream_pos(w), stream_pos(w) + stream_tokens(w) - 1);
            const int shift = pages.sink - pages.win;  // of a window page in the list
            k.sink = (min(mine.sink, pages.sink) + C::PPT - 1) / C::PPT;
            if (mine.end > max(mine.win, pages.win)) {
                k.lo = (max(mine.win, pages.win) + shift) / C::PPT;
                k.hi = (mine.end + shift + C::PPT - 1) / C::PPT;
            }
        }
        return k;
    };

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp < 12) {
            // ---------------------------------------------------------------- loader
            const int lt = tid - 256;
            constexpr int CPR = D / 8, RPP = 128 / CPR;  // 16-byte chunks per row, rows per pass
            const int chunk = lt % CPR, r0 = lt / CPR;
            const char* layer = a.kv.base + (uint64_t)a.kv.layer * a.kv.layer_page_bytes;
            const int64_t* table = a.kv.page_offsets + (int64_t)req * a.kv.max_pages;
            const int win0 = max(0, pos0 - a.window + 1);  // (window 0: no page of it is in the list)
            auto seen = [&](int pos) {
                return pos < pages.last && ((pos >= win0 && a.window > 0) || pos < a.sinks);
            };
            auto place = [&](uint32_t slot, int x, int r) {
                return slot + (uint32_t)((chunk >> 3) * C::KV_SLAB + (x * kPageTokens + r) * 128 +
                                         (((chunk & 7) ^ (r & 7)) << 4));
            };
            // the tile at a place of the order: its index, and whether it holds values
            auto tile_of = [&](int at, bool& is_v) {
                is_v = false;
                if (at < min(n, C::LEAD)) return at;
                const int x = at - min(n, C::LEAD);  // V0 K_LEAD V1 K_(LEAD+1) ... then values alone
                const int both = max(n - C::LEAD, 0);
                if (x < 2 * both) {
                    is_v = (x & 1) == 0;
                    return is_v ? x / 2 : x / 2 + C::LEAD;
                }
                is_v = true;
                return x - both;
            };
            // tiles that some row does not see in full: values that are not finite are taken out
            auto check = [&](int at) {
                bool is_v;
                const int t = tile_of(at, is_v);
                if (!is_v) return;
                const uint32_t slot = ring + (uint32_t)(at % C::SLOTS) * C::SLOT;
                for (int x = 0; x < C::PPT; ++x) {
                    const int v = t * C::PPT + x, b = pages.at(v) * kPageTokens;
                    if (v >= pages.n) break;
                    if (b + kPageTokens - 1 <= pos0 &&
                        (b > pos1 - a.window || b + kPageTokens <= a.sinks)) continue;  // all rows see all of it
                    for (int r = r0; r < kPageTokens; r += RPP) {
                        const uint32_t w = place(slot, x, r);
                        uint32_t u[4];
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                                     : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                                     : "r"(w)
                                     : "memory");
                        bool bad = false;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            bad |= (u[i] & 0x7F80u) == 0x7F80u || (u[i] & 0x7F800000u) == 0x7F800000u;
                        if (bad) {
                            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(w), "r"(0u) : "memory");
                            *(volatile int*)&c->bad = 1;
                        }
                    }
                }
            };
            auto signal = [&](int at) {
                check(at);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                bar_arrive(&c->full[at % C::SLOTS]);
            };
            const int total = 2 * n;
            const int step = RPP * D * 2;  // a pass further in the page; RPP is a multiple of 8: the swizzle stays
            static_assert(RPP % 8 == 0, "");
            int at = 0, slot = 0;
            uint32_t free_phase = 1;  // of the ring's previous round; none for the first
            for (; at < total; ++at) {
                if (at >= C::SLOTS && !bar_wait(c, &c->empty[slot], free_phase, 1)) break;
                bool is_v;
                const int t = tile_of(at, is_v);
#pragma unroll
                for (int x = 0; x < C::PPT; ++x) {
                    const int v = t * C::PPT + x;
                    const int pg = v < pages.n ? pages.at(v) : 0, b = pg * kPageTokens;
                    const uint32_t dst = place(ring + (uint32_t)slot * C::SLOT, x, r0);
                    const char* src = layer;
                    if (v < pages.n)
                        src += __ldg(table + pg) + ((int64_t)(is_v ? a.Hkv : 0) + kvh) * (kPageTokens * D * 2) +
                               (r0 * D + chunk * 8) * 2;
                    if (v < pages.n && b + kPageTokens <= pages.last &&
                        ((b >= win0 && a.window > 0) || b + kPageTokens <= a.sinks)) {  // the whole page
#pragma unroll
                        for (int k = 0; k < kPageTokens / RPP; ++k) cp_async16(dst + k * RPP * 128, src + k * step, 16u);
                    } else {
#pragma unroll
                        for (int k = 0; k < kPageTokens / RPP; ++k) {
                            const bool ok = v < pages.n && seen(b + r0 + k * RPP);
                            cp_async16(dst + k * RPP * 128, ok ? src + k * step : layer, ok ? 16u : 0u);
                        }
                    }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                if (at >= C::LAG) {
                    asm volatile("cp.async.wait_group %0;" ::"n"(C::LAG) : "memory");
                    signal(at - C::LAG);
                }
                if (++slot == C::SLOTS) {
                    slot = 0;
                    free_phase ^= 1;
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (at == total)
                for (int i = max(0, total - C::LAG); i < total; ++i) signal(i);
        } else if (warp == 12 && n > 0) {
            // ---------------------------------------------------------------- MMA issue
            uint32_t pv_n[2] = {0, 0};  // products P V issued per stream
            bool ok = warp_wait(c, &c->q_full, 0, 2);
            // the ring is used in its own order: a cursor and the phase of its round
            int slot = 0;
            uint32_t phase = 0;
            auto advance = [&] {
                commit(&c->empty[slot]);
                if (++slot == C::SLOTS) {
                    slot = 0;
                    phase ^= 1;
                }
            };
            const uint64_t q_desc = sdesc(q_smem, 16), k_desc = sdesc(ring, 16), v_desc = sdesc(ring, C::KV_SLAB);
            auto issue_s = [&](int w) {  // S of the keys at the cursor; P of the stream's last tile has been used
                if (!warp_wait(c, &c->full[slot], phase, 3)) return false;
                if (pv_n[w] && !warp_wait(c, &c->pv_done[w], (pv_n[w] - 1) & 1, 4)) return false;
                fence_after();
                const uint64_t q = q_desc + (QT == 2 ? (uint32_t)w * (NP * C::Q_PLANE / 16) : 0u);
                const uint64_t k = k_desc + (uint32_t)slot * (C::SLOT / 16);
                const uint32_t d = tmem + 256u * w + C::S;
#pragma unroll
                for (int pl = NP - 1; pl >= 0; --pl)
#pragma unroll
                    for (int x = 0; x < D / 64; ++x)
                        mma_ss4(d, q + (pl * C::Q_PLANE + x * C::Q_SLAB) / 16, k + x * C::KV_SLAB / 16,
                                idesc(KT, false), pl != NP - 1 || x != 0);
                commit(&c->s_full[w]);
                return true;
            };
            auto issue_pv = [&](int w) {  // O += P V of the values at the cursor
                if (!warp_wait(c, &c->p_full[w], pv_n[w] & 1, 5) || !warp_wait(c, &c->full[slot], phase, 3)) return false;
                fence_after();
                const uint64_t v = v_desc + (uint32_t)slot * (C::SLOT / 16);
                const uint32_t d = tmem + 256u * w + C::O, pa = tmem + 256u * w;
                const uint32_t first = NP == 1 && pv_n[w] ? 1u : 0u;  // O is kept, or drained per tile
#pragma unroll
                for (int pl = NP - 1; pl >= 0; --pl)
#pragma unroll
                    for (int x = 0; x < KT / 64; ++x)
                        mma_ts4(d, pa + (pl == 0 ? C::P0 : pl == 1 ? C::P1 : C::P2) + 32 * x, v + x * (64 * 128 / 16),
                                idesc(D, true), pl != NP - 1 || x != 0 ? 1u : first);
                ++pv_n[w];
                commit(&c->pv_done[w]);
                return true;
            };
            if (QT == 2) {
                const Takes k0 = takes_of(0), k1 = takes_of(1);
                if (ok && k0(0)) ok = issue_s(0);
                if (ok && k1(0)) ok = issue_s(1);
                advance();
                for (int t = 0; t < n && ok; ++t) {
                    // cursor on V_t; K_(t+1) is the next one
                    const int v_slot = slot;
                    const uint32_t v_phase = phase;
                    const bool more = t + 1 < n;
                    auto to_k = [&] {
                        if (++slot == C::SLOTS) {
                            slot = 0;
                            phase ^= 1;
                        }
                    };
                    auto to_v = [&] {
                        slot = v_slot;
                        phase = v_phase;
                    };
                    if (k0(t)) ok = issue_pv(0);
                    if (ok && more && k0(t + 1)) {
                        to_k();
                        ok = issue_s(0);
                        to_v();
                    }
                    if (ok && k1(t)) ok = issue_pv(1);
                    advance();
                    if (ok && more && k1(t + 1)) ok = issue_s(1);
                    if (more) advance();
                }
            } else {
                for (int t = 0; t < min(2, n) && ok; ++t) {
                    ok = issue_s(t);
                    advance();
                }
                for (int t = 0; t < n && ok; ++t) {
                    ok = issue_pv(t & 1);
                    advance();
                    if (ok && t + 2 < n) {
                        ok = issue_s(t & 1);
                        advance();
                    }
                }
            }
            // nothing may be in flight when the tensor memory is released
            commit(&c->end);
            const uint64_t t0 = now_ns();
            while (!bar_try(&c->end, 0) && now_ns() - t0 < 2000000000ull) {}
        }
    } else {
        // -------------------------------------------------------------------- softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
        const T* qg = static_cast<const T*>(a.q);
        T* og = static_cast<T*>(a.o);
        auto row_at = [&](int tok, int head) {  // element offset of a row of q and o
            return ((int64_t)(row0 + tok) * a.Hq + kvh * G + head0 + head) * D;
        };
        // ---- queries -> shared memory, bf16 planes, swizzled; eight loads in flight per thread
        constexpr int CPR = D / 8, EACH = QT * 128 * CPR / 256, MOST = NP == 1 ? 8 : 4, BATCH = EACH < MOST ? EACH : MOST;
        static_assert(EACH % BATCH == 0, "");
        for (int i0 = tid; i0 < QT * 128 * CPR; i0 += 256 * BATCH) {
            uint4 x[BATCH], y[NP == 1 ? 1 : BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int i = i0 + 256 * k, r = i / CPR % 128, tile = i / CPR / 128;
                const int tk = r / heads, tok = tile * p.tok + tk;
                x[k] = make_uint4(0u, 0u, 0u, 0u);
                if constexpr (NP > 1) y[k] = x[k];
                if (tk < p.tok && tok < tokens) {
                    const uint4* src = reinterpret_cast<const uint4*>(qg + row_at(tok, r - tk * heads) + i % CPR * 8);
                    x[k] = __ldg(src);
                    if constexpr (NP > 1) y[k] = __ldg(src + 1);
                }
            }
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int i = i0 + 256 * k, ch = i % CPR, r = i / CPR % 128, tile = i / CPR / 128;
                uint8_t* dst =
                    sm + tile * NP * C::Q_PLANE + (ch >> 3) * C::Q_SLAB + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
                if constexpr (NP == 1) {
                    *reinterpret_cast<uint4*>(dst) = x[k];
                } else {
                    float v[8] = {asf(x[k].x), asf(x[k].y), asf(x[k].z), asf(x[k].w),
                                  asf(y[k].x), asf(y[k].y), asf(y[k].z), asf(y[k].w)};
#pragma unroll
                    for (int pl = 0; pl < NP; ++pl) {
                        uint32_t u[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) u[e] = peel(v[2 * e], v[2 * e + 1]);
                        *reinterpret_cast<uint4*>(dst + pl * C::Q_PLANE) = make_uint4(u[0], u[1], u[2], u[3]);
                    }
                }
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        bar_arrive(&c->q_full);

        const int w = warp / 4, r = tid % 128;
        const int base_tok = QT == 2 ? w * p.tok : 0, mine = stream_tokens(w);
        const int tk = r / heads;
        const bool live = tk < min(p.tok, mine);
        const int pos = live ? pos0 + base_tok + tk : -1;
        const int first = pos0 + base_tok, final = first + mine - 1;  // positions of the stream's rows
        const uint32_t t_row = tmem + 256u * w + ((uint32_t)(warp % 4) << 21);
        float m = -INFINITY, l = 0.f;  // m: the maximum that the weights are relative to
        uint32_t done = 0;             // tiles computed
        float o[NP == 1 ? 1 : D];
        if constexpr (NP > 1) {
#pragma unroll
            for (int i = 0; i < D; ++i) o[i] = 0.f;
        }
        bool ok = true;
        const Takes takes = takes_of(w);
        for (int t = QT == 1 ? w : 0; t < n; t += QT == 1 ? 2 : 1) {
            if (QT == 2 && !takes(t)) continue;
            // which positions of the tile this row sees, one bit each
            bool masked = false;
            uint32_t see[KT / 32];
#pragma unroll
            for (int x = 0; x < C::PPT; ++x) {
                const int v = t * C::PPT + x, b = pages.at(v) * kPageTokens;
                const bool all = v < pages.n && b + kPageTokens - 1 <= first &&
                                 (b > final - a.window || b + kPageTokens <= a.sinks);
                masked |= !all;
                uint64_t bits = ~0ull;
                if (!all)
                    bits = v < pages.n && live ? low_bits(min(pos, a.max_ctx - 1) - b + 1) &
                                                     (~low_bits(pos - a.window + 1 - b) | low_bits(a.sinks - b))
                                               : 0ull;
                see[2 * x] = (uint32_t)bits;
                see[2 * x + 1] = (uint32_t)(bits >> 32);
            }
            if (!(ok = warp_wait(c, &c->s_full[w], done & 1, 6))) break;
            fence_after();
            if constexpr (NP == 1) {
                uint32_t s[KT];
                tmem_ld32<0>(t_row + C::S, s);
                tmem_ld32<32>(t_row + C::S + 32, s);
                tmem_ld32<64>(t_row + C::S + 64, s);
                tmem_ld32<96>(t_row + C::S + 96, s);
                tmem_landed(s);
                if (masked) {
#pragma unroll
                    for (int i = 0; i < KT; ++i)
                        if (!(see[i / 32] >> (i % 32) & 1u)) s[i] = 0xff800000u;  // -inf
                }
                float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
                for (int i = 0; i < KT; i += 4) {
                    x0 = fmaxf(x0, fmaxf(asf(s[i]), asf(s[i + 1])));
                    x1 = fmaxf(x1, fmaxf(asf(s[i + 2]), asf(s[i + 3])));
                }
                const float mx = fmaxf(x0, x1) * p.scale;
                // O is rescaled when a row's maximum has outgrown the one in use by 2^8; P V of
                // the stream's last tile is complete (S of this one was issued after it)
                const bool grown = mx > m + 8.f;  // the first time too: m is -inf
                if (__any_sync(0xffffffffu, grown)) {
                    const float m_new = grown ? mx : m;
                    const float alpha = m == -INFINITY ? 0.f : ex2(m - m_new);
                    m = m_new;
                    l *= alpha;
                    if (done) {
#pragma unroll
                        for (int i = 0; i < D; i += 32) {
                            uint32_t y[32];
                            tmem_ld32<0>(t_row + C::O + i, y);
                            tmem_landed(y);
#pragma unroll
                            for (int e = 0; e < 32; ++e) y[e] = __float_as_uint(asf(y[e]) * alpha);
                            tmem_st16<0>(t_row + C::O + i, y);
                            tmem_st16<16>(t_row + C::O + i + 16, y);
                        }
                    }
                }
                const float base = m == -INFINITY ? 0.f : m;
                float l0 = 0.f, l1 = 0.f;
#pragma unroll
                for (int i = 0; i < KT; i += 32) {
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const float y0 = ex2(fmaf(asf(s[i + e]), p.scale, -base));
                        const float y1 = ex2(fmaf(asf(s[i + e + 1]), p.scale, -base));
                        l0 += y0;
                        l1 += y1;
                        pk[e / 2] = pack(y0, y1);
                    }
                    tmem_st16<0>(t_row + C::P0 + i / 2, pk);
                }
                l += l0 + l1;
                tmem_stored();
                fence_before();
                bar_arrive(&c->p_full[w]);
                ++done;
            } else {
                float mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < KT; i += 32) {
                    uint32_t s[32];
                    tmem_ld32<0>(t_row + C::S + i, s);
                    tmem_landed(s);
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (see[i / 32] >> e & 1u) mx = fmaxf(mx, asf(s[e]));
                }
                const float m_new = fmaxf(m, mx * p.scale);
                const float alpha = m == -INFINITY ? 0.f : ex2(m - m_new);
                m = m_new;
                const float base = m == -INFINITY ? 0.f : m;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < KT; i += 32) {
                    uint32_t s[32], pk[16];
                    tmem_ld32<0>(t_row + C::S + i, s);
                    tmem_landed(s);
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const float y = see[i / 32] >> e & 1u ? ex2(fmaf(asf(s[e]), p.scale, -base)) : 0.f;
                        sum += y;
                        s[e] = __float_as_uint(y);
                    }
#pragma unroll
                    for (int pl = 0; pl < 3; ++pl) {
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float y0 = asf(s[e]), y1 = asf(s[e + 1]);
                            pk[e / 2] = peel(y0, y1);
                            s[e] = __float_as_uint(y0);
                            s[e + 1] = __float_as_uint(y1);
                        }
                        tmem_st16<0>(t_row + (pl == 0 ? C::P0 : pl == 1 ? C::P1 : C::P2) + i / 2, pk);
                    }
                }
                l = fmaf(l, alpha, sum);
                tmem_stored();
                fence_before();
                bar_arrive(&c->p_full[w]);
                // ---- O of this tile, added in fp32
                if (!(ok = warp_wait(c, &c->pv_done[w], done & 1, 7))) break;
                ++done;
                fence_after();
#pragma unroll
                for (int i = 0; i < D; i += 32) {
                    uint32_t y[32];
                    tmem_ld32<0>(t_row + C::O + i, y);
                    tmem_landed(y);
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[i + e] = fmaf(o[i + e], alpha, asf(y[e]));
                }
            }
        }
        if (NP == 1 && ok && done) {
            ok = warp_wait(c, &c->pv_done[w], (done - 1) & 1, 8);
            fence_after();
        }
        // ---- QT = 1: stream 1 hands its state to stream 0 through the ring, which nothing uses
        // any more once both streams' last products are complete
        float keep = 1.f, take = 0.f;
        float* join = reinterpret_cast<float*>(sm + C::Q_BYTES);  // [D][128]
        float* join_ml = reinterpret_cast<float*>(sm);            // [2][128], where the queries were
        if constexpr (QT == 1) {
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (w == 1) {
                join_ml[r] = m;
                join_ml[128 + r] = l;
#pragma unroll
                for (int i = 0; i < D; i += 32) {
                    uint32_t y[32];
                    if constexpr (NP == 1) {
                        if (done) {
                            tmem_ld32<0>(t_row + C::O + i, y);
                            tmem_landed(y);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        float v;
                        if constexpr (NP == 1) v = done ? asf(y[e]) : 0.f; else v = o[i + e];
                        join[(i + e) * 128 + r] = v;
                    }
                }
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (w == 0) {
                const float m1 = join_ml[r], mt = fmaxf(m, m1);
                keep = m == -INFINITY ? 0.f : ex2(m - mt);
                take = m1 == -INFINITY ? 0.f : ex2(m1 - mt);
                l = l * keep + join_ml[128 + r] * take;
            }
        }
        if (ok && (QT == 2 || w == 0)) {
            const float inv = l == 0.f ? 0.f : 1.0f / l;  // a row that sees nothing: zeros
            T* out = og + row_at(live ? base_tok + tk : 0, live ? r % heads : 0);
#pragma unroll
            for (int i = 0; i < D; i += 32) {
                uint32_t y[32];
                if constexpr (NP == 1) {
                    if (done) {  // the same for a warp: all its lanes load
                        tmem_ld32<0>(t_row + C::O + i, y);
                        tmem_landed(y);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) y[e] = 0u;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) y[e] = __float_as_uint(o[i + e]);
                }
                if (live) {
                    if constexpr (QT == 1) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            y[e] = __float_as_uint(asf(y[e]) * keep + join[(i + e) * 128 + r] * take);
                    }
                    if constexpr (NP == 1) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint32_t u[4];
#pragma unroll
                            for (int x = 0; x < 4; ++x)
                                u[x] = pack(asf(y[e + 2 * x]) * inv, asf(y[e + 2 * x + 1]) * inv);
                            *reinterpret_cast<uint4*>(out + i + e) = make_uint4(u[0], u[1], u[2], u[3]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            *reinterpret_cast<float4*>(out + i + e) = make_float4(
                                asf(y[e]) * inv, asf(y[e + 1]) * inv, asf(y[e + 2]) * inv, asf(y[e + 3]) * inv);
                    }
                }
                __syncwarp();
            }
        }
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    if (warp == 12) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    if (c->bad && warp < 8 && !c->abort) {
        for (int i = warp; i < tokens * heads; i += 8) {
            const int64_t at = ((int64_t)(row0 + i / heads) * a.Hq + kvh * G + head0 + i % heads) * D;
            walk_row<D, T>(a, req, kvh, pos0 + i / heads, static_cast<const T*>(a.q) + at, static_cast<T*>(a.o) + at);
        }
    }
}

template <int D, int NP, int QT, typename T>
cudaError_t launch_t(const PrefillArgs& p, cudaStream_t st) {
    using C = Cfg<D, NP, QT>;
    static std::atomic<uint64_t> ready{0};  // devices whose limit has been raised, one bit each
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !(ready.load() >> dev & 1)) {
        e = cudaFuncSetAttribute(window_prefill_kernel<D, NP, QT, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 C::BYTES);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready.fetch_or(1ull << dev);
    }
    const int64_t tiles = p.a.rows / (QT * p.tok) + p.a.n_prompts;  // at least the sum over prompts
    const int64_t blocks = std::min<int64_t>(tiles, p.a.rows) * p.a.Hkv * p.groups;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    window_prefill_kernel<D, NP, QT, T><<<(unsigned)blocks, kThreads, C::BYTES, st>>>(p);
    return cudaGetLastError();
}

template <int D>
cudaError_t launch_d(const PrefillArgs& p, bool f32, cudaStream_t st) {
    if (f32) return launch_t<D, 3, 1, float>(p, st);
    // two row tiles per block once that leaves no SM without a block
    const int64_t tiles = ((int64_t)p.a.rows / p.tok + p.a.n_prompts) * p.a.Hkv * p.groups;
    return tiles >= 2 * kSms ? launch_t<D, 1, 2, __nv_bfloat16>(p, st) : launch_t<D, 1, 1, __nv_bfloat16>(p, st);
}

}  // namespace

uint64_t window_prefill_scratch(int M, int n_prompts, int Hq, int Hkv, int d, int window, int sinks, int max_ctx) {
    return 16;
}

cudaError_t launch_window_prefill(const WindowArgs& a, bool f32, cudaStream_t st) {
    PrefillArgs p{};
    p.a = a;
    p.a.window = std::min(a.window, 1 << 30);  // positions are below max_ctx <= 2^30
    p.a.sinks = std::min(a.sinks, 1 << 30);
    const int G = a.Hq / a.Hkv;
    p.groups = (G + 127) / 128;
    p.heads = (G + p.groups - 1) / p.groups;
    p.tok = 128 / p.heads;
    p.scale = (float)(1.4426950408889634 / sqrt((double)a.d));
    return a.d == 128 ? launch_d<128>(p, f32, st) : launch_d<64>(p, f32, st);
}

cudaError_t window_prefill_error(int* code) { return cudaMemcpyFromSymbol(code, g_window_error, sizeof(int)); }

}  // namespace loip
