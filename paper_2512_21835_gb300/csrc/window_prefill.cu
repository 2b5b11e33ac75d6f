// window_prefill.cu -- attention of prompt rows over the paged cache, behind a
// sliding window with sinks, on the 5th-generation tensor cores.
//
// Rows.  The `heads` query heads that share a kv head are packed with consecutive
// positions into the 128 rows of an MMA tile (row = token * heads + head), so a
// tile spans 128 / heads positions: keys and values are read once for all heads,
// and a window costs little more than its own length.
//
// Keys.  The pages that some row of the block sees, those of the sinks and then
// those of the window, are a list without a gap; a page is a key tile.  Positions
// that no row of the block sees are not read: their rows in shared memory are
// zero-filled.
//
// Per key tile:  S = Q K^T -> tensor memory -> softmax in registers, one row per
// thread -> P back into tensor memory -> O += P V, V in its cache layout
// (the MMA takes B with d contiguous).  Two streams w = 0, 1 of this chain share the
// tensor core:
//   QT = 2: two row tiles over the same key tiles
//   QT = 1: one row tile, even and odd key tiles; the two partial softmax states are
//           joined at the end.  For fewer row tiles than the card has places; with
//           fewer still, a row tile's pages are split over several blocks, which
//           leave their states in scratch for a second kernel to join.  (Joined by the
//           last block to arrive, 16 row tiles in 9 parts each took 22 us: that block
//           reads 590 KB alone.)
// S and P have columns of their own (P twice for bf16 rows), so the next tile's S is
// computed while this one's weights are, and neither waits for P V.  (With P over S, in
// tiles of 128 keys, the chain softmax - P V - S took 4000 cycles per 128 keys and two
// streams, of which the tensor core worked 2048: an isolated group of eight MMAs answers
// after 840.)  The price is N = 64 for S, 48 cycles an MMA instead of 32: 2560 cycles.
//
// Measured (GB300): 8192 bf16 rows of 32 heads of 128 behind a 4096-token window 444 us,
// 1240 TFLOP/s, tensor pipe active 54%; bound by the chain from P of a tile to S of the
// next but one (waits, issue and answer, 1700 cycles per tile of which the tensor core
// works 1280).  4 x 512 fp32 rows of 64 heads 111 us: half of a block's time is its
// queries, its join and its outputs.  8192 fp32 rows 1330 us.  The registers (168) do not
// hold everything: in the tile loop a softmax warp reloads two or three spilled words a tile
// and stores none.
//
// Precision.  bf16 rows: one MMA per product, weights rounded to bf16 (2^-9: the outputs are
// off by 0.0021 of their size, of which their own rounding is 0.0017; a second plane would
// double the MMAs of P V), O stays in tensor memory; it is rescaled only when a row's
// maximum has grown by 2^8 (weights are relative to an older maximum until then, exact in
// the end).  fp32 rows (NP = 3):
// queries and weights are exact sums of three bf16 planes, three MMAs per product,
// smallest plane first; the tensor core's sums truncate, so O of one key tile is
// drained and added in fp32 registers.
//
// A value that is not finite would spoil rows that do not see it (0 x inf).  In key
// tiles that not all rows see in full, the loader looks for such values, zeroes them
// and flags the block, whose rows are then walked one by one (walk_row).
//
// Roles (384 threads): warps 0-3 and 4-7 softmax of stream 0 and 1 (one row per
// thread), warps 8 and 9 load (cp.async, 128-byte swizzle), warps 10 and 11 issue the
// MMAs of a stream each.  Beside the softmax a barrier operation of an issuing warp takes
// 130 cycles, even a wait for a phase that is complete, and the tensor core's queue is
// two MMAs deep; so the keys of a tile share a slot and a barrier with the values that
// are used in the same step, and each stream has a warp.
// Every wait is bounded (2 s); one that runs out records an error, the block stops,
// lets its copies and MMAs finish, frees its tensor memory and returns.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "internal.h"
#include "window.h"
#include "window_parts.h"

namespace loip {

__device__ int g_window_error;  // first failure code of any launch (0 = none)

namespace {

constexpr int kThreads = 384;
constexpr int kLoaders = 64;                     // threads of warps 8 and 9
constexpr int kSms = 152;
constexpr int kSoftRegs = 200, kOtherRegs = 104;  // 256 x 200 + 128 x 104 = 384 x 168
constexpr int KT = kPageTokens;                  // keys per tile

template <int D, int NP, int QT>
struct Cfg {
    static constexpr int SLABS = D / 64;               // 128-byte columns of a row
    static constexpr int Q_SLAB = 128 * 128;
    static constexpr int Q_PLANE = SLABS * Q_SLAB;
    static constexpr int Q_BYTES = QT * NP * Q_PLANE;  // [tile][plane][slab][row]
    static constexpr int KV_SLAB = KT * 128;
    static constexpr int TILE = SLABS * KV_SLAB;       // one tile of keys or of values
    static constexpr int SLOT = 2 * TILE;              // the keys of one tile, the values of an earlier one
    static constexpr int ROOM = 227 * 1024 - 1024 - 512 - Q_BYTES;
    static constexpr int MOST = ROOM / SLOT < 12 ? ROOM / SLOT : 12;
    static constexpr int SLOTS = QT == 2 ? MOST : MOST / 2 * 2;  // (a stream's own slots: every second one)
    static constexpr int AHEAD = 3 - QT;                 // slot i: keys of tile i, values of tile i - AHEAD
    static constexpr int CTL = Q_BYTES + SLOTS * SLOT;
    static constexpr int BYTES = CTL + 512 + 1024;     // + alignment of the window
    static_assert(SLOTS >= 3, "the loader may signal a slot after it has filled the next");
    static_assert(QT == 2 || SLOTS * SLOT >= 128 * (D + 8) * 4 + 2048, "the join goes through the ring");
    // Tensor memory.  bf16: per stream S, two P buffers and O.  fp32: one O, drained after
    // every tile, then per stream S and the planes of P.
    __host__ __device__ static constexpr uint32_t s_col(int w) { return NP == 1 ? 256 * w : 128 + 160 * w; }
    __host__ __device__ static constexpr uint32_t o_col(int w) { return NP == 1 ? 256 * w + 128 : 0; }
    __host__ __device__ static constexpr uint32_t p_col(int w, int buf, int pl) {
        return s_col(w) + 64 + 32 * (NP == 1 ? buf : pl);
    }
};

struct Ctl {  // control words behind the ring
    uint64_t full[12], empty[12];      // of the ring's slots
    uint64_t s_full[2], s_free[2];     // per stream
    uint64_t p_full[4], pv_done[4];    // per stream and P buffer: for even and odd tiles, no wait is ever two phases behind
    uint64_t o_free, q_full, end;
    uint32_t tmem;
    int abort, bad;
    int row0, tokens, req, pos0;
};
static_assert(sizeof(Ctl) <= 512, "");

struct PrefillArgs {
    WindowArgs a;
    int heads, groups;  // query heads per row tile, groups per kv head
    int tok;            // positions per row tile
    int splits;         // blocks per row tile (QT = 1)
    float scale;        // log2(e) / sqrt(d)
    // in scratch, with splits; a unit is a row tile and kv head (and group)
    float4* part;       // [unit][split][d / 4][128 rows], not normalised
    int4* rows;         // [unit]: first row, tokens, request, position of the first
    float2* ml;         // [unit][split][128 rows]: maximum (log2), sum
    unsigned* ended;    // [unit][split]: PartEnd
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// Barriers by their address in shared memory.
__device__ __forceinline__ void bar_init(uint32_t b, uint32_t n) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(b), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(b) : "memory");
}
// Whether the phase of that parity is complete; waits for it up to a millisecond, asleep.
// (Without the hint the wait ended after some hundred cycles, and the waiting warps'
// polls took issue slots and shared memory from the others.)
__device__ __forceinline__ bool bar_try(uint32_t b, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(b), "r"(parity), "r"(1000000u)
        : "memory");
    return ok != 0;
}
// A thread's waits.  One that runs out (2 s), or the flag of another thread's that did,
// ends all further ones: the thread goes on to its end with whatever it finds, within
// its own buffers.  (No way out in between: a warp stays together, and the code of a wait is
// one instruction and a branch.)  From then on the block stores no row of o (`stopped`, asked
// behind a barrier that the waiting threads have passed), and for a split row tile the kernel
// that joins the parts stores none either (`ended`): those rows stay as they were.
struct Waiter {
    Ctl* c;
    bool dead;
    __device__ __forceinline__ void operator()(uint32_t b, uint32_t parity, int code) {
        if (!dead && !bar_try(b, parity)) slow(b, parity, code);
    }
    __device__ __forceinline__ void slow(uint32_t b, uint32_t parity, int code) {
        const uint64_t t0 = now_ns();
        while (!bar_try(b, parity)) {
            dead = *(volatile int*)&c->abort != 0;
            if (!dead && now_ns() - t0 > 2000000000ull) {
                *(volatile int*)&c->abort = 1;
                atomicCAS(&g_window_error, 0, code);
                dead = true;
            }
            if (dead) return;
        }
    }
};
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
// Copies that have arrived at a barrier, made visible to the tensor core's reads.
__device__ __forceinline__ void fence_loaded() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The MMA warp runs as a whole; its issuing instructions are predicated on the elected
// lane inside one asm block, so that addresses and descriptors stay warp-uniform.  Issued
// from a lane's own branch they took 130 cycles each, twice what an MMA of 128 columns
// takes the tensor core.
__device__ __forceinline__ void commit(uint32_t b) {
    asm volatile(
        "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n"
        " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(b)
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
// Two MMAs (32 of K): A in tensor memory, 8 columns a step; B 16 rows of 128 bytes a step.
__device__ __forceinline__ void mma_ts2(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t acc) {
    asm volatile(
        "{\n .reg .pred e, p, t;\n .reg .b32 a1;\n .reg .b64 b1;\n"
        " elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n setp.eq.b32 t, %4, %4;\n"
        " add.s32 a1, %1, 8;\n add.s64 b1, %2, 128;\n"
        " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
        " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, t;\n}\n" ::"r"(d),
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
// two fp32 lanes in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{\n .reg .b64 a, b, c;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
        " fma.rn.f32x2 a, a, b, c;\n mov.b64 {%0, %1}, a;\n}\n"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{\n .reg .b64 a, b;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n"
        " add.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a;\n}\n"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
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
        const float m_new = fmaxf(m, s), alpha = m == -INFINITY ? 0.f : expf(m - m_new);
        const float w = expf(s - (m_new == -INFINITY ? 0.f : m_new));  // a score of -inf: weight zero, the first one too
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
    const WindowArgs& a = p.a;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    Ctl* c = reinterpret_cast<Ctl*>(sm + C::CTL);
    const uint32_t q_smem = smem_u32(sm), ring = q_smem + C::Q_BYTES, ctl = q_smem + C::CTL;
    const uint32_t bar_full = ctl + offsetof(Ctl, full), bar_empty = ctl + offsetof(Ctl, empty),
                   bar_s = ctl + offsetof(Ctl, s_full), bar_s_free = ctl + offsetof(Ctl, s_free),
                   bar_p = ctl + offsetof(Ctl, p_full), bar_pv = ctl + offsetof(Ctl, pv_done),
                   bar_o_free = ctl + offsetof(Ctl, o_free), bar_q = ctl + offsetof(Ctl, q_full),
                   bar_end = ctl + offsetof(Ctl, end);
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;

    // ---- which rows: splits fastest, then kv heads (and groups of their heads), then
    // prompts and row tiles from the last, whose rows see the most
    const int units = a.Hkv * p.groups;
    const int split = QT == 1 ? blockIdx.x % p.splits : 0;
    const int unit = QT == 1 ? blockIdx.x / p.splits : blockIdx.x;  // row tile and kv head (and group)
    const int kvh = unit % units / p.groups, head0 = unit % units % p.groups * p.heads;
    const int G = a.Hq / a.Hkv, heads = min(p.heads, G - head0);
    pdl_trigger();
    if (warp == 0) {
        pdl_wait();
        int left = unit / units;  // row tiles from the end
        int row0 = 0, tokens = 0, req = 0, pos0 = 0;
        for (int top = a.n_prompts - 1; top >= 0; top -= 32) {
            const int i = top - lane;
            int lo = 0, hi = 0, at = 0;
            if (i >= 0) {
                if (a.first_pos) at = a.first_pos[i];
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
                    pos0 = min(max(at, -(1 << 30)), 1 << 30) + first;
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
        }
    } else if (warp == 8) {
        if (lane == 0) {
            c->abort = 0;
            c->bad = 0;
            for (int i = 0; i < C::SLOTS; ++i) {
                bar_init(bar_full + 8 * i, kLoaders);
                bar_init(bar_empty + 8 * i, QT);
            }
            for (int w = 0; w < 2; ++w) {
                bar_init(bar_s + 8 * w, 1);
                bar_init(bar_s_free + 8 * w, 128);
            }
            for (int i = 0; i < 4; ++i) {
                bar_init(bar_p + 8 * i, 128);
                bar_init(bar_pv + 8 * i, 1);
            }
            bar_init(bar_o_free, 128);
            bar_init(bar_q, 256);
            bar_init(bar_end, 2);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
    } else if (warp == 10) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&c->tmem)),
                     "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = c->tmem;
    const int row0 = c->row0, tokens = c->tokens, req = c->req, pos0 = c->pos0;

    const int pos1 = pos0 + tokens - 1;
    const Pages pages(a, pos0, pos1);
    // this block's part of the list (the grid is an upper bound: blocks without rows have none)
    const int begin = tokens == 0 ? 0 : (int)((int64_t)pages.n * split / p.splits);
    const int n = tokens == 0 ? 0 : (int)((int64_t)pages.n * (split + 1) / p.splits) - begin;
    auto page_at = [&](int t) { return pages.at(begin + t); };
    // the rows of stream w: its row tile's
    auto stream_pos = [&](int w) { return QT == 2 ? pos0 + w * p.tok : pos0; };
    auto stream_tokens = [&](int w) { return QT == 2 ? min(max(tokens - w * p.tok, 0), p.tok) : tokens; };
    // the key tiles that stream w computes (QT = 2): [0, sink) and [lo, hi)
    struct Takes {
        int sink, lo, hi;
        __device__ bool operator()(int t) const { return t < sink || (t >= lo && t < hi); }
    };
    auto takes_of = [&](int w) {
        Takes k{0, 0, 0};
        if (stream_tokens(w) > 0) {
            const Pages mine(a, stream_pos(w), stream_pos(w) + stream_tokens(w) - 1);
            const int shift = pages.sink - pages.win;  // of a window page in the list
            k.sink = min(mine.sink, pages.sink);
            k.lo = max(mine.win, pages.win) + shift;
            k.hi = mine.end + shift;
        }
        return k;
    };

    Waiter wait{c, false};
    auto stopped = [&] { return *(volatile int*)&c->abort != 0; };
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp < 10) {
            // ---------------------------------------------------------------- loader
            const int lt = tid - 256;
            constexpr int CPR = D / 8, RPP = kLoaders / CPR;  // 16-byte chunks per row, rows per pass
            constexpr int PASSES = KT / RPP;
            const int chunk = lt % CPR, r0 = lt / CPR;
            const char* layer = a.kv.base + (uint64_t)a.kv.layer * a.kv.layer_page_bytes;
            const int64_t* table = a.kv.page_offsets + (int64_t)req * a.kv.max_pages;
            const int win0 = max(0, pos0 - a.window + 1);  // (window 0: no page of it is in the list)
            auto seen = [&](int pos) {
                return pos < pages.last && ((pos >= win0 && a.window > 0) || pos < a.sinks);
            };
            // place in a slot of this thread's chunk of pass k: row r0 + k RPP, chunk ^ row % 8
            static_assert(RPP == 4 || RPP == 8, "");
            const uint32_t place0 = (uint32_t)((chunk >> 3) * C::KV_SLAB + r0 * 128 + (((chunk & 7) ^ (r0 & 7)) << 4));
            const uint32_t place1 = RPP == 8 ? place0 : place0 ^ 64;  // odd passes: row % 8 differs by 4
            auto place = [&](int k) { return (k & 1 ? place1 : place0) + k * RPP * 128; };
            // Slots arrive at their barrier by themselves, except with values of a page that not all rows
            // see in full: of those, the ones that are not finite are taken out first, one slot later.
            auto checked = [&](uint32_t slot) {
                for (int k = 0; k < PASSES; ++k) {
                    const uint32_t w = ring + slot * C::SLOT + C::TILE + place(k);
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
                bar_arrive(bar_full + 8 * slot);
            };
            constexpr int STEP = RPP * D * 2;  // bytes from a pass to the next in the page
            auto load = [&](int t, bool is_v, uint32_t dst) {
                const int pg = page_at(t), b = pg * KT;
                const char* src = layer + table[pg] + ((int64_t)(is_v ? a.Hkv : 0) + kvh) * (KT * D * 2) +
                                  (r0 * D + chunk * 8) * 2;
                if (b + KT <= pages.last && ((b >= win0 && a.window > 0) || b + KT <= a.sinks)) {  // the whole page
#pragma unroll
                    for (int k = 0; k < PASSES; ++k) cp_async16(dst + place(k), src + k * STEP, 16u);
                } else {
#pragma unroll 2
                    for (int k = 0; k < PASSES; ++k) {
                        const bool ok = seen(b + r0 + k * RPP);
                        cp_async16(dst + place(k), ok ? src + k * STEP : layer, ok ? 16u : 0u);
                    }
                }
            };
            int slot = 0, late = -1;  // late: the slot before, if it is yet to be checked
            uint32_t free_phase = 1;  // of the ring's previous round (before the first one: complete)
#pragma unroll 1
            for (int i = 0; i < n + C::AHEAD && n > 0; ++i) {
                const int t = i - C::AHEAD;  // whose values
                const uint32_t dst = ring + (uint32_t)slot * C::SLOT;
                wait(bar_empty + 8 * slot, free_phase, 1);
                if (i < n) load(i, false, dst);
                bool some = false;
                if (t >= 0) {
                    load(t, true, dst + C::TILE);
                    const int b = page_at(t) * KT;
                    some = !(b + KT - 1 <= pos0 && (b > pos1 - a.window || b + KT <= a.sinks));
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                if (!some)
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar_full + 8 * slot)
                                 : "memory");
                if (late >= 0) {
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    checked(late);
                }
                late = some ? slot : -1;
                if (++slot == C::SLOTS) {
                    slot = 0;
                    free_phase ^= 1;
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (late >= 0) checked(late);
        } else if (n > 0) {
            // ---------------------------------------------------------------- MMA issue
            const int w = warp - 10;  // the stream
            const Takes takes = takes_of(w);
            auto mine = [&](int t) { return t >= 0 && t < n && (QT == 1 ? (t & 1) == w : takes(t)); };
            const uint64_t q_desc = sdesc(q_smem + (QT == 2 ? w * NP * C::Q_PLANE : 0), 16), k_desc = sdesc(ring, 16),
                           v_desc = sdesc(ring + C::TILE, C::KV_SLAB);
            constexpr int STRIDE = QT == 2 ? 1 : 2;  // a slot's keys and values are of both streams, or of one
            uint32_t slot = QT == 2 ? 0 : w, phase = 0;  // a cursor in the ring, and the phase of its round
            uint32_t free = 1;                // of S (before the first tile: complete)
            uint32_t done = 0;                // products P V
            int used = -1;                    // slot to be released (QT = 2)
            const int steps = n + C::AHEAD;
            wait(bar_q, 0, 2);
            if (QT == 2 || w < steps) wait(bar_full + 8 * slot, phase, 3);
            // From P of a tile to S of the next but one the stream waits for this warp, so with two row
            // tiles the next slot is waited for before P, and the last one released after S (467 -> 454
            // us for 8192 rows behind 4096).  With one row tile a stream has two slots, and there the
            // release has to come first (4 x 512 fp32 rows: 109 us, 121 the other way).
#pragma unroll 1
            for (int i = QT == 2 ? 0 : w; i < steps; i += STRIDE) {
                const uint32_t k_at = slot * (C::SLOT / 16);
                fence_loaded();
                if (mine(i)) {  // S = Q K^T, once the softmax has read the last one
                    wait(bar_s_free + 8 * w, free, 4);
                    free ^= 1;
                    fence_after();
                    const uint64_t k = k_desc + k_at;
#pragma unroll
                    for (int pl = NP - 1; pl >= 0; --pl)
#pragma unroll
                        for (int x = 0; x < D / 64; ++x)
                            mma_ss4(tmem + C::s_col(w), q_desc + (pl * C::Q_PLANE + x * C::Q_SLAB) / 16,
                                    k + x * C::KV_SLAB / 16, idesc(KT, false), pl != NP - 1 || x != 0);
                    commit(bar_s + 8 * w);
                }
                if (QT == 2 && used >= 0) commit(bar_empty + 8 * used);
                used = slot;
                slot += STRIDE;
                if (slot >= C::SLOTS) {
                    slot -= C::SLOTS;
                    phase ^= 1;
                }
                if (QT == 2 && i + STRIDE < steps) wait(bar_full + 8 * slot, phase, 3);
                if (mine(i - C::AHEAD)) {  // O += P V
                    const uint32_t buf = done & 1;
                    wait(bar_p + 16 * w + 8 * buf, done / 2 & 1, 5);
                    // O is one for both streams: the other one's last tile has been drained.  (This
                    // stream's own last one has, as its P is here, so the phase is the right one.)
                    if (NP > 1) wait(bar_o_free, (i - C::AHEAD + 1) & 1, 9);
                    fence_after();
                    const uint64_t v = v_desc + k_at;
#pragma unroll
                    for (int pl = NP - 1; pl >= 0; --pl)
#pragma unroll
                        for (int x = 0; x < 2; ++x)  // O is kept (bf16), or drained after every tile
                            mma_ts2(tmem + C::o_col(w), tmem + C::p_col(w, buf, pl) + 16 * x,
                                    v + x * (32 * 128 / 16), idesc(D, true),
                                    pl != NP - 1 || x != 0 || (NP == 1 && done) ? 1u : 0u);
                    commit(bar_pv + 16 * w + 8 * buf);
                    ++done;
                }
                if (QT == 1) {
                    commit(bar_empty + 8 * used);
                    if (i + STRIDE < steps) wait(bar_full + 8 * slot, phase, 3);
                }
            }
            // nothing may be in flight when the tensor memory is released
            commit(bar_end);
            const uint64_t t0 = now_ns();
            while (!bar_try(bar_end, 0) && now_ns() - t0 < 2000000000ull) {}
        }
    } else if (tokens > 0) {
        // -------------------------------------------------------------------- softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
        const T* qg = static_cast<const T*>(a.q);
        T* og = static_cast<T*>(a.o);
        auto row_at = [&](int tok, int head) {  // element offset of a row of q and o
            return ((int64_t)(row0 + tok) * a.Hq + kvh * G + head0 + head) * D;
        };
        const uint32_t per_head = 65536u / heads + 1;  // row / heads for rows below 128, without a division
        auto tok_of = [&](int row) { return (int)(row * per_head >> 16); };
        // ---- queries -> shared memory, bf16 planes, swizzled; all of a thread's loads in flight
        constexpr int CPR = D / 8, EACH = QT * 128 * CPR / 256, MOST = NP == 1 ? 16 : 8, BATCH = EACH < MOST ? EACH : MOST;
        static_assert(EACH % BATCH == 0, "");
        for (int i0 = tid; i0 < QT * 128 * CPR; i0 += 256 * BATCH) {
            uint4 x[BATCH], y[NP == 1 ? 1 : BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int i = i0 + 256 * k, r = i / CPR % 128, tile = i / CPR / 128;
                const int tk = tok_of(r), tok = tile * p.tok + tk;
                x[k] = make_uint4(0u, 0u, 0u, 0u);
                if constexpr (NP > 1) y[k] = x[k];
                if (tk < p.tok && tok < tokens) {
                    const uint4* src = reinterpret_cast<const uint4*>(qg + row_at(tok, r - tk * heads) + i % CPR * 8);
                    x[k] = src[0];
                    if constexpr (NP > 1) y[k] = src[1];
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
                        for (int e = 0; e < 4; ++e)
                            u[e] = pl < 2 ? peel(v[2 * e], v[2 * e + 1]) : pack(v[2 * e], v[2 * e + 1]);
                        *reinterpret_cast<uint4*>(dst + pl * C::Q_PLANE) = make_uint4(u[0], u[1], u[2], u[3]);
                    }
                }
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        bar_arrive(bar_q);

        const int w = warp / 4, r = tid % 128;
        const int base_tok = QT == 2 ? w * p.tok : 0, mine = stream_tokens(w);
        const int tk = tok_of(r);
        const bool live = tk < min(p.tok, mine);
        const int pos = live ? pos0 + base_tok + tk : -1;
        const int first = pos0 + base_tok, final = first + mine - 1;  // positions of the stream's rows
        // key tiles [full0, full1) of the window are seen in full by all of the stream's rows
        const int list0 = pages.sink - pages.win - begin;  // tile of page 0, were it in the window's part
        const int full0 = max(pages.win, final - a.window < 0 ? 0 : (final - a.window) / KT + 1) + list0;
        const int full1 = max(min(first + 1, pages.last), 0) / KT + list0;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;  // this warp's lanes of tensor memory
        float m = -INFINITY, l = 0.f;  // m: the maximum that the weights are relative to
        uint32_t done = 0;             // tiles computed
        // P V of the stream's tile j is complete (j the last or the last but one whose P is handed over,
        // or -2 or -1: complete)
        auto pv_wait = [&](uint32_t j, int code) { wait(bar_pv + 16 * w + 8 * (j & 1), (uint32_t)((int)j >> 1) & 1, code); };
        float o[NP == 1 ? 1 : D];
        if constexpr (NP > 1) {
#pragma unroll
            for (int i = 0; i < D; ++i) o[i] = 0.f;
        }
        const Takes takes = takes_of(w);
        for (int t = QT == 1 ? w : 0; t < n; t += QT == 1 ? 2 : 1) {
            if (QT == 2 && !takes(t)) continue;
            // which positions of the page this row sees, one bit each
            const bool masked = t < full0 || t >= full1;
            uint32_t see[2] = {0xffffffffu, 0xffffffffu};
            if (masked) {
                const int b = page_at(t) * KT;
                const uint64_t bits =
                    live ? low_bits(min(pos, a.max_ctx - 1) - b + 1) &
                               (~low_bits(pos - a.window + 1 - b) | low_bits(a.sinks - b))
                         : 0ull;
                see[0] = (uint32_t)bits;
                see[1] = (uint32_t)(bits >> 32);
            }
            const uint32_t buf = done & 1;
            wait(bar_s + 8 * w, done & 1, 6);
            __syncwarp();
            fence_after();
            const uint32_t s_at = tmem + lanes + C::s_col(w);
            if constexpr (NP == 1) {
                uint32_t s[KT];
                tmem_ld32<0>(s_at, s);
                tmem_ld32<32>(s_at + 32, s);
                tmem_landed(s);
                fence_before();
                bar_arrive(bar_s_free + 8 * w);
                pv_wait(done - 2, 8);  // P of that tile is free
                __syncwarp();
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
                // O is rescaled when a row's maximum has outgrown the one in use by 2^8
                const bool grown = mx > m + 8.f;  // the first time too: m is -inf
                if (__any_sync(0xffffffffu, grown)) {
                    const float m_new = grown ? mx : m;
                    const float alpha = m == -INFINITY ? 0.f : ex2(m - m_new);
                    m = m_new;
                    l *= alpha;
                    if (done) {
                        pv_wait(done - 1, 8);
                        __syncwarp();
                        fence_after();
#pragma unroll
                        for (int i = 0; i < D; i += 32) {
                            uint32_t y[32];
                            tmem_ld32<0>(tmem + lanes + C::o_col(w) + i, y);
                            tmem_landed(y);
#pragma unroll
                            for (int e = 0; e < 32; ++e) y[e] = __float_as_uint(asf(y[e]) * alpha);
                            tmem_st16<0>(tmem + lanes + C::o_col(w) + i, y);
                            tmem_st16<16>(tmem + lanes + C::o_col(w) + i + 16, y);
                        }
                    }
                }
                const float base = m == -INFINITY ? 0.f : m;
                const float2 scale2 = make_float2(p.scale, p.scale), base2 = make_float2(-base, -base);
                float2 l0 = make_float2(0.f, 0.f), l1 = l0;
#pragma unroll
                for (int i = 0; i < KT; i += 32) {
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        float2 y = fma2(make_float2(asf(s[i + e]), asf(s[i + e + 1])), scale2, base2);
                        float2 z = fma2(make_float2(asf(s[i + e + 2]), asf(s[i + e + 3])), scale2, base2);
                        y.x = ex2(y.x); y.y = ex2(y.y); z.x = ex2(z.x); z.y = ex2(z.y);
                        l0 = add2(l0, y);
                        l1 = add2(l1, z);
                        pk[e / 2] = pack(y.x, y.y);
                        pk[e / 2 + 1] = pack(z.x, z.y);
                    }
                    tmem_st16<0>(tmem + lanes + C::p_col(w, buf, 0) + i / 2, pk);
                }
                l0 = add2(l0, l1);
                l += l0.x + l0.y;
                tmem_stored();
                fence_before();
                bar_arrive(bar_p + 16 * w + 8 * buf);
                ++done;
            } else {
                float mx = -INFINITY;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t s[32];
                    tmem_ld32<0>(s_at + 32 * h, s);
                    tmem_landed(s);
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!(see[h] >> e & 1u)) s[e] = 0xff800000u;
                    }
                    float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        x0 = fmaxf(x0, fmaxf(asf(s[e]), asf(s[e + 1])));
                        x1 = fmaxf(x1, fmaxf(asf(s[e + 2]), asf(s[e + 3])));
                    }
                    mx = fmaxf(mx, fmaxf(x0, x1));
                }
                const float m_new = fmaxf(m, mx * p.scale);
                const float alpha = m == -INFINITY ? 0.f : ex2(m - m_new);
                m = m_new;
                const float base = m == -INFINITY ? 0.f : m;
                const float2 scale2 = make_float2(p.scale, p.scale), base2 = make_float2(-base, -base);
                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t s[32], pk[16];
                    tmem_ld32<0>(s_at + 32 * h, s);
                    tmem_landed(s);
                    if (h == 1) {
                        fence_before();
                        bar_arrive(bar_s_free + 8 * w);
                    }
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!(see[h] >> e & 1u)) s[e] = 0xff800000u;
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float2 y = fma2(make_float2(asf(s[e]), asf(s[e + 1])), scale2, base2);
                        y.x = ex2(y.x); y.y = ex2(y.y);
                        sum = add2(sum, y);
                        s[e] = __float_as_uint(y.x);
                        s[e + 1] = __float_as_uint(y.y);
                    }
#pragma unroll
                    for (int pl = 0; pl < 3; ++pl) {
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float y0 = asf(s[e]), y1 = asf(s[e + 1]);
                            pk[e / 2] = pl < 2 ? peel(y0, y1) : pack(y0, y1);
                            s[e] = __float_as_uint(y0);
                            s[e + 1] = __float_as_uint(y1);
                        }
                        tmem_st16<0>(tmem + lanes + C::p_col(w, 0, pl) + 16 * h, pk);
                    }
                }
                l = fmaf(l, alpha, sum.x + sum.y);
                tmem_stored();
                fence_before();
                bar_arrive(bar_p + 16 * w + 8 * buf);
                // ---- O of this tile, added in fp32
                pv_wait(done, 7);
                __syncwarp();
                ++done;
                fence_after();
#pragma unroll
                for (int i = 0; i < D; i += 32) {
                    uint32_t y[32];
                    tmem_ld32<0>(tmem + lanes + C::o_col(w) + i, y);
                    tmem_landed(y);
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[i + e] = fmaf(o[i + e], alpha, asf(y[e]));
                }
                fence_before();
                bar_arrive(bar_o_free);
            }
        }
        if constexpr (NP == 1) {
            pv_wait(done - 2, 8);
            pv_wait(done - 1, 8);
            __syncwarp();
            fence_after();
        }
        // the row's 32 elements from i of O as it stands
        auto o_part = [&](int i, uint32_t (&y)[32]) {
            if constexpr (NP == 1) {
                if (done) {  // the same for a warp: all its lanes load
                    tmem_ld32<0>(tmem + lanes + C::o_col(w) + i, y);
                    tmem_landed(y);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) y[e] = 0u;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 32; ++e) y[e] = __float_as_uint(o[i + e]);
            }
        };
        // The finished 32 elements from i of the row, through shared memory where the stream's queries
        // were (same swizzle, so that neither side has bank conflicts), to leave in whole rows.
        uint8_t* stage = sm + (QT == 2 ? w * C::Q_PLANE : 0);
        constexpr int OPR = D * (int)sizeof(T) / 16;  // 16-byte chunks of an output row
        auto stage_at = [&](int row, int ch) { return stage + (ch >> 3) * C::Q_SLAB + row * 128 + (((ch & 7) ^ (row & 7)) << 4); };
        auto put = [&](int i, const uint32_t (&y)[32], float f) {
#pragma unroll
            for (int e = 0; e < 32; e += 16 / (int)sizeof(T)) {
                uint4 u;
                if constexpr (NP == 1)
                    u = make_uint4(pack(asf(y[e]) * f, asf(y[e + 1]) * f), pack(asf(y[e + 2]) * f, asf(y[e + 3]) * f),
                                   pack(asf(y[(e + 4) % 32]) * f, asf(y[(e + 5) % 32]) * f),
                                   pack(asf(y[(e + 6) % 32]) * f, asf(y[(e + 7) % 32]) * f));
                else
                    u = make_uint4(__float_as_uint(asf(y[e]) * f), __float_as_uint(asf(y[e + 1]) * f),
                                   __float_as_uint(asf(y[e + 2]) * f), __float_as_uint(asf(y[e + 3]) * f));
                *reinterpret_cast<uint4*>(stage_at(r, (i + e) * (int)sizeof(T) / 16)) = u;
            }
        };
        auto leave = [&](int thread, int threads) {
            const int pieces = min(p.tok, mine) * heads * OPR;
#pragma unroll 4
            for (int i = thread; i < pieces; i += threads) {
                const int row = i / OPR, ch = i % OPR, t_row = tok_of(row);
                reinterpret_cast<uint4*>(og + row_at(base_tok + t_row, row - t_row * heads))[ch] =
                    *reinterpret_cast<const uint4*>(stage_at(row, ch));
            }
        };
        if constexpr (QT == 2) {
            {
                const float inv = l == 0.f ? 0.f : 1.0f / l;  // a row that sees nothing: zeros
#pragma unroll
                for (int i = 0; i < D; i += 32) {
                    uint32_t y[32];
                    o_part(i, y);
                    put(i, y, inv);
                }
            }
            if (w == 0)
                asm volatile("bar.sync 1, 128;" ::: "memory");
            else
                asm volatile("bar.sync 2, 128;" ::: "memory");
            if (!stopped()) leave(r, 128);
        } else {
            // ---- join the streams through the ring, which nothing uses any more once both streams'
            // last products are complete: each gives the other half of its columns
            constexpr int PITCH = D / 2 + 4;  // floats: rows 16 bytes apart in the banks
            float* join = reinterpret_cast<float*>(sm + C::Q_BYTES);  // [2][128][D / 2]
            float2* join_ml = reinterpret_cast<float2*>(join + 256 * PITCH);  // [2][128]
            auto give = [&](auto which) {
                constexpr int half = decltype(which)::value;
#pragma unroll
                for (int i = 0; i < D / 2; i += 32) {
                    uint32_t y[32];
                    o_part(half * (D / 2) + i, y);
                    float4* to = reinterpret_cast<float4*>(join + (half * 128 + r) * PITCH + i);
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        to[e / 4] = make_float4(asf(y[e]), asf(y[e + 1]), asf(y[e + 2]), asf(y[e + 3]));
                }
            };
            const int64_t part = ((int64_t)unit * p.splits + split) * 128;
            auto finish = [&](auto which, float keep, float take, float f) {
                constexpr int half = decltype(which)::value;
#pragma unroll
                for (int i = half * (D / 2); i < (half + 1) * (D / 2); i += 32) {
                    uint32_t y[32];
                    o_part(i, y);
                    const float4* from =
                        reinterpret_cast<const float4*>(join + (half * 128 + r) * PITCH + i - half * (D / 2));
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        const float4 v = from[e / 4];
                        y[e] = __float_as_uint(asf(y[e]) * keep + v.x * take);
                        y[e + 1] = __float_as_uint(asf(y[e + 1]) * keep + v.y * take);
                        y[e + 2] = __float_as_uint(asf(y[e + 2]) * keep + v.z * take);
                        y[e + 3] = __float_as_uint(asf(y[e + 3]) * keep + v.w * take);
                    }
                    if (p.splits > 1) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            __stcg(p.part + part * (D / 4) + (i + e) / 4 * 128 + r,
                                   make_float4(asf(y[e]), asf(y[e + 1]), asf(y[e + 2]), asf(y[e + 3])));
                    } else {
                        put(i, y, f);
                    }
                }
            };
            asm volatile("bar.sync 1, 256;" ::: "memory");
            join_ml[w * 128 + r] = make_float2(m, l);
            if (w == 0) give(std::integral_constant<int, 1>{}); else give(std::integral_constant<int, 0>{});
            asm volatile("bar.sync 1, 256;" ::: "memory");
            const float2 his = join_ml[(1 - w) * 128 + r];
            const float mt = fmaxf(m, his.x);
            const float keep = m == -INFINITY ? 0.f : ex2(m - mt), take = his.x == -INFINITY ? 0.f : ex2(his.x - mt);
            const float lt = l * keep + his.y * take, inv = lt == 0.f ? 0.f : 1.0f / lt;
            if (p.splits > 1 && w == 0) __stcg(p.ml + part + r, make_float2(mt, lt));
            if (w == 0) finish(std::integral_constant<int, 0>{}, keep, take, inv);
            else finish(std::integral_constant<int, 1>{}, keep, take, inv);
            if (p.splits == 1) {
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (!stopped()) leave(tid, 256);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    if (warp == 10) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    const unsigned end = part_end(stopped(), c->bad != 0);
    if (QT == 1 && p.splits > 1) {
        if (tid == 0) {
            p.ended[unit * p.splits + split] = end;
            if (split == 0) p.rows[unit] = make_int4(row0, tokens, req, pos0);
        }
    } else if (end == kPartNotFinite && warp < 8) {
        for (int i = warp; i < tokens * heads; i += 8) {
            const int64_t at = ((int64_t)(row0 + i / heads) * a.Hq + kvh * G + head0 + i % heads) * D;
            walk_row<D, T>(a, req, kvh, pos0 + i / heads, static_cast<const T*>(a.q) + at, static_cast<T*>(a.o) + at);
        }
    }
}

// The parts of a row tile, in their order: a block per unit and 16 columns, a thread per row
// and 8 columns.
template <int D, typename T>
__global__ void __launch_bounds__(256) window_join_kernel(const __grid_constant__ PrefillArgs p) {
    const WindowArgs& a = p.a;
    pdl_trigger();
    pdl_wait();
    constexpr int PIECES = D / 16;
    const int unit = blockIdx.x / PIECES, c4 = blockIdx.x % PIECES * 4 + threadIdx.x / 128 * 2, r = threadIdx.x % 128;
    const int units = a.Hkv * p.groups;
    const int kvh = unit % units / p.groups, head0 = unit % units % p.groups * p.heads;
    const int G = a.Hq / a.Hkv, heads = min(p.heads, G - head0);
    const int4 rows = __ldcg(p.rows + unit);  // first row, tokens, request, position
    const int tk = r / heads;
    unsigned end = kPartGood;
    for (int x = 0; x < p.splits; ++x) end = worse(end, __ldcg(p.ended + unit * p.splits + x));
    if (end == kPartStopped) return;
    if (end == kPartNotFinite) {  // as without splits; the unit's blocks share the rows
        const int warp = threadIdx.x / 32 + blockIdx.x % PIECES * 8;
        for (int i = warp; i < rows.y * heads; i += 8 * PIECES) {
            const int64_t at = ((int64_t)(rows.x + i / heads) * a.Hq + kvh * G + head0 + i % heads) * D;
            walk_row<D, T>(a, rows.z, kvh, rows.w + i / heads, static_cast<const T*>(a.q) + at,
                           static_cast<T*>(a.o) + at);
        }
        return;
    }
    if (tk >= min(p.tok, rows.y)) return;
    const int64_t first = (int64_t)unit * p.splits;
    float m = -INFINITY, l = 0.f;
    float4 y[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
    constexpr int BATCH = 8;  // parts whose loads are in flight together
    for (int x0 = 0; x0 < p.splits; x0 += BATCH) {
        float2 ml[BATCH];
        float4 v[BATCH][2];
#pragma unroll
        for (int x = 0; x < BATCH; ++x) {
            const int64_t at = first + min(x0 + x, p.splits - 1);
            ml[x] = __ldcg(p.ml + at * 128 + r);
            v[x][0] = __ldcg(p.part + (at * (D / 4) + c4) * 128 + r);
            v[x][1] = __ldcg(p.part + (at * (D / 4) + c4 + 1) * 128 + r);
        }
        float top = m;
#pragma unroll
        for (int x = 0; x < BATCH; ++x) top = fmaxf(top, ml[x].x);
        const float keep = m == -INFINITY ? 0.f : ex2(m - top);
        m = top;
        l *= keep;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            y[e].x *= keep; y[e].y *= keep; y[e].z *= keep; y[e].w *= keep;
        }
#pragma unroll
        for (int x = 0; x < BATCH; ++x) {
            const float f = x0 + x < p.splits && ml[x].x != -INFINITY ? ex2(ml[x].x - m) : 0.f;
            l = fmaf(f, ml[x].y, l);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                y[e].x = fmaf(f, v[x][e].x, y[e].x); y[e].y = fmaf(f, v[x][e].y, y[e].y);
                y[e].z = fmaf(f, v[x][e].z, y[e].z); y[e].w = fmaf(f, v[x][e].w, y[e].w);
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    T* out = static_cast<T*>(a.o) + ((int64_t)(rows.x + tk) * a.Hq + kvh * G + head0 + r - tk * heads) * D + 4 * c4;
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(out) = make_uint4(pack(y[0].x * inv, y[0].y * inv), pack(y[0].z * inv, y[0].w * inv),
                                                    pack(y[1].x * inv, y[1].y * inv), pack(y[1].z * inv, y[1].w * inv));
    } else {
#pragma unroll
        for (int e = 0; e < 2; ++e)
            reinterpret_cast<float4*>(out)[e] = make_float4(y[e].x * inv, y[e].y * inv, y[e].z * inv, y[e].w * inv);
    }
}

// Row tiles of a call, at most, and the blocks that share one.
struct Plan {
    int heads, groups, tok, splits;
    int64_t tiles;  // of one row tile per block, over all prompts and units
};

// Pages that a row tile of `tok` positions sees, at most.
int64_t visible_pages(int tok, int window, int sinks, int max_ctx) {
    return std::min<int64_t>(((int64_t)max_ctx + KT - 1) / KT,
                             ((int64_t)window + tok + KT - 1) / KT + 1 + ((int64_t)sinks + KT - 1) / KT);
}

// A row tile is split when there are fewer row tiles than SMs, into parts of two pages
// (one per stream) or more.
Plan make_plan(int M, int n_prompts, int Hq, int Hkv, int window, int sinks, int max_ctx) {
    Plan p{};
    const int G = Hq / Hkv;
    p.groups = (G + 127) / 128;
    p.heads = (G + p.groups - 1) / p.groups;
    p.tok = 128 / p.heads;
    p.tiles = std::min<int64_t>((int64_t)M / p.tok + n_prompts, M) * Hkv * p.groups;
    const int64_t pages = visible_pages(p.tok, window, sinks, max_ctx);
    p.splits = p.tiles < kSms ? (int)std::max<int64_t>(1, std::min<int64_t>(kSms / std::max<int64_t>(p.tiles, 1), pages / 2)) : 1;
    return p;
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
    const int64_t blocks = std::min<int64_t>(tiles, p.a.rows) * p.a.Hkv * p.groups * p.splits;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    e = launch_pdl(window_prefill_kernel<D, NP, QT, T>, dim3((unsigned)blocks), kThreads, C::BYTES, st, p);
    if (e != cudaSuccess || p.splits == 1) return e;
    return launch_pdl(window_join_kernel<D, T>, dim3((unsigned)(blocks / p.splits) * (D / 16)), 256, 0, st, p);
}

template <int D>
cudaError_t launch_d(const PrefillArgs& p, bool f32, int64_t tiles, cudaStream_t st) {
    if (f32) return launch_t<D, 3, 1, float>(p, st);
    // two row tiles per block once that leaves no SM without a block
    return tiles >= 2 * kSms ? launch_t<D, 1, 2, __nv_bfloat16>(p, st) : launch_t<D, 1, 1, __nv_bfloat16>(p, st);
}

}  // namespace

// Enough for every smaller call too: a call's row tiles are split into kSms parts at most, of two
// pages or more.
uint64_t window_prefill_scratch(int M, int n_prompts, int Hq, int Hkv, int d, int window, int sinks, int max_ctx) {
    if (M == 0) return 16;
    const Plan p = make_plan(M, n_prompts, Hq, Hkv, window, sinks, max_ctx);
    const int64_t most = visible_pages(p.tok, window, sinks, max_ctx) / 2;  // parts of a row tile
    if (most < 2) return 16;
    const uint64_t parts = std::min<int64_t>(kSms, p.tiles * most), tiles = std::min<int64_t>(kSms, p.tiles);
    const uint64_t n = kCounterBytes + tiles * 16 + parts * (128 * (d + 2) * sizeof(float) + sizeof(unsigned));
    return (n + 15) / 16 * 16;
}

cudaError_t launch_window_prefill(const WindowArgs& a, bool f32, cudaStream_t st) {
    const Plan plan = make_plan(a.rows, a.n_prompts, a.Hq, a.Hkv, a.window, a.sinks, a.max_ctx);
    PrefillArgs p{};
    p.a = a;
    p.a.window = std::min(a.window, 1 << 30);  // positions are below max_ctx <= 2^30
    p.a.sinks = std::min(a.sinks, 1 << 30);
    p.heads = plan.heads;
    p.groups = plan.groups;
    p.tok = plan.tok;
    p.splits = plan.splits;
    p.scale = (float)(1.4426950408889634 / sqrt((double)a.d));
    p.part = reinterpret_cast<float4*>(static_cast<char*>(a.scratch) + kCounterBytes);
    p.rows = reinterpret_cast<int4*>(p.part + plan.tiles * plan.splits * 128 * (a.d / 4));
    p.ml = reinterpret_cast<float2*>(p.rows + plan.tiles);
    p.ended = reinterpret_cast<unsigned*>(p.ml + plan.tiles * plan.splits * 128);
    return a.d == 128 ? launch_d<128>(p, f32, plan.tiles, st) : launch_d<64>(p, f32, plan.tiles, st);
}

cudaError_t window_prefill_error(int* code) { return cudaMemcpyFromSymbol(code, g_window_error, sizeof(int)); }

}  // namespace loip
