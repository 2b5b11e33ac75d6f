// q8.h -- the 8-bit cache: block-floating rows in granules of 16 tokens.
//
// A row (a token's key or value of one kv head, d elements) is d / 32 blocks of 32 elements.
// A block has an exponent byte E and 32 code bytes, a sign and a 7-bit magnitude m:
//   value = +-m 2^(E - 133)
// E is the smallest, and 8 at least, for which no magnitude exceeds 127; at most 253.  254 and 255
// stand for NaN in the whole block; the append writes 255 (codes 0) for a block that holds
// something that is not finite, or 127.5 2^120 or more.  A value has 7 significant bits and is
// 2^-125 or more in size: a normal bf16 number.
//
// A granule is 16 tokens of a kv head, in one piece of 33 d bytes: codes of the keys [16][d],
// codes of the values [16][d], exponents of the keys [16][d / 32], of the values [16][d / 32].
// A layer's part of a page is [kv head][4 granules].  The 16-byte piece c of token t's codes
// lies at c ^ (t d / 128 % (d / 16)) of its row: tokens 0, 2, 4, .. (and 1, 3, 5, ..) then have
// the same piece in different banks of shared memory, and so have the pieces 2c of two
// neighbours.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace loip {
namespace q8 {

constexpr int kGranule = 16;  // tokens in one contiguous piece
constexpr int kMostExponent = 253;

constexpr uint64_t granule_bytes(int d) { return 33 * (uint64_t)d; }
// A layer's part of a page of 64 tokens.
constexpr uint64_t layer_bytes(int Hkv, int d) { return (uint64_t)Hkv * 4 * granule_bytes(d); }

#ifdef __CUDACC__
template <int D>
struct Granule {
    static constexpr int BYTES = 33 * D;
    static constexpr int PIECES = D / 16;   // 16-byte pieces of a row
    static constexpr int BLOCKS = D / 32;   // exponents of a row
    // Byte offsets in a granule: of piece c of token t's codes, and of its first exponent.
    __device__ static constexpr int piece(int is_v, int t, int c) {
        return is_v * 16 * D + t * D + (c ^ (t * D / 128 % PIECES)) * 16;
    }
    __device__ static constexpr int exponents(int is_v, int t) { return 32 * D + is_v * (D / 2) + t * BLOCKS; }
};

// The granule of a position in a layer's part of its page, for one kv head.
template <int D>
__device__ __forceinline__ int64_t granule_at(int kvh, int pos) {
    return (int64_t)(kvh * 4 + pos % 64 / kGranule) * Granule<D>::BYTES;
}

// Exponent of a block whose largest magnitude has these bits: a magnitude rounds to 128 from 127.5
// on, that is from 255/256 of the next power of two, and E is one more then.
__device__ __forceinline__ uint32_t exponent_of(uint32_t most) {
    const uint32_t e = (most + 0x10000u) >> 23;  // not finite: 255 or 256
    return e > kMostExponent ? 255u : max(e, 8u);
}
// 2^(133 - E), exactly
__device__ __forceinline__ float inverse_step(uint32_t E) { return __uint_as_float((260u - E) << 23); }
// 2^(E - 133); NaN for the exponents that stand for it
__device__ __forceinline__ float step_of(uint32_t E) {
    return __uint_as_float(E > kMostExponent ? 0x7fc00000u : (max(E, 7u) - 6u) << 23);
}
// rint(x / step), below 128 in size, as sign and magnitude: the sum with 1.5 2^23 is rounded once,
// to the nearest whole number (ties to even).
__device__ __forceinline__ uint32_t code_of(float x, float inv) {
    const int m = __float_as_int(fmaf(x, inv, 12582912.f)) - 0x4b400000;
    return m < 0 ? 128u - (uint32_t)m : (uint32_t)m;
}
// Four codes, the first in the low byte.
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d, float inv) {
    return code_of(a, inv) | code_of(b, inv) << 8 | code_of(c, inv) << 16 | code_of(d, inv) << 24;
}
__device__ __forceinline__ float value_of(uint32_t code, float step) {
    const float m = (float)(code & 127u);
    return (code & 128u ? -m : m) * step;
}

// Codes to pairs of bf16, exactly.  Sign and magnitude of a code, put where a bf16 number has its sign
// and its mantissa, are the subnormal number +-m 2^-133, and times 2^E that is the value.  (The byte
// permute and the mask are the integer pipe's, which takes an instruction every second cycle, and
// bound the conversion.)  2^E is a bf16 number up to E = 127 only, so
//   pair_of     takes two products by powers of two, 2^127 and 2^(E - 127): four instructions
//   shifted_of  makes the value times 2^-kShift in one, for the exponents of shift_holds: three
//
// The second factor for a pair of blocks with exponents E[0] + 2^16 E[1] (or for one, twice).
__device__ __forceinline__ uint32_t scale2(uint32_t e) {
    const uint32_t nan = (e + 0x00020002u & 0x01000100u) >> 2;  // 0x40 where it is 254 or 255
    return e * 128u | nan * 511u;                               // 0x40 x 511 = 0x7fc0
}
// (code byte, the same again) twice -> the pair of values
__device__ __forceinline__ uint32_t pair_of(uint32_t twice, uint32_t scale) {
    uint32_t r;
    asm("{\n .reg .b32 x;\n and.b32 x, %1, 0x807f807f;\n mul.rn.bf16x2 x, x, %3;\n mul.rn.bf16x2 %0, x, %2;\n}\n"
        : "=r"(r)
        : "r"(twice), "r"(scale), "r"(0x7f007f00u));
    return r;
}

// Values times 2^-64 are normal bf16 numbers for exponents 71 to 191 (elements of 2^-62 to 2^58 in
// size), and the factor 2^(E - 64) is one too.  (shifted2 as scale2.)
constexpr int kShift = 64;
__device__ __forceinline__ bool shift_holds(uint32_t E) { return E - 71u <= 191u - 71u; }
__device__ __forceinline__ uint32_t shifted2(uint32_t e) { return e * 128u + (127 - kShift) * 0x00800080u; }
__device__ __forceinline__ uint32_t shifted_of(uint32_t twice, uint32_t scale) {
    uint32_t r;
    asm("{\n .reg .b32 x;\n and.b32 x, %1, 0x807f807f;\n mul.rn.bf16x2 %0, x, %2;\n}\n"
        : "=r"(r)
        : "r"(twice), "r"(scale));
    return r;
}
#endif

}  // namespace q8
}  // namespace loip
