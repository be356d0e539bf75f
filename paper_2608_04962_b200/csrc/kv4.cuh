// The 4-bit cache's format (include/specroll.h says what it stands for) and its decoding.
#pragma once

#include "common.cuh"

namespace specroll {

template <int D>
struct Kv4 {
    static constexpr int ROW = D / 2, SROW = D / 32;  // bytes of codes and of scales of a token's K or V
    static constexpr int CODES = SPECROLL_PAGE_TOKENS * ROW, TILE = CODES + SPECROLL_PAGE_TOKENS * SROW;
    static_assert(TILE % 16 == 0 && CODES % 16 == 0, "bulk copies move multiples of 16 bytes");
};

constexpr uint32_t KV4_EXP0 = 107u << 7;  // bf16 exponent field of the smallest scale, 2^-20

#ifdef __CUDACC__
// bf16 bits of the scale that a byte stands for: four bits of exponent field and three of mantissa are where bf16 has them, but
// for the shift and the offset.
__device__ __forceinline__ uint32_t kv4_scale_bits(uint32_t c) { return (c << 4) + KV4_EXP0; }

__device__ __forceinline__ uint32_t hfma2_bf16(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t hmul2_bf16(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Decoding to 2^-KV4_DOWN of the values.  Bits 0 .. 7 of a bf16 number are linear from zero on (the subnormal numbers and the first normal
// ones), so that a code in its place is a number already, code 2^-133 from bits 0 .. 3 and code 2^-129 from bits 4 .. 7: one mask and one
// multiplication and addition a pair, and one shift for the upper byte's two.  The factor is s 2^(133 - KV4_DOWN), or an 16th of it, the
// addend -8 s 2^-KV4_DOWN; everything is exact, the result has at most seven bits.  Whoever multiplies with the decoded values
// gives the factor 2^KV4_DOWN back.  (With 128 + code as a number, which needs every code in bits 0 .. 3, three shifts of eight
// codes instead of one took a quarter of the few rows' kernel's time.)
constexpr int KV4_DOWN = 20;
constexpr float KV4_UP = 1048576.0f;            // 2^KV4_DOWN
constexpr uint32_t KV4_UP_PAIR = ((127u + KV4_DOWN) << 7) * 0x10001u;  // the same as a bf16 pair
struct Kv4Scale {
    uint32_t even, odd, off;  // factors for codes in bits 0 .. 3 and 4 .. 7, addend; pairs
};
__device__ __forceinline__ Kv4Scale kv4_scales(uint32_t twice) {  // twice: both scale bytes, 4 bits up
    constexpr uint32_t TWO = 0x10001u;
    return {twice + (KV4_EXP0 + ((133u - KV4_DOWN) << 7)) * TWO, twice + (KV4_EXP0 + ((129u - KV4_DOWN) << 7)) * TWO,
            twice + (KV4_EXP0 + ((3u - KV4_DOWN) << 7) + 0x8000u) * TWO};
}
__device__ __forceinline__ Kv4Scale kv4_scale_of(uint32_t c) { return kv4_scales(c * 0x100010u); }
__device__ __forceinline__ Kv4Scale kv4_scale_of(uint32_t lo, uint32_t hi) { return kv4_scales(lo * 16u + hi * 0x100000u); }
// The eight elements of a word, in their order, as four pairs.
__device__ __forceinline__ void kv4_word(uint32_t w, const Kv4Scale &s, uint32_t (&r)[4]) {
    r[0] = hfma2_bf16(w & 0x000F000Fu, s.even, s.off);
    r[1] = hfma2_bf16(w & 0x00F000F0u, s.odd, s.off);
    r[2] = hfma2_bf16((w >> 8) & 0x000F000Fu, s.even, s.off);
    r[3] = hfma2_bf16((w >> 8) & 0x00F000F0u, s.odd, s.off);
}
#endif

}  // namespace specroll
