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
// The same twice, as a pair; and of two bytes.
__device__ __forceinline__ uint32_t kv4_scale_twice(uint32_t c) { return c * 0x100010u + KV4_EXP0 * 0x10001u; }
__device__ __forceinline__ uint32_t kv4_scale_pair(uint32_t lo, uint32_t hi) { return lo * 16u + (hi * 0x100000u + KV4_EXP0 * 0x10001u); }

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
// The term that takes the codes' offset away again: -136 s.  17 (8 + m) has at most eight bits, so this is exact, and so is
// (128 + code) s - 136 s: the decoded value has at most seven.
__device__ __forceinline__ uint32_t kv4_offset(uint32_t s2) { return hmul2_bf16(s2, 0xC308C308u); }
// Values of the codes at nibble j of either half of w, as a bf16 pair: 128 + code is a bf16 whose last four bits are the code.
template <int J>
__device__ __forceinline__ uint32_t kv4_pair(uint32_t w, uint32_t s2, uint32_t off2) {
    uint32_t x;  // (w >> 4 J) & 0x000F000F | 0x43004300: written as one operation, because the compiler makes two of it
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(x) : "r"(w >> (4 * J)), "r"(0x000F000Fu), "r"(0x43004300u));
    return hfma2_bf16(x, s2, off2);
}
// The eight elements of a word, in their order, as four pairs.
__device__ __forceinline__ void kv4_word(uint32_t w, uint32_t s2, uint32_t off2, uint32_t (&r)[4]) {
    r[0] = kv4_pair<0>(w, s2, off2);
    r[1] = kv4_pair<1>(w, s2, off2);
    r[2] = kv4_pair<2>(w, s2, off2);
    r[3] = kv4_pair<3>(w, s2, off2);
}
#endif

}  // namespace specroll
