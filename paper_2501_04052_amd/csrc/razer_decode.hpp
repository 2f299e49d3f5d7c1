// Decode of scale-byte weights through byte tables, into operands of v_mfma_f32_16x16x32_bf16: shared by the kernels for few
// activation rows.
#pragma once
#include "razer_device.hpp"

namespace razer {

// ---- decode through byte tables ----------------------------------------------------------------------------
// A block's eight scaled magnitudes and its special value are 8 bf16 numbers: their high bytes fill one pair of
// registers and their low bytes another, and v_perm_b32 looks up four codes per instruction.  Table position of
// FP4 magnitude m: m ^ 4, position 4 (the magnitude 0) holds the negated special value; the selector of the true
// zero (code 0) gets bit 3 set as well: 12, which v_perm_b32 answers with 0x00.  The codes' sign bits flip the high
// bytes' signs afterwards (code 8 carries one, hence the negation).  The pairs come out in the order (0,2) (4,6)
// (1,3) (5,7) of the dword's codes: sk_permute_pairs() puts the activations in the same order.
// Per dword 8 byte permutes (4.2 clk each, measured) and 10 plain logic operations (2.3-2.5 clk): 58 clk against 89
// for convert, two multiplications, convert and patch per pair.
__device__ __forceinline__ uint4 sk_byte_table(uint32_t sb, float sv0, float sv1)
{
    float s, sv;
    decode_scale_byte<0>(sb, sv0, sv1, s, sv);
    // bf16 bits of s x {2, 3, 4, 6} and {special, .5, 1, 1.5}; a zero scale makes all of them 0
    const uint32_t b1 = f2u(s) >> 16, b15 = f2u(1.5f * s) >> 16, live = s != 0.0f ? 0xFFFFu : 0u;
    const uint32_t sp = (uint32_t)f32_to_bf16_rne(-(sv * s));            // (exact but for 9.5 times a significand of 15 / 8: 19 x 15, 9 bits)
    const uint32_t v0 = (b1 + 0x80u) & live, v1 = (b15 + 0x80u) & live, v2 = (b1 + 0x100u) & live, v3 = (b15 + 0x100u) & live;
    const uint32_t v4 = sp, v5 = (b1 - 0x80u) & live, v6 = b1, v7 = b15;
    return make_uint4((v0 >> 8) | ((v1 >> 8) << 8) | ((v2 >> 8) << 16) | ((v3 >> 8) << 24),
                      (v4 >> 8) | ((v5 >> 8) << 8) | ((v6 >> 8) << 16) | ((v7 >> 8) << 24),
                      (v0 & 255u) | ((v1 & 255u) << 8) | ((v2 & 255u) << 16) | (v3 << 24),
                      (v4 & 255u) | ((v5 & 255u) << 8) | ((v6 & 255u) << 16) | (v7 << 24));
}
__device__ __forceinline__ v8bf sk_decode_dword_table(uint32_t x, v4u t)
{
    const uint32_t z = x ^ 0x44444444u, nz = (x | 0x88888888u) - 0x11111111u;          // bit 3 of nz: magnitude not 0
    const uint32_t sel = __builtin_amdgcn_bitop3_b32(nz, z, 0x77777777u, 0x89);         // low bits of z, bit 3 of ~(nz | z)
    const uint32_t se = sel & 0x0F0F0F0Fu, so = (sel >> 4) & 0x0F0F0F0Fu;
    const uint32_t he = __builtin_amdgcn_bitop3_b32(__builtin_amdgcn_perm(t.y, t.x, se), x << 4, 0x80808080u, 0x78);
    const uint32_t ho = __builtin_amdgcn_bitop3_b32(__builtin_amdgcn_perm(t.y, t.x, so), x, 0x80808080u, 0x78);
    const uint32_t le = __builtin_amdgcn_perm(t.w, t.z, se), lo = __builtin_amdgcn_perm(t.w, t.z, so);
    return __builtin_bit_cast(v8bf, make_uint4(__builtin_amdgcn_perm(he, le, 0x05010400u), __builtin_amdgcn_perm(he, le, 0x07030602u),
                                               __builtin_amdgcn_perm(ho, lo, 0x05010400u), __builtin_amdgcn_perm(ho, lo, 0x07030602u)));
}
// 8 bf16 activations in the pair order of sk_decode_dword_table
__device__ __forceinline__ v4u sk_permute_pairs(v4u a)
{
    return v4u{__builtin_amdgcn_perm(a.y, a.x, 0x05040100u), __builtin_amdgcn_perm(a.w, a.z, 0x05040100u),
               __builtin_amdgcn_perm(a.y, a.x, 0x07060302u), __builtin_amdgcn_perm(a.w, a.z, 0x07060302u)};
}

}  // namespace razer
