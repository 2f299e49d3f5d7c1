// The block encoder of RaZeR on a run of 16 elements in registers (arxiv 2501.04052, Eq. 2, 4 and 5): what razer_quantize's
// kernel and the kernels that encode what they have just computed share.  How it reaches the literal computation's bits is
// described at encode_kernel in razer_quantize.hip.
#pragma once
#include "razer_device.hpp"

namespace razer {

// ---------------------------------------------------------------- scale rounding (Eq. 2)
// Nearest value of the scale grid, ties to the even code, saturating at the top.
template <int FMT>
__device__ __forceinline__ uint32_t round_scale(float t)
{
    if (FMT == 2) {
        // the hardware's round-to-nearest-even cast to half; anything that would land on 2.0 or
        // above saturates at the largest 14-bit code
        const uint32_t h = __builtin_bit_cast(uint16_t, (_Float16)t);
        return (t >= 2.0f || h > 0x3FFFu) ? 0x3FFFu : h;
    }
    constexpr float kMinNormal = (FMT == 0) ? 0.25f : 0.015625f;          // 2^-2 / 2^-6
    constexpr float kSubScale = (FMT == 0) ? 32.0f : 512.0f;              // 1 / subnormal step
    constexpr uint32_t kBiasAdj = (FMT == 0) ? (124u << 3) : (120u << 3);
    constexpr uint32_t kMaxCode = (FMT == 0) ? 63u : 126u;
    uint32_t code;
    if (t < kMinNormal) {
        code = (uint32_t)__builtin_rintf(t * kSubScale);                  // exact product, RNE
    } else {
        uint32_t b = f2u(t);
        b += 0x7FFFFu + ((b >> 20) & 1u);                                 // RNE to 3 mantissa bits
        code = (b >> 20) - kBiasAdj;
    }
    return code > kMaxCode ? kMaxCode : code;
}

// Nearest FP4 value, ties to the even code, saturating at +-6: the hardware conversion (verified against the threshold
// form of the same rule on every boundary +- 1 ulp and 10^6 random values).  It writes the two codes into byte `i` of
// the packed dword; a negative value that rounds to zero comes out as code 0x8 and is cleared later.
__device__ __forceinline__ uint32_t encode_pair(uint32_t word, float a, float b, int i)
{
    return (i == 0)   ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, a, b, 1.0f, 0)
           : (i == 1) ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, a, b, 1.0f, 1)
           : (i == 2) ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, a, b, 1.0f, 2)
                      : __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, a, b, 1.0f, 3);
}
__device__ __forceinline__ v2f decode_pair_f32(uint32_t word, int i)      // the values of those two codes
{
    return (i == 0)   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 0)
           : (i == 1) ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 1)
           : (i == 2) ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 2)
                      : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 3);
}

// Eq. 4 and the codes literally: fp32 division, squared errors in fp64, one chain over the block's elements in index
// order (lane j of the block continues where lane j - 1 ended).  lo / hi: the 16 codes as the hardware rounds them;
// take: bit k set if element k takes the chosen special value.  NP candidates go side by side; with more than one such
// pass the empty asm keeps the compiler from holding what does not depend on the candidate (the base errors, in fp64)
// over all of them: where this path is the rare one, its registers count against the occupancy of the other.
template <int FMT, int G, int NP>
__device__ __forceinline__ void encode_literal(const float (&xv)[kBlock], float den, float sv0, float sv1, uint32_t& lo,
                                               uint32_t& hi, uint32_t& meta, uint32_t& take)
{
    constexpr int NC = (FMT == 1) ? 2 : 4;
    float xs[kBlock];                                                     // X^Scaled
    lo = hi = 0;
#pragma unroll
    for (int k = 0; k < kBlock; k += 2) {
        xs[k] = xv[k] / den;
        xs[k + 1] = xv[k + 1] / den;
        uint32_t& word = (k < 8) ? lo : hi;
        word = encode_pair(word, xs[k], xs[k + 1], (k % 8) / 2);
    }
    const int sub = (int)(threadIdx.x & 63u) & (G - 1), base = (int)(threadIdx.x & 63u) & ~(G - 1);
    double best = 0.0;
    meta = 0;
    take = 0;
#pragma unroll 1
    for (int pass = 0; pass < NC / NP; ++pass) {
        // metadata index of candidate c of this pass: +sv0, (+sv1,) -sv0, (-sv1); two of four at once: one magnitude's signs
        auto index = [&](int c) { return NP == 2 && NC == 4 ? pass + 2 * c : NP == 1 ? pass : c; };
        double sse[NP], e2[G > 1 ? NP : 1][kBlock];
        uint32_t bits[NP];
#pragma unroll
        for (int c = 0; c < NP; ++c) { sse[c] = 0.0; bits[c] = 0u; }
#pragma unroll
        for (int k = 0; k < kBlock; k += 2) {
            float x0 = xs[k], x1 = xs[k + 1];
            uint32_t word = (k < 8) ? lo : hi;
            if constexpr (NP < NC) {
                asm volatile("" : "+v"(x0), "+v"(x1), "+v"(word));
#pragma unroll
                for (int c = 0; c < NP; ++c) asm volatile("" : "+v"(sse[c]), "+v"(bits[c]));
            }
            const v2f q = decode_pair_f32(word, (k % 8) / 2);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const double xd = (double)(j ? x1 : x0), eb = xd - (double)(j ? q.y : q.x);
#pragma unroll
                for (int c = 0; c < NP; ++c) {
                    const int m = index(c);
                    const float mag = (FMT != 1 && (m & 1)) ? sv1 : sv0;
                    const double ev = xd - (double)(m >= NC / 2 ? -mag : mag);
                    const bool sp = fabs(ev) < fabs(eb);
                    const double e = sp ? ev : eb;
                    if (G > 1) e2[c][k + j] = e * e;                      // exact in fp64
                    else sse[c] = __builtin_fma(e, e, sse[c]);            // the same as sse + e*e
                    bits[c] |= (uint32_t)sp << (k + j);
                }
            }
        }
        if constexpr (G > 1) {
            // round p is the one in which lane base + p of the block holds the right starting value (its predecessor's
            // total of round p - 1)
#pragma unroll 1
            for (int p = 0; p < G; ++p) {
#pragma unroll
                for (int c = 0; c < NP; ++c) {
                    double a = (p == 0) ? 0.0 : __shfl(sse[c], base + p - 1);
#pragma unroll
                    for (int k = 0; k < kBlock; ++k) a += e2[c][k];
                    sse[c] = (sub == p) ? a : sse[c];
                }
            }
        }
#pragma unroll
        for (int c = 0; c < NP; ++c) {                                    // Eq. 4: smallest error, ties to the smallest index
            const uint32_t m = (uint32_t)index(c);
            const double s = G > 1 ? __shfl(sse[c], base + G - 1) : sse[c];   // (every lane of the block: the block's sum)
            if (m == 0 || s < best || (s == best && m < meta)) {
                best = s;
                meta = m;
                take = bits[c];
            }
        }
    }
}

// x / den, correctly rounded, from y = 1 / den (correctly rounded)
__device__ __forceinline__ float quotient(float x, float den, float y)
{
    float q = x * y;
    q = __builtin_fmaf(__builtin_fmaf(-q, den, x), y, q);
    return __builtin_fmaf(__builtin_fmaf(-q, den, x), y, q);
}

// Eq. 4 between the two candidates a and b alone, the sums as above: the block is scaled and rounded, and which elements
// take a candidate is seen in fp32 -- xs - q is exact, and so is xs - v where v is the nearer of the two.
template <int FMT, int G, bool SCALED>
__device__ __forceinline__ uint32_t nearest_two(const float (&xv)[kBlock], float den, uint32_t lo, uint32_t hi, float sv0, float sv1,
                                                uint32_t a, uint32_t b)
{
    constexpr uint32_t NM = (FMT == 1) ? 1 : 2;
    const uint32_t m0 = a < b ? a : b, m1 = a < b ? b : a;
    auto value = [&](uint32_t m) { const float v = (NM == 2 && (m & 1u)) ? sv1 : sv0; return m >= NM ? -v : v; };
    const float v0 = value(m0), v1 = value(m1), y = SCALED ? 1.0f : 1.0f / den;
    double e0[G > 1 ? kBlock : 1], e1[G > 1 ? kBlock : 1];                // squared errors
    double s0 = 0.0, s1 = 0.0;
#pragma unroll
    for (int k = 0; k < kBlock; k += 2) {
        float x0 = xv[k], x1 = xv[k + 1];
        uint32_t word = (k < 8) ? lo : hi;
        asm volatile("" : "+v"(x0), "+v"(x1), "+v"(word), "+v"(s0), "+v"(s1));   // (one pair after the other: registers)
        const v2f q = decode_pair_f32(word, (k % 8) / 2);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float xk = j ? x1 : x0, x = SCALED ? xk : quotient(xk, den, y), eb = x - (j ? q.y : q.x), f0 = x - v0, f1 = x - v1;
            const double t0 = (double)(fabsf(f0) < fabsf(eb) ? f0 : eb), t1 = (double)(fabsf(f1) < fabsf(eb) ? f1 : eb);
            if constexpr (G > 1) {
                e0[k + j] = t0 * t0;                                      // exact
                e1[k + j] = t1 * t1;
                asm volatile("" : "+v"(e0[k + j]), "+v"(e1[k + j]));
            } else {
                s0 = __builtin_fma(t0, t0, s0);
                s1 = __builtin_fma(t1, t1, s1);
            }
        }
    }
    if constexpr (G > 1) {
        const int sub = (int)(threadIdx.x & 63u) & (G - 1), base = (int)(threadIdx.x & 63u) & ~(G - 1);
#pragma unroll 1
        for (int p = 0; p < G; ++p) {
            double c0 = (p == 0) ? 0.0 : __shfl(s0, base + p - 1), c1 = (p == 0) ? 0.0 : __shfl(s1, base + p - 1);
#pragma unroll
            for (int k = 0; k < kBlock; ++k) {
                c0 += e0[k];
                c1 += e1[k];
            }
            s0 = (sub == p) ? c0 : s0;
            s1 = (sub == p) ? c1 : s1;
        }
        s0 = __shfl(s0, base + G - 1);
        s1 = __shfl(s1, base + G - 1);
    }
    return s1 < s0 ? m1 : m0;
}

// One run of 16 elements of a block of 16 G (lane j of the block's G consecutive lanes holds its j-th run), whole: Eq. 2, 4
// and 5.  lo, hi: its 16 codes; meta, sc: the metadata and the code of the block's scale, the same in all lanes of the
// block.  checked: the elements are known to be finite (Eq. 1's maximum has seen them).  KEEP: xv holds the scaled elements
// afterwards (what nearest_two then reads instead of scaling again).
template <int FMT, int G, bool KEEP>
__device__ __forceinline__ void encode_run(float (&xv)[kBlock], float delta32, float sv0, float sv1, bool checked, uint32_t& lo,
                                           uint32_t& hi, uint32_t& meta, uint32_t& sc)
{
    constexpr int NM = (FMT == 1) ? 1 : 2;                                // special magnitudes
    float bmax = 0.0f;
#pragma unroll
    for (int k = 0; k < kBlock; ++k) bmax = fmaxf(bmax, fabsf(xv[k]));
    bool finite = true;                                                   // (fmaxf drops a NaN)
    if (!checked) {                                                       // else Eq. 1's maximum has seen every element
        float z = 0.0f;
#pragma unroll
        for (int k = 0; k < kBlock; ++k) z = __builtin_fmaf(xv[k], 0.0f, z);
        finite = z == 0.0f;
    }
#pragma unroll
    for (int off = 1; off < G; off <<= 1) {                               // the block's maximum
        bmax = fmaxf(bmax, __shfl_xor(bmax, off));
        finite = __shfl_xor((int)finite, off) != 0 && finite;
    }

    // Eq. 2
    const float d = delta32 * 6.0f;
    const float t = bmax / d;
    sc = round_scale<FMT>(t);
    const float s = (FMT == 0) ? e3m3_value(sc) : (FMT == 1) ? e4m3_value(sc) : half14_value(sc);

    lo = hi = meta = 0;
    if (s != 0.0f) {
        float den = delta32 * s;
        uint32_t tlo = 0, thi = 0;                                        // bit 3 of a nibble: the element takes the special value
        uint32_t runner = 0;
        bool two = false, decided = finite && den >= 0x1p-70f && delta32 <= 0x1p60f && bmax <= 512.0f * den;
        uint32_t took[NM][2];
#pragma unroll
        for (int m = 0; m < NM; ++m) took[m][0] = took[m][1] = 0u;
        if (decided) {
            const float y = 1.0f / den;
            float all[NM], dir[NM];                                       // gains / 4096: sum, and sum with the element's sign
#pragma unroll
            for (int m = 0; m < NM; ++m) all[m] = dir[m] = 0.0f;
#pragma unroll
            for (int k = 0; k < kBlock; k += 2) {
                const float xs[2] = {quotient(xv[k], den, y), quotient(xv[k + 1], den, y)};
                uint32_t& word = (k < 8) ? lo : hi;
                word = encode_pair(word, xs[0], xs[1], (k % 8) / 2);
                if constexpr (KEEP) { xv[k] = xs[0]; xv[k + 1] = xs[1]; }  // (kept: the next pass needs them often)
                const v2f q2 = decode_pair_f32(word, (k % 8) / 2);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float q = j ? q2.y : q2.x;
                    const float u = fabsf(__builtin_fmaf(2.0f, xs[j], -q));
#pragma unroll
                    for (int m = 0; m < NM; ++m) {
                        const float v = m ? sv1 : sv0;
                        // gain / 4096 (below 1 up to 512 scales), 0 where the special value is no better
                        const float g = __builtin_amdgcn_fmed3f(__builtin_fmaf(fabsf(q), -0x1p-12f, v * 0x1p-12f) * (u - v), 0.0f, 1.0f);
                        all[m] += g;
                        dir[m] += u2f(__builtin_amdgcn_bitop3_b32(f2u(g), f2u(xs[j]), 0x80000000u, 0xF8));
                        // sign bit of 0 - g: set where g > 0; eight elements shift it into the nibbles' top bits
                        uint32_t& b = took[m][k >= 8];
                        b = __builtin_amdgcn_bitop3_b32(b >> 4, f2u(0.0f - g), 0x80000000u, 0xF8);
                    }
                }
            }
            float gain[2 * NM], total = 0.0f;
#pragma unroll
            for (int m = 0; m < NM; ++m) {
#pragma unroll
                for (int off = 1; off < G; off <<= 1) { all[m] += __shfl_xor(all[m], off); dir[m] += __shfl_xor(dir[m], off); }
                gain[m] = 0.5f * (all[m] + dir[m]);                       // metadata order: +sv0, (+sv1,) -sv0, (-sv1)
                gain[NM + m] = 0.5f * (all[m] - dir[m]);
                total += all[m];
            }
            float first = gain[0], second = -1.0f;
#pragma unroll
            for (int c = 1; c < 2 * NM; ++c) {
                const bool up = gain[c] > first;
                second = fmaxf(second, up ? first : gain[c]);
                meta = up ? (uint32_t)c : meta;
                first = up ? gain[c] : first;
            }
            // (the second term covers the rounding of the fp64 sums themselves: each at most 16 G xm^2)
            const float xm = bmax * y, margin = total * ((16.0f * G + 8.0f) * 0x1p-23f) + 1e-15f * xm * xm;
            decided = total == 0.0f || first - second > margin;
            if (!decided) {
                int near = 0;
#pragma unroll
                for (int c = 0; c < 2 * NM; ++c) {
                    const bool close = meta != (uint32_t)c && !(first - gain[c] > margin);
                    near += close;
                    runner = close ? (uint32_t)c : runner;
                }
                two = decided = near == 1;
            }
            if (KEEP) den = 1.0f;
        }
        if (!decided) {
            uint32_t bits;
            encode_literal<FMT, G, (G == 1 ? 2 : 1)>(xv, den, sv0, sv1, lo, hi, meta, bits);
            // bit k of a byte-wide mask to bit 4 k + 3
            auto spread = [](uint32_t b) {
                b = (b | (b << 12)) & 0x000F000Fu;
                b = (b | (b << 6)) & 0x03030303u;
                return ((b | (b << 3)) & 0x11111111u) << 3;
            };
            tlo = spread(bits & 0xFFu);
            thi = spread((bits >> 8) & 0xFFu);
        }
        if (two) meta = nearest_two<FMT, G, KEEP>(xv, den, lo, hi, sv0, sv1, meta, runner);   // (here the elements are needed no more)
        if (decided) {
            const bool one = NM == 2 && (meta & 1u) != 0;
            const uint32_t mlo = one ? took[NM - 1][0] : took[0][0], mhi = one ? took[NM - 1][1] : took[0][1];
            const uint32_t flip = meta >= (uint32_t)NM ? 0u : 0xFFFFFFFFu;  // + candidates: elements with a clear sign bit
            tlo = mlo & (lo ^ flip);
            thi = mhi & (hi ^ flip);
        }
        // Eq. 5 on the packed nibbles: zero keeps code 0x0 whatever its sign, taken elements get the remapped code 0x8
        auto finish = [](uint32_t w, uint32_t taken) {
            const uint32_t nz = (w & 0x77777777u) + 0x77777777u;              // bit 3: magnitude not zero
            w &= nz | 0x77777777u;                                            // -0 -> +0
            return (w & ~(taken - (taken >> 3))) | taken;
        };
        lo = finish(lo, tlo);
        hi = finish(hi, thi);
    }
}

}  // namespace razer
