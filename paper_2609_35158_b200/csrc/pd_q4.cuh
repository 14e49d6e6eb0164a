// The 4-bit KV page format: layout, the quantiser of one row and its inverse, shared by the kernels that write,
// read back and attend over 4-bit pages.
//
// A (page, KV head) block is 18 * D bytes in one piece, so that one bulk copy fetches all a worker needs:
//   [0, 8D)     K codes, 16 rows of D/2 bytes      [8D, 16D)  V codes
//   [16D, 18D)  records: per token and group of 64 values {k_scale, k_min, v_scale, v_min}, bf16
// value = scale * code + min, code in [0, 15]. Value 2j of a row is the low nibble of its byte j, 2j + 1 the high
// one; the row's 16-byte piece c lies at piece position c ^ swizzle(slot), which spreads the eight rows that an
// ldmatrix phase reads at equal c over all 32 banks although untiled bulk copies cannot swizzle.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include <type_traits>

#include "pd_kernels.cuh"

namespace pd {

namespace {

constexpr int kQ4Group = 64;

template <int D>
__host__ __device__ constexpr int q4_block_bytes() { return 18 * D; }

template <int D>
__device__ __forceinline__ int q4_piece_pos(int piece, int slot) {
    return D == 128 ? (piece ^ ((slot >> 1) & 3)) : (piece ^ ((slot >> 2) & 1));
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ uint32_t bf16x2_min_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t bf16x2_max_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Quantises 16 values of a row (one lane's share); the 4 lanes of a group of 64 call it together (their lane numbers
// differ in the low two bits). Returns the 16 codes, the first value in the lowest nibble; `rec` = {scale, min}.
//
//   min    the group's smallest value: a bf16 already, stored exactly
//   scale  (max - min) / 15 rounded UP to bf16, or down where 15 * scale + min would round past bf16's largest value (a code
//          then stands for at most 15.12 steps, which is 15 after rounding); NaN where the group holds a non-finite value
//          or its range leaves fp32 (min and codes are then 0 and the whole group reads back as NaN), 0 where it is below 2^-100 (all codes 0)
//   code   (x - min) / scale to the nearest integer, ties to even; x - min is rounded to fp32 first
//
// Quotients without dividing: with 1/scale as an unevaluated sum hi + lo (to some 2^-44), fma(r, hi, r * lo) differs from
// r / scale by little more than half a unit in the last place before the only rounding that counts. A tie
// r = (k + 1/2) * scale is a float, so it comes out exactly; any other r / scale is at least one part in 2^24 away from
// k + 1/2 (scale has 8 significant bits, r at most 24), more than the error, and falls on its own side. The same holds
// for range / 15: no float's quotient by 15 is within 1/30 of a unit of a rounding boundary, so the result is the
// correctly rounded one. Scales above 2^64, where lo could leave the normal range, divide instead. Adding 1.5 * 2^23
// rounds to an integer and leaves the code in the low bits; the constant parts are taken off after eight are joined.
//
// Bound by instructions before bytes: with the compiler's divisions and 8 values per lane the append took 217 warp
// instructions per 256 values, with the two-part reciprocal 128; 16 values per lane and two per fp32 instruction, 105.
__device__ __forceinline__ uint64_t f32x2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ uint2 q4_quantize16(const uint4 &x0, const uint4 &x1, uint32_t &rec) {
    const uint32_t w[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
    uint32_t mn = w[0], mx = w[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        mn = bf16x2_min_nan(mn, w[i]);
        mx = bf16x2_max_nan(mx, w[i]);
    }
    mx ^= 0x80008000u;  // as {min, -max} both are minima, and one shuffle carries them
    uint32_t m = bf16x2_min_nan(__byte_perm(mn, mx, 0x5410), __byte_perm(mn, mx, 0x7632));
    m = bf16x2_min_nan(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = bf16x2_min_nan(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const float lo = __fadd_rn(bf16_lo(m), 0.f), hi = __fsub_rn(0.f, bf16_hi(m));  // subnormals and -0 become 0
    const float range = __fsub_rn(hi, lo);
    constexpr float k15hi = 0.06666667014360427856f, k15lo = -3.4769376121e-09f;  // 1/15 = hi + lo
    float s = __fmaf_rn(range, k15hi, __fmul_rn(range, k15lo));
    const bool bad = !(range < INFINITY);  // NaN compares false too
    if (bad) s = __uint_as_float(0x7fc00000u);
    else s = s < 7.888609052210118e-31f ? 0.f : __uint_as_float((__float_as_uint(s) + 0xffffu) & 0xffff0000u);
    rec = (__float_as_uint(s) >> 16) | (bad ? 0u : __float_as_uint(lo) & 0xffff0000u);
    uint32_t out[2];
    if (s <= 18446744073709551616.f) {
        float inv;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
        inv = s > 0.f ? inv : 0.f;  // scale 0: codes 0
        const float inv_lo = __fmul_rn(__fmaf_rn(-s, inv, 1.f), inv);
        const uint64_t base2 = f32x2(-lo, -lo), inv2 = f32x2(inv, inv), lo2 = f32x2(inv_lo, inv_lo), round2 = f32x2(12582912.f, 12582912.f);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint64_t r = f32x2(bf16_lo(w[4 * h + i]), bf16_hi(w[4 * h + i])), e, t;
                asm("add.rn.ftz.f32x2 %0, %0, %1;" : "+l"(r) : "l"(base2));
                asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(e) : "l"(r), "l"(lo2));
                asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(t) : "l"(r), "l"(inv2), "l"(e));
                asm("add.rn.ftz.f32x2 %0, %0, %1;" : "+l"(t) : "l"(round2));
                sum += (static_cast<uint32_t>(t) << (8 * i)) + (static_cast<uint32_t>(t >> 32) << (8 * i + 4));
            }
            out[h] = sum - 0x4b400000u * 0x11111111u;  // 0x4b400000 is 1.5 * 2^23
        }
    } else {
        if (__fmaf_rn(s, 15.f, lo) >= __uint_as_float(0x7f7f8000u)) {  // halfway between bf16's largest value and 2^128
            s = __uint_as_float(__float_as_uint(s) - 0x10000u);       // (a range / 15 that is a bf16 does not get here)
            rec -= 1u;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            out[h] = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t v = w[4 * h + (i >> 1)];
                const float r = __fsub_rn((i & 1) ? bf16_hi(v) : bf16_lo(v), lo);
                out[h] |= bad ? 0u : (__float_as_uint(__fadd_rn(__fdiv_rn(r, s), 12582912.f)) & 15u) << (4 * i);
            }
        }
    }
    return make_uint2(out[0], out[1]);
}

// The inverse for one lane's 8 codes: scale * code + min in one bf16 fma. (scale * code has 12 bits at most, so where the
// sum is near a rounding boundary of bf16 it is a float: rounding to fp32 on the way would change nothing.)
__device__ __forceinline__ uint4 q4_dequantize8(uint32_t codes, uint32_t rec) {
    const uint32_t s = __byte_perm(rec, 0u, 0x1010), m = __byte_perm(rec, 0u, 0x3232);
    uint32_t v[4];  // values i and i + 4
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t c = ((codes >> (4 * i)) & 0x000f000fu) | 0x43004300u;  // 128 + code
        asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(c) : "r"(0xc300c300u));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[i]) : "r"(s), "r"(c), "r"(m));
    }
    return make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[0], v[1], 0x7632),
                      __byte_perm(v[2], v[3], 0x7632));
}

// Where lane j of a row (values 8 j .. 8 j + 7; which = 0 for K, 1 for V) finds its codes and its group's record (K's,
// V's follows it).
template <int D, typename Block>
__device__ __forceinline__ auto q4_codes_at(Block *block, int which, int slot, int j) {
    using Word = std::conditional_t<std::is_const<Block>::value, const uint32_t, uint32_t>;
    return reinterpret_cast<Word *>(block + which * 8 * D + slot * (D / 2) + q4_piece_pos<D>(j >> 2, slot) * 16 + (j & 3) * 4);
}
template <int D, typename Block>
__device__ __forceinline__ auto q4_record_at(Block *block, int which, int slot, int j) {
    using Word = std::conditional_t<std::is_const<Block>::value, const uint32_t, uint32_t>;
    return reinterpret_cast<Word *>(block + 16 * D + slot * (D / 8) + (j >> 3) * 8 + which * 4);
}

}  // namespace

}  // namespace pd
