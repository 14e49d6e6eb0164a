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

// Quantises 8 values of a row (one lane's share); the 8 lanes of a group of 64 call it together (their lane numbers
// differ in the low three bits). Returns the 8 codes, the first value in the lowest nibble; `rec` = {scale, min}.
//
//   min    the group's smallest value: a bf16 already, stored exactly
//   scale  (max - min) / 15 rounded UP to bf16, so that no code passes 15; NaN where the group holds a non-finite value
//          or its range leaves fp32 (min and codes are then 0 and the whole group reads back as NaN), 0 where it is below 2^-100 (all codes 0)
//   code   (x - min) / scale to the nearest integer, ties to even; x - min is rounded to fp32 first
//
// The quotient: with 1/scale as an unevaluated sum hi + lo, fma(r, hi, r * lo) differs from r / scale by little more
// than half a unit in the last place before its only rounding that counts. A tie r = (k + 1/2) * scale is a float, so
// it comes out exactly; any other r / scale is at least one part in 2^24 away from k + 1/2 (scale has 8 significant
// bits, r at most 24), more than the error, and falls on its own side. Scales above 2^64, where lo could leave the
// normal range, divide instead. Adding 1.5 * 2^23 then rounds to an integer and leaves the code in the low bits.
__device__ __forceinline__ uint32_t q4_quantize8(const uint4 &x, uint32_t &rec) {
    uint32_t mn = bf16x2_min_nan(bf16x2_min_nan(x.x, x.y), bf16x2_min_nan(x.z, x.w));
    uint32_t mx = bf16x2_max_nan(bf16x2_max_nan(x.x, x.y), bf16x2_max_nan(x.z, x.w));
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
        mn = bf16x2_min_nan(mn, __shfl_xor_sync(0xffffffffu, mn, o));
        mx = bf16x2_max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    }
    mn = bf16x2_min_nan(mn, mn >> 16 | mn << 16);
    mx = bf16x2_max_nan(mx, mx >> 16 | mx << 16);
    const float lo = __fadd_rn(bf16_lo(mn), 0.f), hi = __fadd_rn(bf16_lo(mx), 0.f);  // subnormals and -0 become 0
    const float range = __fsub_rn(hi, lo);
    float s = __fdiv_rn(range, 15.f);
    const bool bad = !(range < INFINITY);  // NaN compares false too
    if (bad) {
        s = __uint_as_float(0x7fc00000u);
    } else {
        s = s < 7.888609052210118e-31f ? 0.f : __uint_as_float((__float_as_uint(s) + 0xffffu) & 0xffff0000u);
    }
    rec = (__float_as_uint(s) >> 16) | (bad ? 0u : __float_as_uint(lo) & 0xffff0000u);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t code[8];
    if (s > 0.f && s <= 18446744073709551616.f) {
        const float inv = __frcp_rn(s);
        const float inv_lo = __fmul_rn(__fmaf_rn(-s, inv, 1.f), inv);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float r = __fsub_rn((i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]), lo);
            code[i] = __float_as_uint(__fadd_rn(__fmaf_rn(r, inv, __fmul_rn(r, inv_lo)), 12582912.f));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float r = __fsub_rn((i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]), lo);
            const float q = s > 0.f ? __fdiv_rn(r, s) : 0.f;
            code[i] = __float_as_uint(__fadd_rn(q, 12582912.f));
        }
    }
    uint32_t out = code[0] & 15u;
#pragma unroll
    for (int i = 1; i < 8; ++i) out |= (code[i] & 15u) << (4 * i);
    return out;
}

// The inverse for one lane's 8 codes: fma in fp32 (scale * code is exact), one rounding to bf16.
__device__ __forceinline__ uint4 q4_dequantize8(uint32_t codes, uint32_t rec) {
    const float s = bf16_lo(rec), m = bf16_hi(rec);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // 2^23 + code as a float, without a conversion instruction
        const float a = __uint_as_float(0x4b000000u | ((codes >> (8 * i)) & 15u)) - 8388608.f;
        const float b = __uint_as_float(0x4b000000u | ((codes >> (8 * i + 4)) & 15u)) - 8388608.f;
        const __nv_bfloat162 v = __floats2bfloat162_rn(__fmaf_rn(s, a, m), __fmaf_rn(s, b, m));
        w[i] = *reinterpret_cast<const uint32_t *>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Where lane j of a row (values 8 j .. 8 j + 7; which = 0 for K, 1 for V) finds its codes and its group's record.
template <int D>
__device__ __forceinline__ uint32_t *q4_codes_at(uint8_t *block, int which, int slot, int j) {
    return reinterpret_cast<uint32_t *>(block + which * 8 * D + slot * (D / 2) + q4_piece_pos<D>(j >> 2, slot) * 16 + (j & 3) * 4);
}
template <int D>
__device__ __forceinline__ uint32_t *q4_record_at(uint8_t *block, int which, int slot, int j) {
    return reinterpret_cast<uint32_t *>(block + 16 * D + slot * (D / 8) + (j >> 3) * 8 + which * 4);
}

}  // namespace

}  // namespace pd
