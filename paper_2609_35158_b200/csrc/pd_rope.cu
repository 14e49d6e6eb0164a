// Rotary positions with several axes, alone and fused with the append of the rotated keys to the cache.
//
// Pair i of a head's first rot_dim values, (a, b), becomes (a cos - b sin, a sin + b cos) with the angle
// position[axis(i)] * inv_freq[i]. Far positions: an fp32 product of position and frequency loses the angle's
// fraction of a turn (at position 10^6 a float angle steps by 1/16 rad). Here a frequency is a 64-bit fixed-point
// fraction of a turn and the product with the position wraps modulo 2^64, i.e. modulo whole turns, exactly; its top
// 32 bits are the angle to 2^-32 turns. The frequency itself is rounded once, to 2^-53 of its value.
//
// Bound by its bytes: every row is read and written once. The sines of a token serve all its heads, so a CTA computes
// them once per token into shared memory; then eight values of each half-row of a pair sit in one lane (16-byte loads
// and stores, D / 16 lanes per row), whichever way the pairs lie.
#include "pd_kernels.cuh"
#include "pd_ptx.cuh"
#include "pd_q4.cuh"

namespace pd {

namespace {

__device__ __forceinline__ void latch(int32_t *status, int code, int seq, int detail) {
    if (atomicCAS(status, kDevOk, code) == kDevOk) {
        status[1] = seq;
        status[2] = detail;
    }
}

constexpr int kThreads = 256;
constexpr int kRopeTokens = 4;  // tokens a CTA takes at a time
constexpr int kRopeRowBytes = 40960;  // rotated K rows a CTA may hold in shared memory

__device__ __forceinline__ uint32_t rotate2(uint32_t x, uint32_t y, const float2 c0, const float2 c1, uint32_t &y_out) {
    const float a0 = bf16_lo(x), a1 = bf16_hi(x), b0 = bf16_lo(y), b1 = bf16_hi(y);
    y_out = pack_bf16x2(a0 * c0.y + b0 * c0.x, a1 * c1.y + b1 * c1.x);
    return pack_bf16x2(a0 * c0.x - b0 * c0.y, a1 * c1.x - b1 * c1.y);
}
// an adjacent pair in one word
__device__ __forceinline__ uint32_t rotate1(uint32_t x, const float2 c) {
    const float a = bf16_lo(x), b = bf16_hi(x);
    return pack_bf16x2(a * c.x - b * c.y, a * c.y + b * c.x);
}

// Lane j of a row of D / 16 lanes: rotates pairs 8 j .. 8 j + 7 of `src` or, past the rotated part, copies two chunks.
template <int D>
__device__ __forceinline__ void rope_row(const RopeParams &p, const __nv_bfloat16 *src, __nv_bfloat16 *dst, int j, const float2 *cs) {
    const int turn_lanes = p.rot_dim / 16;
    int c0, c1;  // the two 8-value chunks this lane holds
    if (j >= turn_lanes || p.adjacent) {
        c0 = 2 * j;
        c1 = c0 + 1;
    } else {
        c0 = j;
        c1 = j + turn_lanes;
    }
    uint4 x = *reinterpret_cast<const uint4 *>(src + 8 * c0), y = *reinterpret_cast<const uint4 *>(src + 8 * c1);
    if (j < turn_lanes) {
        const float4 *t = reinterpret_cast<const float4 *>(cs + 8 * j);  // (cos, sin) of two pairs each
        const float4 t0 = t[0], t1 = t[1], t2 = t[2], t3 = t[3];
        if (p.adjacent) {
            x.x = rotate1(x.x, make_float2(t0.x, t0.y)); x.y = rotate1(x.y, make_float2(t0.z, t0.w));
            x.z = rotate1(x.z, make_float2(t1.x, t1.y)); x.w = rotate1(x.w, make_float2(t1.z, t1.w));
            y.x = rotate1(y.x, make_float2(t2.x, t2.y)); y.y = rotate1(y.y, make_float2(t2.z, t2.w));
            y.z = rotate1(y.z, make_float2(t3.x, t3.y)); y.w = rotate1(y.w, make_float2(t3.z, t3.w));
        } else {
            x.x = rotate2(x.x, y.x, make_float2(t0.x, t0.y), make_float2(t0.z, t0.w), y.x);
            x.y = rotate2(x.y, y.y, make_float2(t1.x, t1.y), make_float2(t1.z, t1.w), y.y);
            x.z = rotate2(x.z, y.z, make_float2(t2.x, t2.y), make_float2(t2.z, t2.w), y.z);
            x.w = rotate2(x.w, y.w, make_float2(t3.x, t3.y), make_float2(t3.z, t3.w), y.w);
        }
    }
    *reinterpret_cast<uint4 *>(dst + 8 * c0) = x;
    *reinterpret_cast<uint4 *>(dst + 8 * c1) = y;
}

enum { kNoAppend = 0, kAppendBf16 = 1, kAppendQ4 = 2 };

template <int D, int APPEND>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ RopeParams p) {
    constexpr int LANES = D / 16;
    constexpr int PAIRS = D / 2;
    __shared__ __align__(16) float2 cs[kRopeTokens][PAIRS];
    extern __shared__ __align__(16) uint8_t dyn[];  // kAppendQ4: the tile's rotated K rows, [tokens][Hkv][D]
    __nv_bfloat16 *k_rows = reinterpret_cast<__nv_bfloat16 *>(dyn);
    const int b = blockIdx.y, tid = threadIdx.x, j = tid % LANES, sub = tid / LANES;
    grid_dependency_wait();
    launch_dependents();
    int r0 = 0, n = p.total, L = 0;
    if (APPEND != kNoAppend) {
        r0 = p.q_indptr[b];
        n = p.q_indptr[b + 1] - r0;
        L = p.ctx_lens[b];
        if (n <= 0) return;
    }
    const bool room = APPEND != kNoAppend && L >= 0 && L <= p.MP * kPageSize - n;
    if (APPEND != kNoAppend && !room && tid == 0 && blockIdx.x == 0) latch(p.status, kDevBadLength, b, L);
    const int half = p.rot_dim / 2;
    const int rows = p.Hq + (APPEND == kNoAppend ? p.Hkv : (APPEND == kAppendBf16 ? 2 * p.Hkv : p.Hkv));  // q, k and the copied v of a token

    for (int i0 = blockIdx.x * p.tile; i0 < n; i0 += gridDim.x * p.tile) {
        const int nt = min(p.tile, n - i0);
        for (int x = tid; x < nt * half; x += kThreads) {
            const int t = x / half, i = x - t * half;
            const long long pos = p.positions != nullptr ? p.positions[p.axis_of_pair[i] * p.position_stride + r0 + i0 + t] : L + i0 + t;
            const uint64_t turns = static_cast<uint64_t>(pos) * p.freq[i];
            float sn, c;
            sincospif(static_cast<float>(static_cast<int32_t>(turns >> 32)) * 4.656612873077393e-10f, &sn, &c);  // 2^-31: half turns
            cs[t][i] = make_float2(c * p.magnitude, sn * p.magnitude);
        }
        __syncthreads();
        for (int x = sub; x < nt * rows; x += kThreads / LANES) {
            const int t = x / rows, r = x - t * rows;
            const size_t row = static_cast<size_t>(r0 + i0 + t);
            if (r < p.Hq) {
                rope_row<D>(p, p.q + (row * p.Hq + r) * D, p.q_out + (row * p.Hq + r) * D, j, cs[t]);
            } else if (APPEND == kNoAppend) {
                const size_t at = (row * p.Hkv + (r - p.Hq)) * D;
                rope_row<D>(p, p.k_new + at, p.k_out + at, j, cs[t]);
            } else if (APPEND == kAppendQ4) {
                rope_row<D>(p, p.k_new + (row * p.Hkv + (r - p.Hq)) * D, k_rows + (t * p.Hkv + (r - p.Hq)) * D, j, cs[t]);
            } else if (room) {
                const int pos = L + i0 + t, page = p.page_table[static_cast<size_t>(b) * p.MP + pos / kPageSize];
                if (page < 0 || page >= p.num_pages) {
                    if (j == 0) latch(p.status, kDevBadPage, b, page);
                    continue;
                }
                const int which = (r - p.Hq) / p.Hkv, kvh = r - p.Hq - which * p.Hkv;
                const size_t src = (row * p.Hkv + kvh) * D;
                const size_t dst = ((static_cast<size_t>(page) * p.Hkv + kvh) * kPageSize + pos % kPageSize) * D;
                if (which == 0) {
                    rope_row<D>(p, p.k_new + src, p.k_pages + dst, j, cs[t]);
                } else {
                    const uint4 *s = reinterpret_cast<const uint4 *>(p.v_new + src);
                    uint4 *d = reinterpret_cast<uint4 *>(p.v_pages + dst);
                    const uint4 v0 = s[2 * j], v1 = s[2 * j + 1];
                    d[2 * j] = v0;
                    d[2 * j + 1] = v1;
                }
            }
        }
        __syncthreads();  // the tile's sines (and rotated K rows) are done with, or ready to be quantised
        if (APPEND == kAppendQ4) {
            constexpr int QL = D / 8;  // lanes per row of the quantiser
            const int qj = tid % QL, items = room ? nt * 2 * p.Hkv : 0;
            for (int x0 = 0; x0 < items; x0 += kThreads / QL) {
                const int x = min(x0 + tid / QL, items - 1);
                const int t = x / (2 * p.Hkv), hw = x - t * 2 * p.Hkv, kvh = hw >> 1, which = hw & 1;
                const int pos = L + i0 + t, page = p.page_table[static_cast<size_t>(b) * p.MP + pos / kPageSize];
                const bool ok = page >= 0 && page < p.num_pages;
                const __nv_bfloat16 *src = which ? p.v_new + (static_cast<size_t>(r0 + i0 + t) * p.Hkv + kvh) * D : k_rows + (t * p.Hkv + kvh) * D;
                uint32_t rec;
                const uint32_t codes = q4_quantize8(*reinterpret_cast<const uint4 *>(src + qj * 8), rec);
                if (!ok) {
                    if (qj == 0) latch(p.status, kDevBadPage, b, page);
                } else if (x0 + tid / QL < items) {
                    uint8_t *block = p.kv4 + (static_cast<size_t>(page) * p.Hkv + kvh) * q4_block_bytes<D>();
                    *q4_codes_at<D>(block, which, pos % kPageSize, qj) = codes;
                    if ((qj & 7) == 0) *q4_record_at<D>(block, which, pos % kPageSize, qj) = rec;
                }
            }
            __syncthreads();
        }
    }
    if (APPEND != kNoAppend && p.advance && gridDim.x == 1 && room) {
        __syncthreads();
        if (tid == 0) p.ctx_lens[b] = L + n;
    }
}

}  // namespace

cudaError_t launch_rope(const RopeParams &base, int append, int max_q_len, int num_sms, int *launched, cudaStream_t stream) {
    RopeParams p = base;
    const int seqs = append == kNoAppend ? 1 : p.B;
    const long long most = static_cast<long long>(max_q_len) * seqs;
    if (most <= 0) return cudaSuccess;
    // one token per CTA until that fills the device, then four (their sines are then computed by all 256 threads)
    p.tile = most <= num_sms * 8 || (append == kAppendQ4 && kRopeTokens * p.Hkv * p.D * 2 > kRopeRowBytes) ? 1 : kRopeTokens;
    if (append == kAppendQ4 && p.Hkv * p.D * 2 > kRopeRowBytes) return cudaErrorInvalidValue;
    const int tiles = (max_q_len + p.tile - 1) / p.tile, want = (num_sms * 8 + seqs - 1) / seqs;
    const dim3 grid(tiles < want ? tiles : want, seqs);
    const size_t dyn = append == kAppendQ4 ? static_cast<size_t>(p.tile) * p.Hkv * p.D * 2 : 0;
    auto go = [&](auto *k) { return launch_pdl(k, grid, dim3(kThreads), dyn, stream, p.pdl != 0, p); };
    cudaError_t err;
    if (p.D == 128) err = append == kNoAppend ? go(rope_kernel<128, kNoAppend>) : append == kAppendBf16 ? go(rope_kernel<128, kAppendBf16>) : go(rope_kernel<128, kAppendQ4>);
    else err = append == kNoAppend ? go(rope_kernel<64, kNoAppend>) : append == kAppendBf16 ? go(rope_kernel<64, kAppendBf16>) : go(rope_kernel<64, kAppendQ4>);
    if (err != cudaSuccess) return err;
    *launched = 1;
    if (append == kNoAppend || !p.advance || grid.x == 1) return err;
    AppendTokensParams a{};
    a.q_indptr = p.q_indptr;
    a.ctx_lens = p.ctx_lens;
    a.B = p.B;
    a.MP = p.MP;
    a.pdl = p.pdl;
    *launched = 2;
    return launch_advance_lens(a, stream);
}

}  // namespace pd
