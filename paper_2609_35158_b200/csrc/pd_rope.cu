// Rotary positions with several axes, alone and fused with the append of the rotated keys to the cache.
//
// Pair i of a head's first rot_dim values, (a, b), becomes (a cos - b sin, a sin + b cos) with the angle
// position[axis(i)] * inv_freq[i]. Far positions: an fp32 product of position and frequency loses the angle's
// fraction of a turn (at position 10^6 a float angle steps by 1/16 rad). Here a frequency is a 64-bit fixed-point
// fraction of a turn and the product with the position wraps modulo 2^64, i.e. modulo whole turns, exactly; its top
// 32 bits are the angle to 2^-32 turns. The frequency itself is off by less than 2^-63 turns (the host converts it in integers),
// so the angle by less than 2^-31 at every int32 position.
//
// Bound by its bytes: every row is read and written once. The sines of a token serve all its heads, so a CTA computes
// them once per token into shared memory, laid out so that the lanes of a row read neighbouring 16 bytes. A lane holds two
// 8-value chunks of a row, the two halves of its pairs or two chunks D / 16 apart, so that every store of a warp covers
// whole 32-byte sectors; two rows per lane are in flight, the first two while the sines are computed. What it measured, 16
// turns of 256-2048 tokens at 32/8 heads (533 MB): 117 us with a row at a time and bank conflicts on the sines, 95 us
// without, 88.6 us (0.93 of the copy bandwidth) with the registers held to 48 so that five CTAs fit an SM; three rows in
// flight instead of two 105 us.
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
template <int D>
constexpr int kRopeTokens = D == 128 ? 4 : 16;  // most tokens a CTA takes at a time
// rotated K rows a CTA may hold in shared memory: beside at most 8.3 KB of sines and page ids, five CTAs still fit an SM
constexpr int kRopeRowBytes = 28672;

// pairs of the half-split form: x holds the first elements, y the second
__device__ __forceinline__ void rotate2(uint32_t &x, uint32_t &y, const float4 &cs) {
    const float a0 = bf16_lo(x), a1 = bf16_hi(x), b0 = bf16_lo(y), b1 = bf16_hi(y);
    x = pack_bf16x2(a0 * cs.x - b0 * cs.y, a1 * cs.z - b1 * cs.w);
    y = pack_bf16x2(a0 * cs.y + b0 * cs.x, a1 * cs.w + b1 * cs.z);
}
// an adjacent pair in one word
__device__ __forceinline__ uint32_t rotate1(uint32_t x, float c, float sn) {
    const float a = bf16_lo(x), b = bf16_hi(x);
    return pack_bf16x2(a * c - b * sn, a * sn + b * c);
}

// The (cos, sin) of a token, two pairs per entry. Half-split: unit u is pairs 8 u .. 8 u + 7, entries k = 0..3 its pairs
// 2 k and 2 k + 1. Adjacent: unit u is chunk u, pairs 4 u .. 4 u + 3, entries k = 0, 1.
template <int D>
struct Turns {
    float4 at[4][D / 8];
};
// where pair i of the configuration lies, as an index of float2
template <int D>
__device__ __forceinline__ int turns_at(int i, bool adjacent) {
    const int unit = adjacent ? i >> 2 : i >> 3, k = adjacent ? (i & 3) >> 1 : (i & 7) >> 1;
    return (k * (D / 8) + unit) * 2 + (i & 1);
}

// One lane's share of a row: its two chunks and what becomes of them.
struct Share {
    int c0, c1;       // 8-value chunks
    bool pair, t0, t1;  // pair: c0 and c1 rotate against each other; t0, t1: chunk c0, c1 rotates in itself
};
template <int D>
__device__ __forceinline__ Share share_of(const RopeParams &p, int j) {
    const int turn_lanes = p.rot_dim / 16;
    Share s;
    if (p.adjacent) {
        s.c0 = j;
        s.c1 = j + D / 16;
        s.pair = false;
        s.t0 = 8 * s.c0 < p.rot_dim;
        s.t1 = 8 * s.c1 < p.rot_dim;
    } else {
        s.pair = j < turn_lanes;
        s.c0 = s.pair ? j : turn_lanes + j;  // turn_lanes pairs of chunks, then the rest in two halves
        s.c1 = s.pair ? j + turn_lanes : s.c0 + D / 16 - turn_lanes;
        s.t0 = s.t1 = false;
    }
    return s;
}

template <int D>
__device__ __forceinline__ void rope_chunks(const Share &s, int j, const Turns<D> &turns, uint4 &x, uint4 &y) {
    if (s.pair) {
        rotate2(x.x, y.x, turns.at[0][j]);
        rotate2(x.y, y.y, turns.at[1][j]);
        rotate2(x.z, y.z, turns.at[2][j]);
        rotate2(x.w, y.w, turns.at[3][j]);
    }
    if (s.t0) {
        const float4 u = turns.at[0][s.c0], v = turns.at[1][s.c0];
        x = make_uint4(rotate1(x.x, u.x, u.y), rotate1(x.y, u.z, u.w), rotate1(x.z, v.x, v.y), rotate1(x.w, v.z, v.w));
    }
    if (s.t1) {
        const float4 u = turns.at[0][s.c1], v = turns.at[1][s.c1];
        y = make_uint4(rotate1(y.x, u.x, u.y), rotate1(y.y, u.z, u.w), rotate1(y.z, v.x, v.y), rotate1(y.w, v.z, v.w));
    }
}

enum { kNoAppend = 0, kAppendBf16 = 1, kAppendQ4 = 2 };

template <int D, int APPEND>
__global__ void __launch_bounds__(kThreads, 5) rope_kernel(const __grid_constant__ RopeParams p) {
    constexpr int LANES = D / 16;
    constexpr int SUBS = kThreads / LANES;
    __shared__ Turns<D> turns[kRopeTokens<D>];
    __shared__ int32_t page_of[kRopeTokens<D>];
    extern __shared__ __align__(16) uint8_t dyn[];  // kAppendQ4: the tile's rotated K rows, [tokens][Hkv][D]
    __nv_bfloat16 *k_rows = reinterpret_cast<__nv_bfloat16 *>(dyn);
    const int b = blockIdx.y, tid = threadIdx.x, j = tid % LANES, sub = tid / LANES;
    const Share mine = share_of<D>(p, j);
    grid_dependency_wait();
    launch_dependents();
    int r0 = 0, n = p.total, L = 0;
    if (APPEND != kNoAppend) {
        r0 = p.q_indptr[b];
        n = p.q_indptr[b + 1] - r0;
        L = p.ctx_lens[b];
        if (n <= 0) return;
        if (p.positions != nullptr && r0 + n > p.position_stride) {  // some of its positions would lie past the array
            if (tid == 0 && blockIdx.x == 0) latch(p.status, kDevBadLength, b, r0 + n);
            return;
        }
    }
    // the append to 4-bit pages takes no more tokens than announced where that is one, and this stands for it
    const bool room = APPEND != kNoAppend && L >= 0 && L <= p.MP * kPageSize - n && !(APPEND == kAppendQ4 && p.single && n > 1);
    if (APPEND != kNoAppend && !room && tid == 0 && blockIdx.x == 0) latch(p.status, kDevBadLength, b, L);
    const int half = p.rot_dim / 2;
    // rows of a token: q, then k, then (bf16 pages) v, which is copied; without room for them k and v are left out
    const int rows = p.Hq + (APPEND == kAppendBf16 ? (room ? 2 * p.Hkv : 0) : p.Hkv);

    for (int i0 = blockIdx.x * p.tile; i0 < n; i0 += gridDim.x * p.tile) {
        const int nt = min(p.tile, n - i0);
        // this lane group's rows of the tile, two at a time: (token, row) of each and its two chunks
        int t = sub / rows, r = sub - t * rows, at_t[2]; bool rot[2]; __nv_bfloat16 *to[2];
        uint4 x[2], y[2];
        auto load2 = [&]() {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                at_t[u] = t;
                if (t < nt) {
                    const size_t row = static_cast<size_t>(r0 + i0 + t);
                    const int kv = r - p.Hq, which = kv >= p.Hkv, kvh = which ? kv - p.Hkv : kv;
                    rot[u] = !which;
                    const __nv_bfloat16 *from;
                    if (kv < 0) {
                        from = p.q + (row * p.Hq + r) * D;
                        to[u] = p.q_out + (row * p.Hq + r) * D;
                    } else {
                        from = (which ? p.v_new : p.k_new) + (row * p.Hkv + kvh) * D;
                        if (APPEND == kNoAppend) to[u] = p.k_out + (row * p.Hkv + kv) * D;
                        else if (APPEND == kAppendQ4) to[u] = k_rows + (t * p.Hkv + kv) * D;
                        else {
                            const int pos = L + i0 + t, page = p.page_table[static_cast<size_t>(b) * p.MP + pos / kPageSize];
                            to[u] = static_cast<uint32_t>(page) >= static_cast<uint32_t>(p.num_pages) ? nullptr : (which ? p.v_pages : p.k_pages) +
                               ((static_cast<size_t>(page) * p.Hkv + kvh) * kPageSize + pos % kPageSize) * D;
                        }
                    }
                    x[u] = reinterpret_cast<const uint4 *>(from)[mine.c0];
                    y[u] = reinterpret_cast<const uint4 *>(from)[mine.c1];
                    for (r += SUBS; r >= rows; r -= rows) ++t;
                }
            }
        };
        load2();  // on their way while the sines are computed

        if (APPEND != kNoAppend && tid < nt && room) {
            const int page = p.page_table[static_cast<size_t>(b) * p.MP + (L + i0 + tid) / kPageSize];
            page_of[tid] = page;
            if (page < 0 || page >= p.num_pages) latch(p.status, kDevBadPage, b, page);
        }
        for (int u0 = 0; u0 < nt; u0 += kThreads / (D / 2)) {
            const int u = u0 + tid / (D / 2), i = tid % (D / 2);
            if (u < nt && i < half) {
                const long long pos = p.positions != nullptr ? p.positions[p.axis_of_pair[i] * p.position_stride + r0 + i0 + u] : L + i0 + u;
                const uint64_t turn = static_cast<uint64_t>(pos) * p.freq[i];
                float sn, c;
                sincospif(static_cast<float>(static_cast<int32_t>(turn >> 32)) * 4.656612873077393e-10f, &sn, &c);  // 2^-31: half turns
                reinterpret_cast<float2 *>(turns[u].at)[turns_at<D>(i, p.adjacent != 0)] = make_float2(c * p.magnitude, sn * p.magnitude);
            }
        }
        __syncthreads();
        while (at_t[0] < nt) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (at_t[u] >= nt) continue;
                if (to[u] == nullptr) continue;
                if (rot[u]) rope_chunks<D>(mine, j, turns[at_t[u]], x[u], y[u]);
                reinterpret_cast<uint4 *>(to[u])[mine.c0] = x[u];
                reinterpret_cast<uint4 *>(to[u])[mine.c1] = y[u];
            }
            load2();
        }
        __syncthreads();  // the tile's sines (and rotated K rows) are done with, or ready to be quantised
        if (APPEND == kAppendQ4) {
            constexpr int QL = D / 16;  // lanes per row of the quantiser
            const int qj = tid % QL, items = room ? nt * 2 * p.Hkv : 0;  // K and V of every (token, KV head)
            for (int x0 = 0; x0 < items; x0 += kThreads / QL) {
                const int item = min(x0 + tid / QL, items - 1), which = item & 1;  // (lanes past the end follow along)
                const int u = (item >> 1) / p.Hkv, kvh = (item >> 1) - u * p.Hkv;
                const uint4 *src = reinterpret_cast<const uint4 *>(which ? p.v_new + (static_cast<size_t>(r0 + i0 + u) * p.Hkv + kvh) * D
                                                                         : k_rows + (item >> 1) * D) + 2 * qj;
                uint32_t rec;
                const uint2 codes = q4_quantize16(src[0], src[1], rec);
                if (x0 + tid / QL < items && static_cast<uint32_t>(page_of[u]) < static_cast<uint32_t>(p.num_pages)) {
                    const int slot = (L + i0 + u) % kPageSize;
                    uint8_t *block = p.kv4 + (static_cast<size_t>(page_of[u]) * p.Hkv + kvh) * q4_block_bytes<D>();
                    *reinterpret_cast<uint2 *>(q4_codes_at<D>(block, which, slot, 2 * qj)) = codes;
                    if ((qj & 3) == 0) *q4_record_at<D>(block, which, slot, 2 * qj) = rec;
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
    // One token per CTA until that fills the device, then as many as give every lane group about six rows (three rounds of
    // two loads; four and eight measured the same within 1 %). For 4-bit pages the tile's rotated K rows have to fit beside the sines.
    const int rows = p.Hq + (append == kAppendBf16 ? 2 : 1) * p.Hkv, subs = kThreads / (p.D / 16);
    const int most_tokens = p.D == 128 ? kRopeTokens<128> : kRopeTokens<64>;
    p.tile = most <= num_sms * 8 ? 1 : 6 * subs / rows;
    if (append == kAppendQ4 && p.tile > kRopeRowBytes / (p.Hkv * p.D * 2)) p.tile = kRopeRowBytes / (p.Hkv * p.D * 2);
    if (append == kAppendQ4 && p.Hkv * p.D * 2 > kRopeRowBytes) return cudaErrorInvalidValue;
    p.tile = p.tile < 1 ? 1 : (p.tile > most_tokens ? most_tokens : p.tile);
    const int tiles = (max_q_len + p.tile - 1) / p.tile, want = (num_sms * 64 + seqs - 1) / seqs;
    const dim3 grid(tiles < want ? tiles : want, seqs);
    p.single = max_q_len == 1;
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
    a.row_limit = p.positions != nullptr ? p.position_stride : 0;
    *launched = 2;
    return launch_advance_lens(a, stream);
}

}  // namespace pd
