// New tokens' rows into a cache of shared latent vectors: c' = c / rms(c) * weight, the key part and the queries rotated.
//
// One pass over packed tokens. A CTA takes `tile` tokens of a sequence: the sines of each once into shared memory (angles as
// in pd_rope.cu: 64-bit fixed-point turns, exact at every int32 position), then a warp per latent (16 values per lane in two
// 16-byte pieces, the mean square by shuffles in fp32) and four lanes per rotated row of 64 values (the key's and one per
// query head; a lane holds pieces j and j + 4, the two halves of its pairs). Bound by its bytes: 22K tokens of 16 turns with 32
// query heads of 128 bytes inside rows of 384 take 49.3 us, 4.7 TB/s, 45 without the rotation. Nothing but the wanted bytes is read;
// memory serves them more slowly: a copy of such rows alone, without barriers, runs at 4.9 to 5.2 TB/s, of dense ones at 5.5 to 6.0.
// Four lanes a row and two rows in flight each: with eight lanes a row the same work took 62 us or more.
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
constexpr int kMaxTile = kThreads / 32;  // tokens a CTA takes at a time: a warp per latent
constexpr int kFlight = 2;               // rotated rows of a lane group in flight
constexpr int kPairs = kLatentRope / 2;

// (cos, sin) of a token, two pairs per entry, so that the lanes of a row read neighbouring entries. Halves: entry 4 k + u holds pairs
// 8 u + 2 k and 8 u + 2 k + 1 (lane u's); adjacent: entry 8 k + u pairs 4 u + 2 k and 4 u + 2 k + 1 (piece u's).
__device__ __forceinline__ int turns_at(int i, bool adjacent) {  // where pair i lies, as an index of float2
    return adjacent ? (8 * ((i & 3) >> 1) + (i >> 2)) * 2 + (i & 1) : (4 * ((i & 7) >> 1) + (i >> 3)) * 2 + (i & 1);
}
// eight values of a row that rotate against eight others (halves), lane u
__device__ __forceinline__ void rotate_halves(uint4 &x, uint4 &y, const float4 *cs) {
    uint32_t *a = &x.x, *b = &y.x;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float a0 = bf16_lo(a[k]), a1 = bf16_hi(a[k]), b0 = bf16_lo(b[k]), b1 = bf16_hi(b[k]);
        const float4 t = cs[4 * k];
        a[k] = pack_bf16x2(a0 * t.x - b0 * t.y, a1 * t.z - b1 * t.w);
        b[k] = pack_bf16x2(a0 * t.y + b0 * t.x, a1 * t.w + b1 * t.z);
    }
}
// eight values that are four adjacent pairs, piece u
__device__ __forceinline__ void rotate_adjacent(uint4 &x, const float4 *cs) {
    uint32_t *a = &x.x;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float u = bf16_lo(a[k]), v = bf16_hi(a[k]);
        const float4 t = cs[8 * (k >> 1)];
        const float c = (k & 1) ? t.z : t.x, s = (k & 1) ? t.w : t.y;
        a[k] = pack_bf16x2(u * c - v * s, u * s + v * c);
    }
}

__global__ void __launch_bounds__(kThreads, 4) rope_append_latent_kernel(const __grid_constant__ LatentAppendParams p) {
    __shared__ float4 turns[kMaxTile][kPairs / 2];
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 31;
    grid_dependency_wait();
    launch_dependents();
    const int r0 = p.q_indptr[b], n = p.q_indptr[b + 1] - r0, L = p.ctx_lens[b];
    if (n <= 0) return;
    if (p.positions != nullptr && r0 + n > p.position_stride) {  // some of its positions would lie past the array
        if (tid == 0 && blockIdx.x == 0) latch(p.status, kDevBadLength, b, r0 + n);
        return;
    }
    const bool room = L >= 0 && L <= p.MP * kPageSize - n;
    if (!room && tid == 0 && blockIdx.x == 0) latch(p.status, kDevBadLength, b, L);
    const int half = p.rot_dim / 2;
    // where a token's row goes, or null
    auto row_of = [&](int i) -> __nv_bfloat16 * {
        if (!room) return nullptr;
        const int pos = L + i, page = p.page_table[static_cast<size_t>(b) * p.MP + pos / kPageSize];
        if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(p.num_pages)) {
            latch(p.status, kDevBadPage, b, page);
            return nullptr;
        }
        return p.kv_pages + (static_cast<size_t>(page) * kPageSize + pos % kPageSize) * kLatentRow;
    };
    const int rows = 1 + (p.q != nullptr ? p.Hq : 0), j = tid & 3;
    // halves: pieces of 8 values c0 and c1 = c0 + rot_dim / 16 rotate against each other, then the rest is copied
    const int pieces = p.rot_dim / 16;
    const int c0 = p.adjacent ? j : (j < pieces ? j : pieces + j), c1 = p.adjacent ? j + 4 : (j < pieces ? j + pieces : j + 4);
    for (int i0 = blockIdx.x * p.tile; i0 < n; i0 += gridDim.x * p.tile) {
        const int nt = min(p.tile, n - i0);
        // ---- this lane group's first rotated rows (the key's is row 0 of a token) and this warp's latent are on their way while the
        // sines are computed
        int x = tid >> 2, at_u[kFlight];
        uint4 a[kFlight], c[kFlight];
        __nv_bfloat16 *to[kFlight];
        auto fetch = [&]() {
#pragma unroll
            for (int f = 0; f < kFlight; ++f, x += kThreads / 4) {
                to[f] = nullptr;
                if (x >= nt * rows) continue;
                const int u = x / rows, r = x - u * rows;
                const long long row = r0 + i0 + u;
                const __nv_bfloat16 *from;
                at_u[f] = u;
                if (r == 0) {
                    from = p.kv_new + row * p.kv_stride + kLatentDim;
                    to[f] = row_of(i0 + u);
                    if (to[f] == nullptr) continue;
                    to[f] += kLatentDim;
                } else {
                    from = p.q + row * p.q_token_stride + (r - 1) * p.q_head_stride;
                    to[f] = p.q_out + row * p.q_out_token_stride + (r - 1) * p.q_out_head_stride;
                }
                a[f] = reinterpret_cast<const uint4 *>(from)[c0];
                c[f] = reinterpret_cast<const uint4 *>(from)[c1];
            }
        };
        fetch();
        const int lt = tid >> 5;  // the token whose latent this warp takes
        uint4 v[2];
        __nv_bfloat16 *latent_to = nullptr;
        if (lt < nt) {
            const uint4 *src = reinterpret_cast<const uint4 *>(p.kv_new + (r0 + i0 + lt) * p.kv_stride);
            v[0] = src[lane], v[1] = src[lane + 32];
            latent_to = row_of(i0 + lt);
        }
        for (int y = tid; y < nt * kPairs; y += kThreads) {
            const int u = y / kPairs, i = y % kPairs;
            float sn = 0.f, cs = 1.f, mag = 1.f;
            if (i < half) {
                const long long pos = p.positions != nullptr ? p.positions[p.axis_of_pair[i] * p.position_stride + r0 + i0 + u] : L + i0 + u;
                const uint64_t turn = static_cast<uint64_t>(pos) * p.freq[i];
                sincospif(static_cast<float>(static_cast<int32_t>(turn >> 32)) * 4.656612873077393e-10f, &sn, &cs);  // 2^-31: half turns
                mag = p.magnitude;
            }
            reinterpret_cast<float2 *>(turns[u])[turns_at(i, p.adjacent != 0)] = make_float2(cs * mag, sn * mag);
        }
        // ---- latents: a warp per token
        if (lt < nt && p.norm_weight != nullptr) {
            float f[16], ss = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t w = (&v[k >> 2].x)[k & 3];
                f[2 * k] = bf16_lo(w), f[2 * k + 1] = bf16_hi(w);
                ss = fmaf(f[2 * k], f[2 * k], ss);
                ss = fmaf(f[2 * k + 1], f[2 * k + 1], ss);
            }
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            const float inv = rsqrtf(ss * (1.f / kLatentDim) + p.norm_eps);
            const uint4 *wt = reinterpret_cast<const uint4 *>(p.norm_weight);
            const uint4 g[2] = {wt[lane], wt[lane + 32]};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t w = (&g[k >> 2].x)[k & 3];
                (&v[k >> 2].x)[k & 3] = pack_bf16x2(f[2 * k] * inv * bf16_lo(w), f[2 * k + 1] * inv * bf16_hi(w));
            }
        }
        if (latent_to != nullptr) {
            reinterpret_cast<uint4 *>(latent_to)[lane] = v[0];
            reinterpret_cast<uint4 *>(latent_to)[lane + 32] = v[1];
        }
        __syncthreads();  // the sines
        // ---- rotated rows, four lanes each
        for (;;) {
#pragma unroll
            for (int f = 0; f < kFlight; ++f) {
                if (to[f] == nullptr) continue;
                const float4 *cs = turns[at_u[f]];
                if (p.adjacent) {
                    if (8 * c0 < p.rot_dim) rotate_adjacent(a[f], cs + c0);
                    if (8 * c1 < p.rot_dim) rotate_adjacent(c[f], cs + c1);
                } else if (j < pieces) {
                    rotate_halves(a[f], c[f], cs + j);
                }
                reinterpret_cast<uint4 *>(to[f])[c0] = a[f];
                reinterpret_cast<uint4 *>(to[f])[c1] = c[f];
            }
            if (x >= nt * rows) break;
            fetch();
        }
        __syncthreads();
    }
    if (p.advance && gridDim.x == 1 && room && tid == 0) p.ctx_lens[b] = L + n;
}

}  // namespace

cudaError_t launch_rope_append_latent(const LatentAppendParams &base, int max_q_len, int num_sms, int *launched, cudaStream_t stream) {
    LatentAppendParams p = base;
    const long long most = static_cast<long long>(max_q_len) * p.B;
    if (most <= 0) return cudaSuccess;
    // one token per CTA until that fills the device
    p.tile = most <= num_sms * 8 ? 1 : kMaxTile;
    const int tiles = (max_q_len - 1) / p.tile + 1, want = (num_sms * 64 + p.B - 1) / p.B;
    const dim3 grid(tiles < want ? tiles : want, p.B);
    const cudaError_t err = launch_pdl(rope_append_latent_kernel, grid, dim3(kThreads), 0, stream, p.pdl != 0, p);
    if (err != cudaSuccess) return err;
    *launched = 1;
    if (!p.advance || grid.x == 1) return err;
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
