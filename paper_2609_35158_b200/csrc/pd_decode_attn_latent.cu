// Decode attention over a cache of shared latent vectors (the absorbed form), on the fifth-generation tensor cores.
//
// A token's cached row is 576 values, a latent c (512) and a rotated key part r (64), and every head reads the same row:
// s_t = scale q . (c_t, r_t), out = sum_t softmax(s)_t c_t. A token costs 1152 bytes and 2 * 1088 operations per head, so
// up to about 100 heads the bound is memory. The form of decode_attn_split_kernel (warp MMAs, one ring per warp) would have to
// read every row once per 8 heads; here a CTA takes up to 64 heads over one row in shared memory.
//
// One CTA per SM walks its range of pages in tiles of 64 tokens (4 pages). TOKENS are the M dimension of the logits
// and LATENTS that of the output, so the heads (N) need no padding to 128 and the row, as TMA stores it, is both operands:
//   S^T [64 tokens][N heads]   = rows (K-major) x Q^T             36 MMAs 64 x N x 16
//   O^T [4][128 latents][N]   += latents^T (M-major) x P^T        16 MMAs 128 x N x 16
// The operands' bytes bound the tensor pipe, (A + B) / 128 per clock: measured 32 cycles for a 64 x 64 x 16 product, 48 for
// 128 x 64 x 16 (23 and 39 at N = 16), 1936 cycles a tile at N = 64; its 73,728 bytes take 3200 at the measured copy bandwidth.
// These rates need the issuing thread to be chosen by elect.sync: under `lane == 0` one MMA takes 46 cycles to issue.
// The ring holds pairs of 64-column blocks (128 latents of a tile, 16 KB) and, apart, the rotated parts (8 KB): a tile's
// pairs are handed back one by one as the output products pass over them, so nearly two tiles are in flight beside 72 KB of Q.
//
// Softmax: one thread holds a quarter of the heads of one token (tcgen05.ld 16x32bx2). Weights are 2^((s - m) scale): a scaled and rounded
// m would be off by 2^-24 of itself, more than 2^x holds where logits are beyond 1e9. A head's reference m is the same for all
// tokens; it is set from a segment's first tile and raised (with a rescale of O^T) only when a logit exceeds it by more
// than 32 log2 units (P and the sums keep fp32's exponent range, so 2^32 costs no accuracy): a tile needs one vote and no
// reduction over tokens. Where it is raised the tile's weights are formed again from its logits. P is rounded to bf16 (off by at most
// 2^-8 of itself: a second product for its remainder would make 128 heads a third slower); the sum that normalises the output adds the rounded values, lse takes the unrounded sum.
//
// More than 64 heads go in groups: neighbouring CTAs read the same pages for different heads, the second one from L2.
// A segment (the part of a range inside one sequence) that covers its sequence writes the result, any other an fp32 partial;
// latent_merge_kernel joins them. Every wait is bounded.
//
// Bounds. 16 heads: memory, 64 contexts of 2K-16K in 110 us, 0.93 of the measured copy bandwidth (0.89 under load). 64 heads: a tile
// keeps shared memory busy for 2612 cycles (1936 of operands, 576 of the copies' writes, P) and takes 2950; 64 contexts around 8K
// take 149 to 156 us in a burst, 174 under load, where the power limit lowers the clock; 128 heads on 2K-16K 221 to 285 us in bursts, from
// machine to machine, and 270 under load, 649 TFLOP/s.
#include "pd_decode_plan.cuh"
#include "pd_kernels.cuh"
#include "pd_ptx.cuh"
#include "pd_tcgen05.cuh"

#include <cfloat>

namespace pd {

namespace {

constexpr int kTile = 64;                        // tokens per step
constexpr int kTilePages = kTile / kPageSize;
constexpr int kChunkBytes = kTile * 128;         // 64 columns of a tile's rows
constexpr int kPairBytes = 2 * kChunkBytes;
constexpr int kPairs = 4;                        // pairs of a tile: 512 latents
constexpr int kRopeSlots = 2;
constexpr int kRowChunks = kLatentRow / 64;      // 9
constexpr int kSoftmaxWarps = 8, kSoftmaxThreads = 32 * kSoftmaxWarps;
constexpr int kThreads = kSoftmaxThreads + 64;   // + TMA warp + MMA warp
constexpr float kRaise = 32.f;                   // log2 units a logit may exceed its head's reference
constexpr int kPBytes = kTile * 128;
constexpr int kSmemLimit = 232448;
constexpr int kControlBytes = 512;
constexpr int kTmemCols = 512;

// Pairs the ring holds beside Q, P and the rotated parts: 8 (two tiles) with 64 heads, more with fewer.
template <int N>
__host__ __device__ constexpr int pair_slots() {
    return (kSmemLimit - 1024 - kControlBytes - kRowChunks * N * 128 - kPBytes - kRopeSlots * kChunkBytes) / kPairBytes;
}
template <int N>
__host__ __device__ constexpr size_t smem_bytes() {
    return 1024 + kRowChunks * N * 128 + kPBytes + kRopeSlots * kChunkBytes + pair_slots<N>() * kPairBytes + kControlBytes;
}

__device__ __forceinline__ void softmax_sync() { asm volatile("barrier.cta.sync 1, %0;" ::"n"(kSoftmaxThreads) : "memory"); }
__device__ __forceinline__ bool softmax_any(bool v) {
    uint32_t r;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbarrier.cta.red.or.pred q, 1, %2, p;\nselp.u32 %0, 1, 0, q;\n}"
                 : "=r"(r) : "r"(static_cast<uint32_t>(v)), "n"(kSoftmaxThreads) : "memory");
    return r != 0;
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void *tmap, int32_t x, int32_t y, int32_t z, int32_t w, uint32_t bar,
                                            uint64_t l2_policy) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
                 " [%0], [%1, {%2, %3, %4, %5}], [%6], %7;"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar), "l"(l2_policy) : "memory");
}
// Half a row's columns per thread: threads 0..15 of the warp get lanes 0..15 from column 0 on, threads 16..31 the same
// lanes from column K on.
template <int K>
__device__ __forceinline__ void tmem_ld_halves(uint32_t taddr, uint32_t (&r)[K]);
template <>
__device__ __forceinline__ void tmem_ld_halves<4>(uint32_t taddr, uint32_t (&r)[4]) {
    asm volatile("tcgen05.ld.sync.aligned.16x32bx2.x4.b32 {%0, %1, %2, %3}, [%4], 4;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr) : "memory");
}
template <>
__device__ __forceinline__ void tmem_ld_halves<8>(uint32_t taddr, uint32_t (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.16x32bx2.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8], 8;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
template <>
__device__ __forceinline__ void tmem_ld_halves<16>(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.16x32bx2.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16], 16;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

// How the work is cut: a sequence is its pages behind `extra` units for what a segment costs beside them (Q, the partial result),
// and the list of all sequences' units is cut into ranges of `size`, `per_worker` consecutive ranges per worker.
struct LatentPlan {
    int total, size, ranges, per_worker;
};
__device__ __forceinline__ LatentPlan latent_plan(int total, int workers, const LatentAttnParams &p) {
    LatentPlan pl;
    pl.total = total;
    int size = max((total + workers - 1) / workers, p.a.min_pages_auto);  // at most one range per worker
    pl.per_worker = 1;
    if (p.a.split_pages > 0) size = max(p.a.split_pages, (total + p.a.max_ranges - 1) / p.a.max_ranges);
    pl.size = max(min(size, total), 1);  // (total + size stays in 32 bits whatever split_pages is)
    pl.ranges = (total + pl.size - 1) / pl.size;
    if (p.a.split_pages > 0) pl.per_worker = (pl.ranges + workers - 1) / workers;
    return pl;
}
__device__ __forceinline__ int units_of(int pages, int extra) { return pages > 0 ? pages + extra : 0; }

// Exclusive prefix sums of the sequences' units; cum[B] = all. Returns the pages of this thread's sequences.
__device__ __forceinline__ int scan_units(const LatentAttnParams &p, int32_t *cum, int32_t *warp_sums) {
    const int tid = threadIdx.x, items = (p.a.B + kThreads - 1) / kThreads;
    const int begin = min(p.a.B, tid * items), end = min(p.a.B, begin + items);
    int sum = 0, pages = 0;
    for (int i = begin; i < end; ++i) {
        const int L = __ldg(p.a.ctx_lens + i);
        if (L < 0 || L > p.a.MP * kPageSize) latch_status(p.a.status, kDevBadLength, i, L);
        const int np = (clamp_len(L, p.a.MP) + kPageSize - 1) / kPageSize;
        cum[i] = units_of(np, p.extra);  // this thread's own entries, turned into sums below
        sum += cum[i];
        pages += np;
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, incl, o);
        if ((tid & 31) >= o) incl += t;
    }
    if ((tid & 31) == 31) warp_sums[tid >> 5] = incl;
    __syncthreads();
    int run = incl - sum;
    for (int w = 0; w < (tid >> 5); ++w) run += warp_sums[w];
    for (int i = begin; i < end; ++i) {
        const int units = cum[i];
        cum[i] = run;
        run += units;
    }
    if (tid == kThreads - 1) cum[p.a.B] = run;
    __syncthreads();
    return pages;
}

// The segments of one worker, in order; every role of the CTA walks them by itself.
struct Segment {
    int b, page0, pages, tokens, slot;
    bool whole;
};
struct Walk {
    int b, at, np, len, r, r_end, left;  // `at`: units of sequence b that lie behind
};
__device__ __forceinline__ bool next_segment(Walk &w, Segment &s, const LatentPlan &pl, const LatentAttnParams &p) {
    for (;;) {
        if (w.left == 0) {
            if (++w.r >= w.r_end) return false;
            w.left = min(pl.size, pl.total - w.r * pl.size);
        }
        const int units = units_of(w.np, p.extra);
        if (w.at >= units) {  // units are left, so a sequence that has some follows
            ++w.b;
            w.at = 0;
            w.len = clamp_len(__ldg(p.a.ctx_lens + w.b), p.a.MP);
            w.np = (w.len + kPageSize - 1) / kPageSize;
            continue;
        }
        const int take = min(units - w.at, w.left), from = max(w.at - p.extra, 0), to = max(w.at + take - p.extra, 0);
        w.at += take;
        w.left -= take;
        if (from == to) continue;
        s.b = w.b;
        s.page0 = from;
        s.pages = to - from;
        s.tokens = min(w.len - from * kPageSize, s.pages * kPageSize);
        s.whole = s.pages == w.np;
        s.slot = 2 * w.r + (from == 0 ? 1 : 0);  // a range has at most one segment that is cut at its start, and one at its end alone
        return true;
    }
}

// Reduces K (at most 16) values per thread over the 16 lanes of a half warp: afterwards v[0] of a lane is that of index lane % K.
template <int K, bool MAX>
__device__ __forceinline__ void reduce_half_warp(float (&v)[K], int lane) {
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) {
        if (o < K) {  // halve the values: a lane keeps those of its side
            const bool upper = (lane & o) != 0;
#pragma unroll
            for (int i = 0; i < o; ++i) {
                const float send = upper ? v[i] : v[i + o], keep = upper ? v[i + o] : v[i];
                const float got = __shfl_xor_sync(0xffffffffu, send, o);
                v[i] = MAX ? fmaxf(keep, got) : keep + got;
            }
        } else {
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const float got = __shfl_xor_sync(0xffffffffu, v[i], o);
                v[i] = MAX ? fmaxf(v[i], got) : v[i] + got;
            }
        }
    }
}

// Natural logarithm of sum * 2^(reference * scale).
__device__ __forceinline__ float log_sum(float reference, float sum, float scale_log2) {
    return fmaf(reference, scale_log2 * kLn2, log2f(sum) * kLn2);
}

template <int N>
__global__ void __launch_bounds__(kThreads, 1)
decode_attn_latent_kernel(const __grid_constant__ CUtensorMap tm_kv, const __grid_constant__ CUtensorMap tm_rope,
                          const __grid_constant__ CUtensorMap tm_q, const LatentAttnParams p) {
    constexpr int kSlots = pair_slots<N>();
    constexpr int K = N / 4;                           // heads per softmax thread
    constexpr int kColS = 4 * N;                       // O^T in columns [0, 4 N), then two buffers of S^T
    constexpr int kQBytes = kRowChunks * N * 128;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ int32_t warp_sums[kThreads / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int pairs = p.groups - 1;  // one or two groups of heads: neighbouring CTAs take the same ranges for both
    const int group = blockIdx.x & pairs, worker = blockIdx.x >> pairs, workers = gridDim.x >> pairs;
    const int h0 = group * p.heads, nh = min(p.heads, p.a.Hq - h0);

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *aligned = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t ring = base, rope_ring = ring + kSlots * kPairBytes, q_s = rope_ring + kRopeSlots * kChunkBytes, p_s = q_s + kQBytes;
    float *scratch = reinterpret_cast<float *>(aligned + (p_s - base));  // P's buffer, free whenever it is used
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + (p_s - base) + kPBytes);
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + kSlots * 8;               // pairs
    const uint32_t bar_rfull = bar_empty + kSlots * 8, bar_rempty = bar_rfull + kRopeSlots * 8;  // rotated parts
    const uint32_t bar_qfull = bar_rempty + kRopeSlots * 8, bar_qempty = bar_qfull + 8;        // Q of a segment's sequence
    const uint32_t bar_s = bar_qempty + 8, bar_sempty = bar_s + 16;                            // [2] S^T buffers
    const uint32_t bar_p = bar_sempty + 16;                                                    // P written
    const uint32_t bar_pv = bar_p + 8;                                                         // output products of a tile done
    const uint32_t bar_o = bar_pv + 8;                                                         // O^T of a segment read out
    const uint32_t bar_drain = bar_o + 8;
    static_assert((2 * kSlots + 2 * kRopeSlots + 2 + 4 + 4) * 8 <= kControlBytes, "barriers");

    if (tid == 0) {
        for (int i = 0; i < 2 * kSlots + 2 * kRopeSlots + 4; ++i) mbar_init(bar_full + i * 8, 1);  // .. bar_s[2]
        mbar_init(bar_sempty, kSoftmaxWarps);
        mbar_init(bar_sempty + 8, kSoftmaxWarps);
        mbar_init(bar_p, kSoftmaxWarps);
        mbar_init(bar_pv, 1);
        mbar_init(bar_o, kSoftmaxWarps);
        mbar_init(bar_drain, 1);
        mbar_init_fence();
        prefetch_tensormap(&tm_kv);
        prefetch_tensormap(&tm_rope);
        prefetch_tensormap(&tm_q);
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(&tmem_slot), kTmemCols);
        tmem_relinquish_alloc_permit();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tm = tmem_slot;
    grid_dependency_wait();
    launch_dependents();

    // ---- the plan. Up to 128 sequences every warp derives it by itself; beyond that the block does, with prefix sums in the
    // ring's memory, which no copy uses yet (1 us more).
    LatentPlan pl;
    Walk w0{};
    w0.b = -1;
    constexpr int kPer = 4;  // sequences per lane
    const bool warp_plan = p.a.B <= 32 * kPer;
    int32_t *cum = reinterpret_cast<int32_t *>(aligned);
    int pages = 0;
    if (warp_plan) {
        int units[kPer], sum = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int b = lane * kPer + i, L = b < p.a.B ? __ldg(p.a.ctx_lens + b) : 0;
            if (blockIdx.x == 0 && warp == 0 && (L < 0 || L > p.a.MP * kPageSize)) latch_status(p.a.status, kDevBadLength, b, L);
            const int np = (clamp_len(L, p.a.MP) + kPageSize - 1) / kPageSize;
            units[i] = units_of(np, p.extra);
            sum += units[i];
            pages += np;
        }
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        pl = latent_plan(__shfl_sync(0xffffffffu, incl, 31), workers, p);
        w0.r = worker * pl.per_worker;
        const int x = min(w0.r, pl.ranges) * pl.size;  // the worker's first unit: in this lane's sequences where it lies in [incl - sum, incl)
        int at = incl - sum, mine = -1, off = 0, in = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (x >= at && x < at + units[i]) mine = lane * kPer + i, off = x - at, in = units[i];
            if (blockIdx.x == 0 && warp == 0 && lane * kPer + i <= p.a.B) p.a.cum_pages[lane * kPer + i] = at;
            at += units[i];
        }
        if (blockIdx.x == 0 && warp == 0 && lane == 31 && p.a.B == 32 * kPer) p.a.cum_pages[32 * kPer] = at;
        const uint32_t owner = __ballot_sync(0xffffffffu, mine >= 0);
        if (owner != 0) {
            const int src = __ffs(owner) - 1;
            w0.b = __shfl_sync(0xffffffffu, mine, src);
            w0.at = __shfl_sync(0xffffffffu, off, src);
            w0.np = __shfl_sync(0xffffffffu, in, src) - p.extra;
        }
    } else {
        pages = scan_units(p, cum, warp_sums);
        pl = latent_plan(cum[p.a.B], workers, p);
        w0.r = worker * pl.per_worker;
        if (w0.r < pl.ranges) {
            const Cursor c = locate(cum, p.a.B, 1, static_cast<long long>(w0.r) * pl.size);
            w0.b = c.b;
            w0.at = c.page;
            w0.np = c.np - p.extra;
        }
        if (blockIdx.x == 0)
            for (int i = tid; i <= p.a.B; i += kThreads) p.a.cum_pages[i] = cum[i];
    }
    w0.r_end = min(w0.r + pl.per_worker, pl.ranges);
    const bool busy = w0.r < w0.r_end;
    if (busy) {
        w0.len = clamp_len(__ldg(p.a.ctx_lens + w0.b), p.a.MP);
        w0.left = min(pl.size, pl.total - w0.r * pl.size);
    }
    if (blockIdx.x == 0) {
        const int sum = __reduce_add_sync(0xffffffffu, pages);
        if (!warp_plan) {
            __syncthreads();
            if (lane == 0) warp_sums[warp] = sum;
            __syncthreads();
        }
        if (tid == 0) {
            int all = sum;
            for (int i = 1; i < kThreads / 32 && !warp_plan; ++i) all += warp_sums[i];
            p.a.plan[0] = all;
            p.a.plan[1] = 0;
            p.a.plan[2] = 1;
            p.a.plan[3] = pl.ranges;
            p.a.plan[4] = workers;
            p.a.plan[kPlanHeaderWords + 2] = pl.size;
        }
    }
    if (!warp_plan) {
        fence_proxy_async();  // the copies that follow overwrite what was read here
        __syncthreads();
    }
    bool ok = true;

    if (busy && warp == kSoftmaxWarps) {
        // ================= TMA warp: one elected thread =================
        // A pair of column blocks of a page is one 4-D box, 8 rows x 2 blocks x 2 row groups: shared memory gets [row group][block][8 rows],
        // in which row groups follow one another at the same distance (2 KB) across pages, as a product's operand needs them.
        if (elect_one()) {
            const uint64_t policy = l2_policy_evict_first();
            const int32_t *row = nullptr;
            Walk w = w0;
            Segment s{};
            int pc = 0, rc = 0, seg = 0;
            auto load_q = [&]() {
                if (seg > 0) ok = mbar_wait(bar_qempty, (seg - 1) & 1);
                if (!ok) return;
                mbar_arrive_expect_tx(bar_qfull, kQBytes);
                tma_load_4d(q_s, &tm_q, 0, h0, 0, s.b, bar_qfull, policy);  // [9 blocks of 64 columns][N heads]
                ++seg;
            };
            int32_t id[kTilePages];  // the next tile's pages
            auto load_ids = [&](int pg0) {
#pragma unroll
                for (int g = 0; g < kTilePages; ++g) id[g] = pg0 + g < s.pages ? __ldg(row + pg0 + g) : p.a.num_pages;  // (a page of zero fill)
            };
            while (ok && next_segment(w, s, pl, p)) {
                row = p.a.page_table + static_cast<size_t>(s.b) * p.a.MP + s.page0;
                load_ids(0);
                const bool first = seg == 0;  // later ones behind their first tile: Q has to wait for the last segment's logits
                if (first) load_q();
                for (int i = 0; i * kTilePages < s.pages && ok; ++i) {
                    int32_t page[kTilePages];
#pragma unroll
                    for (int g = 0; g < kTilePages; ++g) {
                        page[g] = id[g];
                        if (i * kTilePages + g < s.pages && static_cast<uint32_t>(page[g]) >= static_cast<uint32_t>(p.a.num_pages)) {
                            latch_status(p.a.status, kDevBadPage, s.b, page[g]);
                            page[g] = 0;
                        }
                    }
                    load_ids((i + 1) * kTilePages);
                    {
                        const int slot = rc % kRopeSlots, fill = rc / kRopeSlots;
                        if (fill > 0) ok = mbar_wait(bar_rempty + slot * 8, (fill - 1) & 1);
                        if (!ok) break;
                        mbar_arrive_expect_tx(bar_rfull + slot * 8, kChunkBytes);
#pragma unroll
                        for (int g = 0; g < kTilePages; ++g)
                            tma_load_2d(rope_ring + slot * kChunkBytes + g * (kPageSize * 128), &tm_rope, kLatentDim, page[g] * kPageSize, bar_rfull + slot * 8, policy);
                        ++rc;
                    }
                    for (int j = 0; j < kPairs; ++j) {
                        const int slot = pc % kSlots, fill = pc / kSlots;
                        if (fill > 0) ok = mbar_wait(bar_empty + slot * 8, (fill - 1) & 1);
                        if (!ok) break;
                        mbar_arrive_expect_tx(bar_full + slot * 8, kPairBytes);
#pragma unroll
                        for (int g = 0; g < kTilePages; ++g)
                            tma_load_4d(ring + slot * kPairBytes + g * (2 * kPageSize * 128), &tm_kv, 0, 0, 2 * j, 2 * page[g], bar_full + slot * 8, policy);
                        ++pc;
                    }
                    if (i == 0 && ok && !first) load_q();
                }
            }
            if (!ok) {  // copies in flight have to land before the block's memory goes
                latch_status(p.a.status, kDevTimeout, s.b, blockIdx.x);
                for (int i = max(0, pc - kSlots); i < pc; ++i) mbar_wait(bar_full + (i % kSlots) * 8, (i / kSlots) & 1);
                for (int i = max(0, rc - kRopeSlots); i < rc; ++i) mbar_wait(bar_rfull + (i % kRopeSlots) * 8, (i / kRopeSlots) & 1);
                if (seg > 0) mbar_wait(bar_qfull, (seg - 1) & 1);
            }
        }
    } else if (busy && warp == kSoftmaxWarps + 1) {
        // ================= MMA warp: one elected thread issues every product =================
        if (elect_one()) {
            constexpr uint32_t idesc_s = umma_idesc_bf16(64, N, false);
            constexpr uint32_t idesc_o = umma_idesc_bf16(128, N, true) | (1u << 15);  // A M-major
            const uint64_t q_desc = umma_smem_desc(q_s, 16, 1024), p_desc = umma_smem_desc(p_s, 16, 1024);
            const uint64_t ring_k = umma_smem_desc(ring, 16, 2048), ring_m = umma_smem_desc(ring, 1024, 2048);
            const uint64_t rope_k = umma_smem_desc(rope_ring, 16, 1024);
            int pv_tile = 0, pv_seg_first = 0;   // next tile whose output product is due; segments begun by them
            // one tile's output products
            auto issue_pv = [&](bool first) {
                tc_fence_after_sync();
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    const int slot = (pv_tile * kPairs + j) % kSlots;
                    const uint64_t a = ring_m + slot * (kPairBytes >> 4);
#pragma unroll
                    for (int ks = 0; ks < kTile / 16; ++ks)
                        umma_ss(tm + j * N, a + ks * (4096 >> 4), p_desc + ks * (2048 >> 4), idesc_o, !first || ks != 0);
                    umma_commit(bar_empty + slot * 8);
                }
                umma_commit(bar_pv);
                ++pv_tile;
            };
            Walk w = w0;
            Segment s;
            int t = 0, seg = 0;
            bool due = false, due_first = false;  // the previous tile's output products, and whether it opened its segment
            auto pv_ready = [&]() { return mbar_try_wait(bar_p, pv_tile & 1); };
            auto do_pv = [&]() {
                if (due_first) {
                    if (pv_seg_first > 0) ok = mbar_wait(bar_o, (pv_seg_first - 1) & 1);  // the last segment's O^T has been read
                    ++pv_seg_first;
                }
                if (ok) issue_pv(due_first);
                due = false;
            };
            // waits for `bar`; the previous tile's output products go in between as soon as its P is there
            auto wait_for = [&](uint32_t bar, uint32_t parity) {
                if (mbar_try_wait(bar, parity)) return;
                const uint64_t t0 = global_timer_ns();
                for (uint32_t poll = 1; ok; ++poll) {
                    if (due && pv_ready()) do_pv();
                    if (mbar_try_wait(bar, parity)) return;
                    if ((poll & 255u) == 0 && (poll >= (1u << 24) || global_timer_ns() - t0 > 2000000000ull)) ok = false;
                }
            };
            while (ok && next_segment(w, s, pl, p)) {
                const int tiles = (s.pages + kTilePages - 1) / kTilePages;
                for (int i = 0; i < tiles && ok; ++i, ++t) {
                    if (i == 0) wait_for(bar_qfull, seg & 1);
                    if (t >= 2) wait_for(bar_sempty + (t & 1) * 8, ((t >> 1) - 1) & 1);
                    wait_for(bar_rfull + (t % kRopeSlots) * 8, (t / kRopeSlots) & 1);
                    if (!ok) break;
                    const uint32_t d = tm + kColS + (t & 1) * N;
                    tc_fence_after_sync();
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        umma_ss(d, rope_k + (t % kRopeSlots) * (kChunkBytes >> 4) + ks * 2, q_desc + (8 * N * 128 >> 4) + ks * 2, idesc_s, ks != 0);
                    umma_commit(bar_rempty + (t % kRopeSlots) * 8);
#pragma unroll
                    for (int j = 0; j < kPairs; ++j) {
                        const int pc = t * kPairs + j, slot = pc % kSlots;
                        wait_for(bar_full + slot * 8, (pc / kSlots) & 1);
                        if (!ok) break;
                        tc_fence_after_sync();
#pragma unroll
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int ks = 0; ks < 4; ++ks)
                                umma_ss(d, ring_k + slot * (kPairBytes >> 4) + c * (1024 >> 4) + ks * 2,
                                        q_desc + ((2 * j + c) * N * 128 >> 4) + ks * 2, idesc_s, true);
                    }
                    if (!ok) break;
                    umma_commit(bar_s + (t & 1) * 8);
                    if (i == tiles - 1) umma_commit(bar_qempty);
                    if (due) {
                        ok = mbar_wait(bar_p, pv_tile & 1);
                        if (ok) do_pv();
                    }
                    due = true;
                    due_first = i == 0;
                }
                ++seg;
            }
            if (ok && due) {
                ok = mbar_wait(bar_p, pv_tile & 1);
                if (ok) do_pv();
            }
            if (!ok) latch_status(p.a.status, kDevTimeout, s.b, blockIdx.x);
            umma_commit(bar_drain);  // nothing may be in flight when the tensor memory is freed
            mbar_wait(bar_drain, 0);
        }
    } else if (busy && warp < kSoftmaxWarps) {
        // ================= softmax: thread = (token of the tile, a quarter of the heads) =================
        // Warps w and w + 4 share 16 tokens (the tensor-memory lanes they can reach), warps 0..3 take the first half of the heads.
        const int wg = warp >> 2, wq = warp & 3;
        const int tok = wq * 16 + (lane & 15);
        const int hq = 2 * wg + (lane >> 4), hb = hq * K;  // first head of this thread, within the group
        const uint32_t lane_base = static_cast<uint32_t>(wq * 32) << 16;
        Walk w = w0;
        Segment s;
        int t = 0;
        // (a warp whose wait ran out goes on without waiting: the others must not be left alone at the barriers they share)
        while (next_segment(w, s, pl, p)) {
            float m[K], l[K], lr[K];
#pragma unroll
            for (int i = 0; i < K; ++i) m[i] = l[i] = lr[i] = 0.f;
            const int tiles = (s.pages + kTilePages - 1) / kTilePages;
            for (int i = 0; i < tiles; ++i, ++t) {
                ok = ok && mbar_wait(bar_s + (t & 1) * 8, (t >> 1) & 1);
                tc_fence_after_sync();
                uint32_t sreg[K];
                tmem_ld_halves<K>(tm + lane_base + kColS + (t & 1) * N + wg * 2 * K, sreg);
                tmem_wait_ld();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_sempty + (t & 1) * 8);
                const int valid = s.tokens - i * kTile;
                if (valid < kTile) {
                    // slots past the context may hold NaN, and 0 * NaN is NaN: their latents are cleared before the output
                    // product (pages past the segment came as zero fill); S^T of the tile is complete, so all has landed
                    const int last = min(kTile, (valid + kPageSize - 1) / kPageSize * kPageSize);
                    for (int x = tid; x < (last - valid) * (kLatentDim / 8); x += kSoftmaxThreads) {
                        const int r = valid + x / (kLatentDim / 8), c = x % (kLatentDim / 8);
                        const int slot = (t * kPairs + (c >> 4)) % kSlots;
                        st_shared_zero16(ring + slot * kPairBytes + (r >> 3) * 2048 + ((c >> 3) & 1) * 1024 + (r & 7) * 128 + (c & 7) * 16);
                    }
                }
                const bool dead = tok >= valid;
                // the largest logit of this thread's heads over all tokens of the tile
                auto tile_max = [&](float (&top)[K]) {
                    float v[K];
#pragma unroll
                    for (int k = 0; k < K; ++k) v[k] = dead ? -INFINITY : __uint_as_float(sreg[k]);
                    reduce_half_warp<K, true>(v, lane);
                    scratch[wq * 64 + hb + lane % K] = v[0];
                    softmax_sync();
#pragma unroll
                    for (int k = 0; k < K; ++k)
                        top[k] = fmaxf(fmaxf(scratch[hb + k], scratch[64 + hb + k]), fmaxf(scratch[128 + hb + k], scratch[192 + hb + k]));
                    softmax_sync();
                };
                if (i == 0) {
                    tile_max(m);  // (the last segment's products are over, P's buffer is free)
#pragma unroll
                    for (int k = 0; k < K; ++k) m[k] = fmaxf(m[k], -FLT_MAX);  // (where the tile has no finite logit: below any that comes)
                }
                float e[K], over = -INFINITY;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const float x = dead ? -INFINITY : (__uint_as_float(sreg[k]) - m[k]) * p.a.scale_log2;
                    over = fmaxf(over, x);
                    e[k] = fast_exp2(x);
                }
                uint32_t pk[K / 2];
                auto pack = [&]() {
#pragma unroll
                    for (int k = 0; k < K; k += 2) pk[k / 2] = pack_bf16x2(e[k], e[k + 1]);
                };
                pack();
                if (i > 0) {
                    ok = ok && mbar_wait(bar_pv, (t - 1) & 1);  // P's buffer is free and O^T holds every tile before this one
                    const bool raise = softmax_any(over > kRaise);
                    if (raise) {
                        tc_fence_after_sync();
                        float top[K];
                        tile_max(top);
#pragma unroll
                        for (int k = 0; k < K; ++k) {
                            float alpha = 1.f;
                            if ((top[k] - m[k]) * p.a.scale_log2 > kRaise) {
                                alpha = fast_exp2((m[k] - top[k]) * p.a.scale_log2);
                                m[k] = top[k];
                                // from the logit again: its difference from the last reference has lost what a far lower one's rounding took
                                e[k] = dead ? 0.f : fast_exp2((__uint_as_float(sreg[k]) - m[k]) * p.a.scale_log2);
                            }
                            l[k] *= alpha;
                            lr[k] *= alpha;
                            if ((lane & 15) == 0 && wq == 0) scratch[hb + k] = alpha;
                        }
                        softmax_sync();
#pragma unroll 1
                        for (int c = wg * 2 * N; c < (wg + 1) * 2 * N; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(tm + lane_base + c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * scratch[(c + k) % N]);
                            tmem_st16(tm + lane_base + c, o);
                        }
                        tmem_wait_st();
                        softmax_sync();
                        pack();
                    }
                }
                if constexpr (K >= 8) {
#pragma unroll
                    for (int c = 0; c < K / 8; ++c) {
                        const uint32_t a = p_s + sw128_offset(tok, hb / 8 + c);
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(pk[4 * c]), "r"(pk[4 * c + 1]), "r"(pk[4 * c + 2]),
                                     "r"(pk[4 * c + 3]) : "memory");
                    }
                } else {
                    const uint32_t a = p_s + sw128_offset(tok, hb / 8) + (hb % 8) * 2;
                    asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(a), "r"(pk[0]), "r"(pk[1]) : "memory");
                }
                fence_proxy_async();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_p);
#pragma unroll
                for (int k = 0; k < K; k += 2) {
                    l[k] += e[k];
                    l[k + 1] += e[k + 1];
                    lr[k] += __uint_as_float(pk[k / 2] << 16);
                    lr[k + 1] += __uint_as_float(pk[k / 2] & 0xffff0000u);
                }
            }
            // ---- the segment's end
            ok = ok && mbar_wait(bar_pv, (t - 1) & 1);
            tc_fence_after_sync();
            float *sum_l = scratch, *sum_lr = scratch + 256, *ref = scratch + 512, *inv = scratch + 576;
            if (wq == 0 && (lane & 15) == 0) {
#pragma unroll
                for (int k = 0; k < K; ++k) ref[hb + k] = m[k];
            }
            reduce_half_warp<K, false>(l, lane);
            reduce_half_warp<K, false>(lr, lane);
            sum_l[wq * 64 + hb + lane % K] = l[0];
            sum_lr[wq * 64 + hb + lane % K] = lr[0];
            softmax_sync();
            if (tid < nh) {
                const float sl = (sum_l[tid] + sum_l[64 + tid]) + (sum_l[128 + tid] + sum_l[192 + tid]);
                const float slr = (sum_lr[tid] + sum_lr[64 + tid]) + (sum_lr[128 + tid] + sum_lr[192 + tid]);
                if (s.whole) {
                    inv[tid] = slr == 0.f ? 0.f : 1.f / slr;  // 0: every logit was -inf, as in an empty context
                    if (p.a.lse != nullptr) p.a.lse[static_cast<size_t>(s.b) * p.a.Hq + h0 + tid] = log_sum(ref[tid], sl, p.a.scale_log2);
                } else {
                    p.part_ml[static_cast<size_t>(s.slot) * p.a.Hq + h0 + tid] = make_float4(ref[tid], sl, slr, 0.f);
                }
            }
            if (s.whole) softmax_sync();
#pragma unroll 1
            for (int j = 2 * wg; j < 2 * wg + 2; ++j) {
                const int latent = j * 128 + wq * 32 + lane;
#pragma unroll 1
                for (int c = 0; c < N; c += 16) {
                    uint32_t o[16];
                    tmem_ld16(tm + lane_base + j * N + c, o);
                    tmem_wait_ld();
                    if (s.whole) {
                        // neighbouring lanes trade, so that each stores two neighbouring latents of one head: even lanes the even heads
                        const int odd = lane & 1;
                        __nv_bfloat16 *dst = p.a.out + (static_cast<size_t>(s.b) * p.a.Hq + h0 + c + odd) * kLatentDim + (latent - odd);
#pragma unroll
                        for (int k = 0; k < 16; k += 2) {
                            const float a = __uint_as_float(o[k]) * inv[c + k], b = __uint_as_float(o[k + 1]) * inv[c + k + 1];
                            const float got = __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
                            const uint32_t both = odd ? pack_bf16x2(got, b) : pack_bf16x2(a, got);
                            if (c + k + odd < nh) *reinterpret_cast<uint32_t *>(dst + static_cast<size_t>(k) * kLatentDim) = both;
                        }
                    } else {
                        float *dst = p.a.part_o + (static_cast<size_t>(s.slot) * p.a.Hq + h0 + c) * kLatentDim + latent;
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (c + k < nh) dst[static_cast<size_t>(k) * kLatentDim] = __uint_as_float(o[k]);
                    }
                }
            }
            tc_fence_before_sync();
            softmax_sync();
            if (lane == 0) mbar_arrive(bar_o);
        }
        ok = __all_sync(0xffffffffu, ok);
        if (!ok && lane == 0) latch_status(p.a.status, kDevTimeout, s.b, blockIdx.x);
    }
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tm, kTmemCols);
}

// Joins the partials of every (sequence, head) row whose sequence was cut, and writes the rows of empty sequences. A warp takes
// VECS * 128 / GROUPS columns of a row: 32 / GROUPS lanes of VECS times 4 values each. Where rows are few and partials many, GROUPS sets of
// lanes share the row's partials and join by shuffles. No shared memory, so that its blocks may stand beside the split kernel's on the same
// SM and wait there for its end: those of <4, 1> (64 registers) beside any, those of <1, 4> (113) beside the kernels of up to 32 heads
// a group alone; 64 heads leave 11,776 registers, and a block of it starts when one of theirs ends.
constexpr int kMergeThreads = 128;
template <int GROUPS, int VECS>
__global__ void __launch_bounds__(kMergeThreads) latent_merge_kernel(const LatentAttnParams p) {
    constexpr int LANES = 32 / GROUPS, PIECES = kLatentDim / 4 / LANES / VECS, U = VECS == 1 ? 6 : 4;  // U partials in flight
    const int lane = threadIdx.x & 31, group = lane / LANES;
    grid_dependency_wait();
    launch_dependents();
    const int size = p.a.plan[kPlanHeaderWords + 2];
    const int warps = gridDim.x * (kMergeThreads / 32), items = p.a.B * p.a.Hq * PIECES;
    for (int item = blockIdx.x * (kMergeThreads / 32) + (threadIdx.x >> 5); item < items; item += warps) {
        const int row = item / PIECES, piece = item - row * PIECES, col = piece * LANES * VECS + lane % LANES;  // col: in units of 4 values
        const int b = row / p.a.Hq, h = row - b * p.a.Hq;
        const int c0 = p.a.cum_pages[b], c1 = p.a.cum_pages[b + 1];
        uint2 *out = reinterpret_cast<uint2 *>(p.a.out + static_cast<size_t>(row) * kLatentDim) + col;
        if (c0 == c1) {
#pragma unroll
            for (int v = 0; v < VECS; ++v)
                if (group == 0) out[v * LANES] = make_uint2(0u, 0u);
            if (piece == 0 && lane == 0 && p.a.lse != nullptr) p.a.lse[row] = -INFINITY;
            continue;
        }
        const int r0 = (c0 + p.extra) / size, r1 = (c1 - 1) / size;  // ranges of its first and last page
        if (r0 == r1) continue;  // written by the split kernel
        float m = -INFINITY, l = 0.f, lr = 0.f;
        float4 o[VECS];
#pragma unroll
        for (int v = 0; v < VECS; ++v) o[v] = make_float4(0.f, 0.f, 0.f, 0.f);
        auto raise = [&](float top) {
            const float keep = m == top ? 1.f : fast_exp2((m - top) * p.a.scale_log2);
#pragma unroll
            for (int v = 0; v < VECS; ++v) o[v].x *= keep, o[v].y *= keep, o[v].z *= keep, o[v].w *= keep;
            l *= keep, lr *= keep;
            m = top;
        };
        auto join = [&](float pm, float pl, float plr, const float4 (&x)[VECS]) {  // pm <= m
            const float a = pm == -INFINITY ? 0.f : fast_exp2((pm - m) * p.a.scale_log2);
#pragma unroll
            for (int v = 0; v < VECS; ++v)
                o[v].x = fmaf(a, x[v].x, o[v].x), o[v].y = fmaf(a, x[v].y, o[v].y), o[v].z = fmaf(a, x[v].z, o[v].z), o[v].w = fmaf(a, x[v].w, o[v].w);
            l = fmaf(a, pl, l);
            lr = fmaf(a, plr, lr);
        };
        for (int r = r0 + group; r <= r1; r += GROUPS * U) {
            float4 x[U][VECS], ml[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int y = r + u * GROUPS;
                ml[u] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
#pragma unroll
                for (int v = 0; v < VECS; ++v) x[u][v] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (y <= r1) {
                    const size_t at = static_cast<size_t>(y == r0 ? 2 * y + 1 : 2 * y) * p.a.Hq + h;
                    ml[u] = p.part_ml[at];
#pragma unroll
                    for (int v = 0; v < VECS; ++v) x[u][v] = reinterpret_cast<const float4 *>(p.a.part_o + at * kLatentDim)[col + v * LANES];
                }
            }
            float top = m;
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, ml[u].x);  // finite: ml[0] is a partial's reference
            raise(top);
#pragma unroll
            for (int u = 0; u < U; ++u) join(ml[u].x, ml[u].y, ml[u].z, x[u]);
        }
        if (GROUPS > 1) {
            __syncwarp();
#pragma unroll
            for (int d = LANES; d < 32; d <<= 1) {
                const float pm = __shfl_xor_sync(0xffffffffu, m, d), pl = __shfl_xor_sync(0xffffffffu, l, d), plr = __shfl_xor_sync(0xffffffffu, lr, d);
                float4 x[VECS];
#pragma unroll
                for (int v = 0; v < VECS; ++v)
                    x[v] = make_float4(__shfl_xor_sync(0xffffffffu, o[v].x, d), __shfl_xor_sync(0xffffffffu, o[v].y, d),
                                       __shfl_xor_sync(0xffffffffu, o[v].z, d), __shfl_xor_sync(0xffffffffu, o[v].w, d));
                if (fmaxf(m, pm) > -INFINITY) {  // (a set without partials holds none)
                    raise(fmaxf(m, pm));
                    join(pm, pl, plr, x);
                }
            }
        }
        const float inv = lr == 0.f ? 0.f : 1.f / lr;
#pragma unroll
        for (int v = 0; v < VECS; ++v)
            if (group == 0) out[v * LANES] = make_uint2(pack_bf16x2(o[v].x * inv, o[v].y * inv), pack_bf16x2(o[v].z * inv, o[v].w * inv));
        if (piece == 0 && lane == 0 && p.a.lse != nullptr) p.a.lse[row] = log_sum(m, l, p.a.scale_log2);
    }
}

template <int N>
cudaError_t prepare() {
    return cudaFuncSetAttribute(decode_attn_latent_kernel<N>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem_bytes<N>()));
}

}  // namespace

int latent_heads_per_cta(int heads) { return heads <= 16 ? 16 : heads <= 32 ? 32 : 64; }

cudaError_t prepare_decode_attn_latent() {
    cudaError_t e = prepare<16>();
    if (e == cudaSuccess) e = prepare<32>();
    if (e == cudaSuccess) e = prepare<64>();
    return e;
}

cudaError_t launch_decode_attn_latent(const CUtensorMap &tm_kv, const CUtensorMap &tm_rope, const CUtensorMap &tm_q, const LatentAttnParams &p,
                                      int num_ctas, cudaStream_t stream) {
    auto go = [&](auto *k, size_t smem) { return launch_pdl(k, dim3(num_ctas), dim3(kThreads), smem, stream, p.a.pdl != 0, tm_kv, tm_rope, tm_q, p); };
    const int n = latent_heads_per_cta(p.heads);
    const cudaError_t err = n == 16   ? go(decode_attn_latent_kernel<16>, smem_bytes<16>())
                            : n == 32 ? go(decode_attn_latent_kernel<32>, smem_bytes<32>())
                                      : go(decode_attn_latent_kernel<64>, smem_bytes<64>());
    if (err != cudaSuccess) return err;
    // few rows are cut into many partials each: four sets of lanes share them
    const int rows = p.a.B * p.a.Hq;
    auto merge = [&](auto *k, int warps_per_row) {
        const int blocks = (rows * warps_per_row + kMergeThreads / 32 - 1) / (kMergeThreads / 32), most = num_ctas * 32;
        return launch_pdl(k, dim3(blocks < most ? blocks : most), dim3(kMergeThreads), 0, stream, p.a.pdl != 0, p);
    };
    return rows <= 4 * num_ctas ? merge(latent_merge_kernel<4, 1>, 16) : merge(latent_merge_kernel<1, 4>, 1);
}

}  // namespace pd
