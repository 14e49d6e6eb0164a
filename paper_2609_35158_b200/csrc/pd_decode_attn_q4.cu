// Split-KV decode attention over 4-bit KV pages (format: pd_q4.cuh).
//
// With K_t = sk_t k_t + mk_t and V_t = sv_t v_t + mv_t (codes k, v in 0..15, one scale and minimum per token and group
// of 64 values) the two products fall apart into products of codes and rank-one terms:
//   S_t = sum_groups sk_t (q . k_t) + mk_t sum(q)          O = sum_t (p_t sv_t) v_t + sum_t p_t mv_t
// so the codes go to the tensor core as they are and scales and minima stay beside them.
//
// Same plan of ranges, partial format and merge kernel as the other split kernels. What differs:
//   * a (page, KV head) block is one piece of 18 D bytes: one untiled bulk copy per page. A tile is TP pages of one
//     segment on one barrier, issued by TP lanes of the worker that will read it. (One producer warp for the CTA, lane i
//     for worker i, was slower, 145 against 137 us then: copies of different lanes are issued one after the other, about
//     120 cycles each, and a stage waited 5200 cycles for its turn.);
//   * codes become fp16 without a conversion: a nibble in the low bits of a 16-bit half IS the fp16 subnormal
//     code * 2^-24, exactly, and mma.sync takes subnormals. For K, (w & 0x000f000f) is an operand register, and so are
//     (w & 0x00f000f0), 16 times larger, and the two of w >> 8; the factor 16 is taken out of Q beforehand. For V, bytes
//     are operands as well (two codes u + 16 v below 1024 are still a subnormal) and v's row of O is recovered at the
//     end as (O_byte - O_u) / 16, which saves the shift;
//   * Q is scaled per head by a power of two so that its largest value lies in [2^14, 2^15): fp16 then holds every
//     bf16 q down to 2^-24 of the largest exactly, whatever q's magnitude;
//   * mk_t sum(q) is one bf16 mma: mk is a bf16, sum(q) the sum of three. Its accumulator starts at -r, r being the
//     reference of the exponentials, so exp2 takes what the products leave;
//   * r is chosen per head so that the largest weight p_t sv_t of the segment lies in [2^2, 2^15]: the weights go to the
//     tensor core in fp16, of which weights below 2^-16 of the largest start to lose bits (under 2^-27 of the largest
//     for each). Taking the product and not p or sv alone keeps a token of huge scale and vanishing probability from
//     pushing the others out of range. The check in the loop is conservative (p and sv against caps whose product is
//     2^15) and the exact one runs only when it fires;
//   * with at most four query heads per KV head (PACK = 2) the eight columns of a product are four heads of one page and the same
//     four of the next: both pages' products go into one accumulator, each with zeros in the other's columns, and the
//     softmax between the products costs two pages what it cost one. O has both pages' sums apart and adds them at the end
//     (134 -> 130 us on 64 contexts of 2K-16K at 32/8 heads, 79 -> 73 us at head_dim 64; both under the power limit).
//   * the tensor core cuts what lies below fp32's last bit off its sums. Codes and weights are positive, so O fell behind with
//     every product of a long segment, and the minima, whose sums are rounded, did not: 65536 tokens in one segment were off
//     by 6 to 13 % of the output's rms (1024 pages: 1 to 3 %, 256: 0.3 to 0.6 %). So every 32 products of a lane's columns O is
//     folded into shared memory, rounded to nearest: 0.18 %, of which bf16 is 0.17. It costs 0.7 to 1.2 % on the long batches;
//     folds twice as far apart save nothing and leave 0.20 %.
// Sums, statistics, O and the rank-one terms are fp32. Weights p_t sv_t are rounded to fp16, 2^-11 of each at most, which adds
// 0.03 % of the output's rms to bf16's 0.17: adding 7.5 times the rounding to the minima's sum, which takes out the codes' mean,
// halved that and made the long batches 1 to 2.5 % slower (2 to 4 % under the power limit).
//
// Bound by its bytes (18 D per page and KV head) and nearly as much by its instructions, 193 per page at head_dim 128 and four
// heads, 227 at eight. Steps and what they gave on 64 contexts of 2K-16K at 32/8 heads, 713 MB (us): a page at a time with a scale
// reference for V beside the softmax maximum 193; two pages, one reference, minima by mma, bytes as V operands 147;
// independent chains of products, nothing cleared beforehand 129; four pages per tile 124; pages marked evict-first 119;
// folds and the check of the minima 120, which is 0.92 of the copy bandwidth (132 to 135, 0.82 to 0.84, when it runs for long
// and the power limit takes the SM clock to about 1.8 GHz). The skeleton without arithmetic takes 117. Pages fetched four at
// a time by a TMA gather instead of four bulk copies: 1 % slower at head_dim 128. Partial results merged inside this kernel
// instead of by the next one: 2 us slower.
#include "pd_decode_plan.cuh"
#include "pd_kernels.cuh"
#include "pd_ptx.cuh"
#include "pd_q4.cuh"

#include <cuda_fp16.h>

namespace pd {

namespace {

__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float pow2_int(int e) { return __int_as_float((e + 127) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ int exponent_of(float x) { return static_cast<int>((__float_as_uint(x) >> 23) & 255u) - 127; }
// Free to be scheduled among one another, unlike the volatile forms of pd_ptx.cuh: four independent chains of products are
// in flight here, and in program order each would wait for the one before.
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The first of a chain, without registers to clear beforehand.
__device__ __forceinline__ void mma_f16_from_zero(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// C (16x8) = A (16x8, bf16, in the low half of a 16x16) * B + {from, from}: rows g and g + 8 start at the same two values.
__device__ __forceinline__ void mma_bf16_from(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t b0, float from_a, float from_b) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%7,%8,%7,%8};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(b0), "f"(from_a), "f"(from_b));
}
// The same with 16 columns of A, the second eight those of the first again.
__device__ __forceinline__ void mma_bf16_from_twice(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1, float from_a, float from_b) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%4,%5}, {%6,%7}, {%8,%9,%8,%9};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(b0), "r"(b1), "f"(from_a), "f"(from_b));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}

__device__ __forceinline__ float4 ld_shared_f4(uint32_t at) {
    float4 f;
    asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "r"(at) : "memory");
    return f;
}
__device__ __forceinline__ float2 ld_shared_f2(uint32_t at) {
    float2 f;
    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(f.x), "=f"(f.y) : "r"(at) : "memory");
    return f;
}
__device__ __forceinline__ void st_shared_f4(uint32_t at, float x, float y, float z, float w) {
    asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(at), "f"(x), "f"(y), "f"(z), "f"(w) : "memory");
}
__device__ __forceinline__ void st_shared_f2(uint32_t at, float x, float y) {
    asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(at), "f"(x), "f"(y) : "memory");
}

// bulk_load with an L2 policy.
__device__ __forceinline__ void bulk_load_hint(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar, uint64_t pol) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar), "l"(pol)
                 : "memory");
}
constexpr int kQ4FoldProducts = 32;   // products (of 16 tokens) that an accumulator of O takes before it is folded
constexpr int kQ4FoldRefBytes = 256;  // a float2 per lane
constexpr uint32_t kNib0 = 0x000f000fu, kNib1 = 0x00f000f0u;

// PACK = 2 (groups of at most four heads): the eight columns of the products are four heads of one page and the same four of the
// next, see the top of the file.
template <int D, int WARPS, int STAGES, int TP, int PACK>
__global__ void __launch_bounds__(WARPS * 32, 1) decode_attn_split_q4_kernel(const AttnParams p) {
    static_assert(D == 64 || D == 128, "head_dim 64 or 128");
    constexpr int THREADS = WARPS * 32;
    constexpr int BLOCK = q4_block_bytes<D>();
    constexpr int STAGE = TP * BLOCK;
    constexpr int PIECES = D / 32;       // 16-byte pieces of a row
    constexpr int GROUPS = D / kQ4Group;
    constexpr int SETS = TP / PACK;      // pages, or pairs of pages, whose softmax is worked on together
    constexpr int COLS = 8 / PACK;       // heads per page among the columns
    constexpr int HEAD_LANES = COLS / 2;  // lanes of a quad that hold different heads
    constexpr int WINDOW = 32 / TP * TP;  // page ids held one per lane, whole tiles of them

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t ring0 = (raw + 127u) & ~127u;
    uint8_t *aligned = smem_raw + (ring0 - raw);
    // the folded part of a warp's O: a float4 per (piece, j) and lane, then per lane the reference it stands at
    constexpr int FOLD = PIECES * 2 * 512, FOLD_BYTES = FOLD + kQ4FoldRefBytes, FOLD_PAGES = kQ4FoldProducts * PACK;
    static_assert(FOLD_PAGES % TP == 0, "folds lie between tiles");
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + WARPS * (STAGES * STAGE + FOLD_BYTES));
    Plan *plan_s = reinterpret_cast<Plan *>(bars + WARPS * STAGES);
    int32_t *stage_range = reinterpret_cast<int32_t *>(plan_s + 1);
    int32_t *warp_sums = stage_range + WARPS * STAGES;
    int32_t *cum = warp_sums + 32;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    launch_dependents();
    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(smem_u32(bars + (warp * STAGES + s)), 1);
        mbar_init_fence();
    }
    grid_dependency_wait();
    scan_pages<THREADS>(p, cum, warp_sums);

    const int n_workers = gridDim.x * WARPS;
    if (tid == 0) make_plan(*plan_s, static_cast<long long>(p.Hkv) * cum[p.B], n_workers, p);
    __syncthreads();
    const Plan &pl = *plan_s;
    if (blockIdx.x == 0) {
        for (int i = tid; i <= p.B; i += THREADS) p.cum_pages[i] = cum[i];
        if (tid == 0) {
            p.plan[0] = static_cast<int32_t>(pl.total & 0xffffffffll);
            p.plan[1] = static_cast<int32_t>(pl.total >> 32);
            p.plan[2] = pl.n_levels;
            p.plan[3] = pl.n_ranges;
            p.plan[4] = n_workers;
        }
        if (tid <= pl.n_levels) {
            int32_t *rec = p.plan + kPlanHeaderWords + 4 * tid;
            rec[0] = static_cast<int32_t>(pl.lv[tid].start & 0xffffffffll);
            rec[1] = static_cast<int32_t>(pl.lv[tid].start >> 32);
            rec[2] = pl.lv[tid].size;
            rec[3] = pl.lv[tid].first;
        }
    }

    const int worker = warp * gridDim.x + blockIdx.x;  // a few ranges spread over all SMs (11.4 against 12.3 us for one sequence of 4096 tokens)
    const uint32_t ring = ring0 + warp * STAGES * STAGE;
    const uint32_t full = smem_u32(bars + warp * STAGES);
    int32_t *my_stage_range = stage_range + warp * STAGES;

    // Pages pass through L2 once; marked so, they leave the partial results, page ids and Q in it (124 -> 119 us on 64 contexts
    // of 2K-16K, 76 -> 72 us with eight heads per KV head).
    const uint64_t policy = l2_policy_evict_first();
    // ---- issuing side: walks STAGES tiles ahead of the reading side
    Cursor prod;
    prod.b = 0; prod.kvh = 0; prod.page = 0; prod.np = 1;
    int p_rid = worker, p_left = 0, p_stage = 0, inflight = 0;
    int ids = 0, ids_next = 0, window = 0;  // page ids [window, window + 32) of the open segment, one per lane, and those from window + WINDOW on
    bool p_first = true, p_done = false, have_next = false;
    int next_raw = 0;
    // With one range per worker at most nothing is ever claimed: no traffic on the counters then (all workers of a small batch
    // at once cost 1.5 us).
    const bool claims = pl.n_ranges > n_workers;
    const int G = p.G;
    const uint8_t *blocks = p.kv4;  // page 0 of the open KV head
    const uint32_t page_bytes = static_cast<uint32_t>(p.Hkv) * BLOCK;
    auto load_ids = [&](int page) {
        return page + lane < prod.np ? __ldg(p.page_table + static_cast<size_t>(prod.b) * p.MP + page + lane) : 0;
    };
    auto issue_next = [&]() {
        if (p_left == 0) {
            if (p_done) return;
            if (!p_first && claims) {
                if (!have_next && lane == 0) next_raw = atomicAdd(p.status + kSchedNext, 1);
                p_rid = n_workers + __shfl_sync(0xffffffffu, next_raw, 0);
                have_next = false;
            }
            if (p_rid >= pl.n_ranges || (!p_first && !claims)) {
                p_done = true;
                return;
            }
            p_first = false;
            long long start;
            range_bounds(pl, p_rid, start, p_left);
            prod = locate(cum, p.B, p.Hkv, start);
            blocks = p.kv4 + prod.kvh * BLOCK;
            window = prod.page;
            ids = load_ids(window);
            ids_next = load_ids(window + WINDOW);
        }
        const int n = min(TP, min(p_left, prod.np - prod.page));
        int pid = __shfl_sync(0xffffffffu, ids, (prod.page - window + lane) & 31);
        if (lane == 0) {
            my_stage_range[p_stage] = p_rid;
            mbar_arrive_expect_tx(full + p_stage * 8, n * BLOCK);
        }
        __syncwarp();
        if (lane < n) {
            if (static_cast<uint32_t>(pid) >= static_cast<uint32_t>(p.num_pages)) {
                latch_status(p.status, kDevBadPage, prod.b, pid);
                pid = 0;
            }
            bulk_load_hint(ring + p_stage * STAGE + lane * BLOCK, blocks + static_cast<uint64_t>(static_cast<uint32_t>(pid)) * page_bytes, BLOCK,
                      full + p_stage * 8, policy);
        }
        p_left -= n;
        prod.page += n;
        if (prod.page == prod.np) {
            prod.page -= 1;
            advance(prod, cum, p.B, p.Hkv);
            if (p_left > 0) {
                blocks = p.kv4 + prod.kvh * BLOCK;
                window = 0;
                ids = load_ids(0);
                ids_next = load_ids(WINDOW);
            }
        } else if (prod.page - window == WINDOW) {
            window += WINDOW;
            ids = ids_next;
            ids_next = load_ids(window + WINDOW);
        }
        if (claims && p_left <= kClaimAhead * TP && !have_next) {
            if (lane == 0) next_raw = atomicAdd(p.status + kSchedNext, 1);
            have_next = true;
        }
        if (++p_stage == STAGES) p_stage = 0;
        ++inflight;
    };
    for (int s = 0; s < STAGES; ++s) issue_next();

    // ---- reading side
    const int quad_row = lane >> 2, quad_t = lane & 3;
    // columns 2 t and 2 t + 1 of the accumulators: heads quad_col (a) and quad_col + 1 (b) of a set's page my_page
    const int quad_col = quad_t * 2 % COLS, my_page = quad_t * 2 / COLS;
    // column g of a B operand: head b_head of the set's page b_page
    const int b_head = quad_row % COLS, b_page = quad_row / COLS;
    // ldmatrix source rows: matrices 0 / 1 = slots 0-7 / 8-15 of a piece, 2 / 3 = the same of the next piece
    const int ld_slot = ((lane >> 3) & 1) * 8 + (lane & 7), ld_piece = lane >> 4;
    uint32_t ld_off[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) ld_off[g] = ld_slot * (D / 2) + q4_piece_pos<D>(2 * g + ld_piece, ld_slot) * 16;
    const uint32_t rec_off = my_page * BLOCK + 16 * D + quad_row * (D / 8);
    const uint32_t first_page = b_page == 0 ? 0xffffffffu : 0u;
    int stage = 0;
    uint32_t parity = 0;
    bool alive = true;

    while (alive && inflight > 0) {
        const int rid = my_stage_range[stage];
        long long start;
        int range_left;
        range_bounds(pl, rid, start, range_left);
        Cursor cur = locate(cum, p.B, p.Hkv, start);

        while (range_left > 0 && alive) {  // one segment: the range's pages of one (sequence, KV head)
            const int page0 = cur.page, pages = min(range_left, cur.np - page0);
            const int L = clamp_len(__ldg(p.ctx_lens + cur.b), p.MP);
            int rem = min(L - page0 * kPageSize, pages * kPageSize);  // tokens of the segment still to come

            // Q^T as the fp16 B operand for each page of a set (zero in the other page's columns), head b_head: register j of
            // piece c holds d = 32 c + 8 t + j and + 4 (odd j: / 16)
            uint32_t qb[PACK][PIECES][4];
            // B operand of the minima: sum(q) by group in three bf16 parts, for PACK = 1 part t in lane t. For two pages lanes
            // 0, 1 meet the first page's minima and 2, 3 the second's, with two rows each: parts 0 and 1, part 2 and 0.
            uint32_t qsum[PACK];
            float unit_a, unit_b;
            {
                const __nv_bfloat16 *qrow = p.q + (static_cast<size_t>(cur.b) * p.Hq + cur.kvh * G + b_head) * D;
                uint4 x[PIECES];
                float amax = 0.f, sum[GROUPS];
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) sum[g] = 0.f;
#pragma unroll
                for (int c = 0; c < PIECES; ++c) {
                    x[c] = make_uint4(0u, 0u, 0u, 0u);
                    if (b_head < G) x[c] = __ldg(reinterpret_cast<const uint4 *>(qrow + c * 32 + quad_t * 8));
                    const uint32_t w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float lo = bf16_lo(w[i]), hi = bf16_hi(w[i]);
                        amax = fmaxf(amax, fmaxf(fabsf(lo), fabsf(hi)));
                        sum[c * GROUPS / PIECES] += lo + hi;
                    }
                }
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], o);
                }
                const int e = max(-100, min(100, 14 - exponent_of(amax)));
                const float up = pow2_int(e), up16 = pow2_int(e - 4);
#pragma unroll
                for (int c = 0; c < PIECES; ++c) {
                    const uint32_t r[4] = {half2_bits(bf16_lo(x[c].x) * up, bf16_lo(x[c].z) * up), half2_bits(bf16_hi(x[c].x) * up16, bf16_hi(x[c].z) * up16),
                                           half2_bits(bf16_lo(x[c].y) * up, bf16_lo(x[c].w) * up), half2_bits(bf16_hi(x[c].y) * up16, bf16_hi(x[c].w) * up16)};
#pragma unroll
                    for (int k = 0; k < PACK; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) qb[k][c][i] = PACK == 1 || b_page == k ? r[i] : 0u;
                }
                // the scale of a head is wanted by the lanes whose accumulator columns it is
                unit_a = p.scale_log2 * pow2_int(24 - __shfl_sync(0xffffffffu, e, quad_col * 4));
                unit_b = p.scale_log2 * pow2_int(24 - __shfl_sync(0xffffffffu, e, quad_col * 4 + 4));
                float part[3][2] = {{0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    const float s = sum[g] * p.scale_log2;
                    part[0][g] = __bfloat162float(__float2bfloat16(s));
                    part[1][g] = __bfloat162float(__float2bfloat16(s - part[0][g]));
                    part[2][g] = s - part[0][g] - part[1][g];
                }
                const uint32_t parts[3] = {pack_bf16x2(part[0][0], part[0][1]), pack_bf16x2(part[1][0], part[1][1]), pack_bf16x2(part[2][0], part[2][1])};
                if (PACK == 1) {
                    qsum[0] = quad_t == 0 ? parts[0] : (quad_t == 1 ? parts[1] : (quad_t == 2 ? parts[2] : 0u));
                } else {
                    const bool own = quad_t >> 1 == b_page;
                    qsum[0] = own ? (quad_t & 1 ? parts[2] : parts[0]) : 0u;
                    qsum[PACK - 1] = own && !(quad_t & 1) ? parts[1] : 0u;
                }
            }
            // O^T, piece c, j: rows d = 32 c + 4 g + 2 j (registers 0, 1 for heads a, b); registers 2, 3: that plus 16 times d + 1
            float O[PIECES][2][4], Ma[GROUPS], Mb[GROUPS];
#pragma unroll
            for (int c = 0; c < PIECES; ++c)
#pragma unroll
                for (int j = 0; j < 2; ++j) { O[c][j][0] = 0.f; O[c][j][1] = 0.f; O[c][j][2] = 0.f; O[c][j][3] = 0.f; }
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) { Ma[g] = 0.f; Mb[g] = 0.f; }
            float l_a = 0.f, l_b = 0.f, nr_a = 0.f, nr_b = 0.f;  // nr = -r
            // O plus what earlier parts of the segment left in shared memory, brought to the present reference
            auto fold_at = [&]() { return ring0 + WARPS * STAGES * STAGE + warp * FOLD_BYTES + lane * 16; };
            auto join_folded = [&]() {
                const float2 nr = ld_shared_f2(fold_at() + FOLD - lane * 8);
                const float g_a = fast_exp2(nr_a - nr.x), g_b = fast_exp2(nr_b - nr.y);
#pragma unroll
                for (int c = 0; c < PIECES; ++c)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float4 f = ld_shared_f4(fold_at() + (c * 2 + j) * 512);
                        O[c][j][0] = fmaf(f.x, g_a, O[c][j][0]); O[c][j][1] = fmaf(f.y, g_b, O[c][j][1]);
                        O[c][j][2] = fmaf(f.z, g_a, O[c][j][2]); O[c][j][3] = fmaf(f.w, g_b, O[c][j][3]);
                    }
            };
            float cap_x = -INFINITY, cap_v = -1.f;  // nothing passes before the first tile has set them

            for (int pg = 0; pg < pages; pg += TP, rem -= TP * kPageSize) {
                if (!__all_sync(0xffffffffu, mbar_wait(full + stage * 8, parity))) { alive = false; break; }
                const uint32_t base = ring + stage * STAGE;
                const uint8_t *recs = aligned + (base - ring0) + rec_off;

                // records of slots g (i = 0) and g + 8 (i = 1) of this lane's page: {k_scale, k_min}, {v_scale, v_min} by group
                uint32_t rk[SETS][2][GROUPS], rv[SETS][2][GROUPS];
#pragma unroll
                for (int u = 0; u < SETS; ++u)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint8_t *at = recs + u * PACK * BLOCK + i * D;  // 8 slots of D / 8 bytes
                        if (GROUPS == 2) {
                            const uint4 w = *reinterpret_cast<const uint4 *>(at);
                            rk[u][i][0] = w.x; rv[u][i][0] = w.y; rk[u][i][GROUPS - 1] = w.z; rv[u][i][GROUPS - 1] = w.w;
                        } else {
                            const uint2 w = *reinterpret_cast<const uint2 *>(at);
                            rk[u][i][0] = w.x; rv[u][i][0] = w.y;
                        }
                    }
                const bool tail = rem < TP * kPageSize;
                // Codes of empty slots are harmless numbers, their records may be anything. What a slot's own columns make of them is
                // overwritten below, but the minima of one page of a pair also meet the other's columns, with a factor of 0.
                if (PACK > 1 && tail) {
#pragma unroll
                    for (int u = 0; u < SETS; ++u)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if ((u * PACK + my_page) * kPageSize + i * 8 + quad_row >= rem) {
#pragma unroll
                                for (int g = 0; g < GROUPS; ++g) rk[u][i][g] = 0u;
                            }
                }

                // x = S - r in log2 units, [slot g: heads a, b; slot g + 8: heads a, b]
                float x[SETS][4];
                {
                    uint32_t w[TP][GROUPS][4];  // (slots 0-7, 8-15) of piece 2 g, then of piece 2 g + 1
                    float acc[SETS][4], A[SETS][GROUPS][4];
#pragma unroll
                    for (int t = 0; t < TP; ++t)
#pragma unroll
                        for (int g = 0; g < GROUPS; ++g)
                            ldmatrix_x4(w[t][g][0], w[t][g][1], w[t][g][2], w[t][g][3], base + t * BLOCK + ld_off[g]);
#pragma unroll
                    for (int u = 0; u < SETS; ++u) {
                        const uint32_t k0 = GROUPS == 2 ? __byte_perm(rk[u][0][0], rk[u][0][GROUPS - 1], 0x7632) : rk[u][0][0] >> 16;
                        const uint32_t k1 = GROUPS == 2 ? __byte_perm(rk[u][1][0], rk[u][1][GROUPS - 1], 0x7632) : rk[u][1][0] >> 16;
                        if (PACK == 1) mma_bf16_from(acc[u], k0, k1, qsum[0], nr_a, nr_b);
                        else mma_bf16_from_twice(acc[u], k0, k1, qsum[0], qsum[PACK - 1], nr_a, nr_b);
                    }
#pragma unroll
                    for (int k = 0; k < PACK; ++k)
#pragma unroll
                        for (int h = 0; h < 4; ++h)  // piece 2 g + h / 2, its even (h = 0, 2) and odd bytes
#pragma unroll
                            for (int u = 0; u < SETS; ++u)
#pragma unroll
                                for (int g = 0; g < GROUPS; ++g) {
                                    const int t = u * PACK + k, c = 2 * g + (h >> 1);
                                    const uint32_t lo = w[t][g][h & 2] >> (8 * (h & 1)), hi = w[t][g][(h & 2) + 1] >> (8 * (h & 1));
                                    const uint32_t b0 = qb[k][c][2 * (h & 1)], b1 = qb[k][c][2 * (h & 1) + 1];
                                    if (h == 0 && k == 0) mma_f16_from_zero(A[u][g], lo & kNib0, hi & kNib0, lo & kNib1, hi & kNib1, b0, b1);
                                    else mma_f16(A[u][g], lo & kNib0, hi & kNib0, lo & kNib1, hi & kNib1, b0, b1);
                                }
#pragma unroll
                    for (int u = 0; u < SETS; ++u) {
                        float sum[4];
#pragma unroll
                        for (int g = 0; g < GROUPS; ++g) {
                            const float s0 = bf16_lo(rk[u][0][g]), s1 = bf16_lo(rk[u][1][g]);
                            sum[0] = g == 0 ? A[u][g][0] * s0 : fmaf(A[u][g][0], s0, sum[0]);
                            sum[1] = g == 0 ? A[u][g][1] * s0 : fmaf(A[u][g][1], s0, sum[1]);
                            sum[2] = g == 0 ? A[u][g][2] * s1 : fmaf(A[u][g][2], s1, sum[2]);
                            sum[3] = g == 0 ? A[u][g][3] * s1 : fmaf(A[u][g][3], s1, sum[3]);
                        }
                        x[u][0] = fmaf(sum[0], unit_a, acc[u][0]);
                        x[u][1] = fmaf(sum[1], unit_b, acc[u][1]);
                        x[u][2] = fmaf(sum[2], unit_a, acc[u][2]);
                        x[u][3] = fmaf(sum[3], unit_b, acc[u][3]);
                    }
                }
                if (tail) {
#pragma unroll
                    for (int u = 0; u < SETS; ++u)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if ((u * PACK + my_page) * kPageSize + i * 8 + quad_row >= rem) {
                                x[u][2 * i] = -INFINITY;
                                x[u][2 * i + 1] = -INFINITY;
#pragma unroll
                                for (int g = 0; g < GROUPS; ++g) rv[u][i][g] = 0u;
                            }
                }

                // The caps are about the largest V scale, vm, and a minimum counts with 2^-24 of itself, as below: behind a tile whose V
                // has tiny scales or none, p * minimum could leave fp32. (A record as a float is its minimum but for bits below bf16's;
                // the check costs 0.5 % on the long batches.)
                float xm_a = x[0][0], xm_b = x[0][1], vm = 0.f, mm = 0.f;
#pragma unroll
                for (int t = 0; t < SETS; ++t) {
                    xm_a = max3(xm_a, x[t][0], x[t][2]);
                    xm_b = max3(xm_b, x[t][1], x[t][3]);
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) {
                        vm = max3(vm, bf16_lo(rv[t][0][g]), bf16_lo(rv[t][1][g]));
                        mm = max3(mm, fabsf(__uint_as_float(rv[t][0][g])), fabsf(__uint_as_float(rv[t][1][g])));
                    }
                }
                vm = fmaxf(vm, mm * 5.9604645e-8f);
                if (__any_sync(0xffffffffu, xm_a > cap_x || xm_b > cap_x || vm > cap_v)) {
                    // largest weight of this tile by head: p * v_scale; a minimum 2^24 times the scale counts like the scale
                    // (the codes no longer matter then), and p itself stays below 2^100
                    float w_a = xm_a - 100.f, w_b = xm_b - 100.f;
#pragma unroll
                    for (int t = 0; t < SETS; ++t)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float v = 0.f;
#pragma unroll
                            for (int g = 0; g < GROUPS; ++g)
                                v = fmaxf(v, fmaxf(bf16_lo(rv[t][i][g]), fabsf(bf16_hi(rv[t][i][g])) * 5.9604645e-8f));
                            const float lv = __log2f(v);  // v = 0: -inf
                            w_a = fmaxf(w_a, x[t][2 * i] + lv);
                            w_b = fmaxf(w_b, x[t][2 * i + 1] + lv);
                        }
#pragma unroll
                    for (int o = HEAD_LANES; o < 32; o <<= 1) {  // the lanes that hold the same heads
                        w_a = fmaxf(w_a, __shfl_xor_sync(0xffffffffu, w_a, o));
                        w_b = fmaxf(w_b, __shfl_xor_sync(0xffffffffu, w_b, o));
                    }
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) vm = fmaxf(vm, __shfl_xor_sync(0xffffffffu, vm, o));
                    // the first tile puts its largest weight at 2^2; later ones only ever raise r
                    const bool fresh = cap_v < 0.f;
                    const float up_a = fresh ? w_a - 2.f : fmaxf(w_a - 2.f, 0.f), up_b = fresh ? w_b - 2.f : fmaxf(w_b - 2.f, 0.f);
                    // 2^-up in two factors: where a reference set by tiny scales meets large ones up passes 126, and the sums of
                    // weights, up to 2^100, still count
                    const float f_a = fresh ? 0.f : fast_exp2(-fminf(up_a, 100.f)), f_b = fresh ? 0.f : fast_exp2(-fminf(up_b, 100.f));
                    const float f2_a = fast_exp2(fminf(100.f - up_a, 0.f)), f2_b = fast_exp2(fminf(100.f - up_b, 0.f));
                    const float fo_a = f_a * f2_a, fo_b = f_b * f2_b;
                    nr_a -= up_a;
                    nr_b -= up_b;
                    l_a = l_a * f_a * f2_a;
                    l_b = l_b * f_b * f2_b;
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) { Ma[g] = Ma[g] * f_a * f2_a; Mb[g] = Mb[g] * f_b * f2_b; }
#pragma unroll
                    for (int c = 0; c < PIECES; ++c)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            O[c][j][0] *= fo_a; O[c][j][2] *= fo_a;
                            O[c][j][1] *= fo_b; O[c][j][3] *= fo_b;
                        }
#pragma unroll
                    for (int t = 0; t < SETS; ++t) {
                        x[t][0] -= up_a; x[t][2] -= up_a;
                        x[t][1] -= up_b; x[t][3] -= up_b;
                    }
                    // caps with cap_v 2^cap_x <= 2^15; v_scale may grow eightfold before the next look
                    const int ev = max(-110, min(100, exponent_of(fmaxf(vm, cap_v * 0.125f)) + 1));
                    cap_v = pow2_int(ev + 3);
                    cap_x = static_cast<float>(min(15 - (ev + 3), 100));
                }

                if (__builtin_expect(pg % FOLD_PAGES == 0 && pg > 0, 0)) {
                    if (pg > FOLD_PAGES) join_folded();
#pragma unroll
                    for (int c = 0; c < PIECES; ++c)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            st_shared_f4(fold_at() + (c * 2 + j) * 512, O[c][j][0], O[c][j][1], O[c][j][2], O[c][j][3]);
                            O[c][j][0] = 0.f; O[c][j][1] = 0.f; O[c][j][2] = 0.f; O[c][j][3] = 0.f;
                        }
                    st_shared_f2(fold_at() + FOLD - lane * 8, nr_a, nr_b);
                }

                // weights, their sums, and the fp16 B operands: P^T transposed from (slot x head) to (head x slot)
                uint32_t pb[SETS][GROUPS][2];
#pragma unroll
                for (int t = 0; t < SETS; ++t) {
                    const float p0 = fast_exp2(x[t][0]), p1 = fast_exp2(x[t][1]), p2 = fast_exp2(x[t][2]), p3 = fast_exp2(x[t][3]);
                    l_a += p0 + p2;
                    l_b += p1 + p3;
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) {
                        const float v0 = bf16_lo(rv[t][0][g]), v1 = bf16_lo(rv[t][1][g]), m0 = bf16_hi(rv[t][0][g]), m1 = bf16_hi(rv[t][1][g]);
                        Ma[g] = fmaf(p0, m0, fmaf(p2, m1, Ma[g]));
                        Mb[g] = fmaf(p1, m0, fmaf(p3, m1, Mb[g]));
                        pb[t][g][0] = transpose8x8(half2_bits(p0 * v0, p1 * v0));
                        pb[t][g][1] = transpose8x8(half2_bits(p2 * v1, p3 * v1));
                    }
                }
                // O^T += V^T P^T; with V's codes in registers the stage goes back to the copies
                uint32_t w[TP][GROUPS][4];
#pragma unroll
                for (int t = 0; t < TP; ++t)
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g)
                        ldmatrix_x4_trans(w[t][g][0], w[t][g][1], w[t][g][2], w[t][g][3], base + t * BLOCK + 8 * D + ld_off[g]);
                __syncwarp();
                --inflight;
                issue_next();
#pragma unroll
                for (int u = 0; u < SETS; ++u)
#pragma unroll
                    for (int k = 0; k < PACK; ++k) {
                        // of a pair's weights, those of page k: the other page's columns must add nothing
                        uint32_t pk[GROUPS][2];
#pragma unroll
                        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                            for (int i = 0; i < 2; ++i) pk[g][i] = PACK == 1 ? pb[u][g][i] : pb[u][g][i] & (k == 0 ? first_page : ~first_page);
#pragma unroll
                        for (int h = 0; h < 4; ++h)
#pragma unroll
                            for (int g = 0; g < GROUPS; ++g) {
                                const int t = u * PACK + k;
                                const uint32_t lo = w[t][g][h & 2], hi = w[t][g][(h & 2) + 1];  // slots 2t, 2t+1 and 2t+8, 2t+9; four consecutive d each
                                const uint32_t pick = (h & 1) ? 0x4341u : 0x4240u;              // d + 2, d + 3 or d, d + 1
                                const uint32_t lb = __byte_perm(lo, 0u, pick), hb = __byte_perm(hi, 0u, pick);
                                mma_f16(O[2 * g + (h >> 1)][h & 1], lb & kNib0, lb, hb & kNib0, hb, pk[g][0], pk[g][1]);
                            }
                    }
                if (++stage == STAGES) { stage = 0; parity ^= 1u; }
            }
            if (!alive) break;
            if (pages > FOLD_PAGES) join_folded();

            if (PACK > 1) {  // a pair's pages have summed the same heads in different lanes
#pragma unroll
                for (int c = 0; c < PIECES; ++c)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) O[c][j][i] += __shfl_xor_sync(0xffffffffu, O[c][j][i], HEAD_LANES);
            }
#pragma unroll
            for (int o = HEAD_LANES; o < 32; o <<= 1) {
                l_a += __shfl_xor_sync(0xffffffffu, l_a, o);
                l_b += __shfl_xor_sync(0xffffffffu, l_b, o);
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    Ma[g] += __shfl_xor_sync(0xffffffffu, Ma[g], o);
                    Mb[g] += __shfl_xor_sync(0xffffffffu, Mb[g], o);
                }
            }
            const size_t row0 = static_cast<size_t>(cur.b) * p.Hq + cur.kvh * G + quad_col;
            const bool has_a = my_page == 0 && quad_col < G, has_b = my_page == 0 && quad_col + 1 < G;
            const bool whole = page0 == 0 && pages == cur.np;
            // Final rows are divided by the sum of weights. Partials carry (reference, sum) with the sum in [1, 2), so that the
            // merge compares references that mean the same thing whatever this segment's scales were.
            const int el_a = max(-126, min(126, exponent_of(l_a))), el_b = max(-126, min(126, exponent_of(l_b)));
            const float da = whole ? 1.f / l_a : pow2_int(-el_a), db = whole ? 1.f / l_b : pow2_int(-el_b);
            // codes came in as code * 2^-24; registers 2, 3 hold the even row plus 16 times the odd one
            float ya[PIECES][4], yb[PIECES][4];
#pragma unroll
            for (int c = 0; c < PIECES; ++c) {
                const float ma = Ma[c * GROUPS / PIECES], mb = Mb[c * GROUPS / PIECES];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    ya[c][2 * j] = (O[c][j][0] * 16777216.f + ma) * da;
                    ya[c][2 * j + 1] = ((O[c][j][2] - O[c][j][0]) * 1048576.f + ma) * da;
                    yb[c][2 * j] = (O[c][j][1] * 16777216.f + mb) * db;
                    yb[c][2 * j + 1] = ((O[c][j][3] - O[c][j][1]) * 1048576.f + mb) * db;
                }
            }
            if (whole) {
                __nv_bfloat16 *oa = p.out + row0 * D + 4 * quad_row, *ob = oa + D;
#pragma unroll
                for (int c = 0; c < PIECES; ++c) {
                    if (has_a)
                        *reinterpret_cast<uint2 *>(oa + 32 * c) = make_uint2(pack_bf16x2(ya[c][0], ya[c][1]), pack_bf16x2(ya[c][2], ya[c][3]));
                    if (has_b)
                        *reinterpret_cast<uint2 *>(ob + 32 * c) = make_uint2(pack_bf16x2(yb[c][0], yb[c][1]), pack_bf16x2(yb[c][2], yb[c][3]));
                }
                if (p.lse != nullptr && quad_row == 0) {
                    if (has_a) p.lse[row0] = (log2f(l_a) - nr_a) * kLn2;
                    if (has_b) p.lse[row0 + 1] = (log2f(l_b) - nr_b) * kLn2;
                }
            } else {
                const size_t slot = static_cast<size_t>(rid) + static_cast<size_t>(cur.b) * p.Hkv + cur.kvh;
                float *oa = p.part_o + (slot * G + quad_col) * D + 4 * quad_row, *ob = oa + D;
#pragma unroll
                for (int c = 0; c < PIECES; ++c) {
                    if (has_a) *reinterpret_cast<float4 *>(oa + 32 * c) = make_float4(ya[c][0], ya[c][1], ya[c][2], ya[c][3]);
                    if (has_b) *reinterpret_cast<float4 *>(ob + 32 * c) = make_float4(yb[c][0], yb[c][1], yb[c][2], yb[c][3]);
                }
                if (quad_row == 0) {
                    if (has_a) p.part_ml[slot * G + quad_col] = make_float2(el_a - nr_a, l_a * da);
                    if (has_b) p.part_ml[slot * G + quad_col + 1] = make_float2(el_b - nr_b, l_b * db);
                }
            }
            range_left -= pages;
            cur.page += pages - 1;
            advance(cur, cum, p.B, p.Hkv);
        }
    }
    if (!alive) {  // copies may still be on their way: shared memory is not given back without another bounded wait for them
        for (; inflight > 0; --inflight) {
            mbar_wait(full + stage * 8, parity);
            if (++stage == STAGES) { stage = 0; parity ^= 1u; }
        }
    }
    if (lane == 0) {
        if (!alive) latch_status(p.status, kDevTimeout, -1, worker);
        if (claims && atomicAdd(p.status + kSchedDone, 1) == n_workers - 1) {  // the last worker re-arms the claim counter
            p.status[kSchedNext] = 0;
            p.status[kSchedDone] = 0;
        }
    }
}

template <int D, int WARPS, int STAGES, int TP>
constexpr size_t q4_smem_bytes() {
    return static_cast<size_t>(WARPS) * (STAGES * TP * q4_block_bytes<D>() + D / 32 * 2 * 512 + kQ4FoldRefBytes) + 128 +
           WARPS * STAGES * 8 + sizeof(Plan) + WARPS * STAGES * 4 + 32 * 4 + (kMaxBatch + 1) * 4;
}

// Worker warps x stages x pages per tile. A tile costs about 140 instructions beside its pages, so large tiles pay; the
// warps have to be the same number on each of the four schedulers, because they get equal ranges (14 and 15 lose to 12).
// One stage is enough: with its V codes in registers a worker hands the stage back before its last products, and the
// other workers' copies keep the memory busy. Measured before O was folded, 64 contexts of 2K-16K at 32/8 heads, head_dim 128 (us):
// 12 x 1 x 4 119.0, 12 x 1 x 5 119.0 (but 13 % slower on short contexts), 16 x 1 x 3 120.3, 12 x 2 x 3 121.9,
// 12 x 1 x 3 124.0, 8 x 2 x 4 126.2. head_dim 64, same lengths / 37 sequences of 0-5000 tokens at 16/2 heads:
// 16 x 1 x 4 73.2 / 19.2, 16 x 1 x 6 69.3 / 20.1, 16 x 2 x 4 73.2 / 19.7, 12 x 2 x 4 74.6 / 19.3.
constexpr int kQ4Warps = 12, kQ4Warps64 = 16, kQ4Stages = 1, kQ4TilePages = 4;
template <int D, int WARPS, typename F>
cudaError_t with_q4_pack(int group, F &&f) {
    constexpr size_t bytes = q4_smem_bytes<D, WARPS, kQ4Stages, kQ4TilePages>();
    return group <= 4 ? f(decode_attn_split_q4_kernel<D, WARPS, kQ4Stages, kQ4TilePages, 2>, bytes, WARPS)
                      : f(decode_attn_split_q4_kernel<D, WARPS, kQ4Stages, kQ4TilePages, 1>, bytes, WARPS);
}
template <typename F>
cudaError_t with_q4_kernel(int head_dim, int group, F &&f) {
    return head_dim == 64 ? with_q4_pack<64, kQ4Warps64>(group, f) : with_q4_pack<128, kQ4Warps>(group, f);
}

}  // namespace

cudaError_t prepare_decode_attn_q4(int head_dim, int group) {
    auto set = [](auto *k, size_t bytes, int) {
        return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
    };
    return with_q4_kernel(head_dim, group, set);
}

cudaError_t launch_decode_attn_q4(int head_dim, const AttnParams &p, int num_ctas, cudaStream_t stream) {
    auto go = [&](auto *k, size_t bytes, int warps) {
        return launch_pdl(k, dim3(num_ctas), dim3(warps * 32), bytes, stream, p.pdl != 0, p);
    };
    return with_q4_kernel(head_dim, p.G, go);
}

}  // namespace pd
