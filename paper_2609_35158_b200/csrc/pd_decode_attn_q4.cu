// Split-KV decode attention over 4-bit KV pages (format: pd_q4.cuh).
//
// With K_t = sk_t k_t + mk_t and V_t = sv_t v_t + mv_t (codes k, v in 0..15, one scale and minimum per token and group
// of 64 values) the two products fall apart into products of codes and rank-one terms:
//   S_t = sum_groups sk_t (q . k_t) + mk_t sum(q)          O = sum_t (p_t sv_t) v_t + sum_t p_t mv_t
// so the codes go to the tensor core as they are and scales and minima stay in fp32 registers.
//
// Same plan of ranges, worker warps, partial format and merge kernel as the other split kernels. What differs:
//   * a (page, KV head) block is one piece of 18 D bytes: one untiled bulk copy on one barrier per stage;
//   * codes become fp16 without a conversion: a nibble in the low bits of a 16-bit half IS the fp16 subnormal
//     code * 2^-24, exactly, and mma.sync takes subnormals. So (w & 0x000f000f) is an operand register, and so are
//     (w & 0x00f000f0), 16 times larger, and the two of w >> 8: five integer instructions for eight values. The factor
//     16 is taken out of Q beforehand for K, and out of the output rows at the end for V;
//   * Q is scaled per head by a power of two so that its largest value lies in [2^14, 2^15): fp16 then holds every
//     bf16 q down to 2^-24 of the largest exactly, whatever q's magnitude;
//   * P * sv goes to the tensor core in fp16 relative to a per-head power of two `f` that keeps the largest weight of
//     the segment between 2^2 and 2^15: weights below 2^-16 of the largest start to lose bits, which is under 2^-27 of
//     the largest for each. Tracking the product and not sv alone keeps a token of huge scale and vanishing
//     probability from pushing the others out of range.
// Sums, statistics, O and the rank-one terms are fp32.
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

constexpr uint32_t kNib0 = 0x000f000fu, kNib1 = 0x00f000f0u;
constexpr float kWeightMax = 32768.f;

template <int D, int WARPS, int STAGES>
__global__ void __launch_bounds__(WARPS * 32, 1) decode_attn_split_q4_kernel(const AttnParams p) {
    static_assert(D == 64 || D == 128, "head_dim 64 or 128");
    constexpr int THREADS = WARPS * 32;
    constexpr int BLOCK = q4_block_bytes<D>();
    constexpr int PIECES = D / 32;       // 16-byte pieces of a row
    constexpr int GROUPS = D / kQ4Group;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t ring0 = (raw + 127u) & ~127u;
    uint8_t *aligned = smem_raw + (ring0 - raw);
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + WARPS * STAGES * BLOCK);
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

    const int worker = blockIdx.x * WARPS + warp;
    const uint32_t ring = ring0 + warp * STAGES * BLOCK;
    const uint32_t bar0 = smem_u32(bars + warp * STAGES);
    int32_t *my_stage_range = stage_range + warp * STAGES;
    const int quad_row = lane >> 2, quad_t = lane & 3, quad_col = quad_t * 2;
    const int G = p.G;
    // ldmatrix source rows: matrices 0 / 1 = slots 0-7 / 8-15 of a piece, 2 / 3 = the same of the next piece
    const int mat = lane >> 3, ld_slot = (mat & 1) * 8 + (lane & 7), ld_piece = mat >> 1;
    const uint32_t ld_row = ld_slot * (D / 2);

    PageIdCache pt;
    pt.b = -1; pt.blk = -1; pt.val = -1; pt.nval = -1;
    Cursor prod;
    prod.b = 0; prod.kvh = 0; prod.page = 0; prod.np = 1;
    int p_rid = -1, p_left = 0;
    bool p_first = true, p_done = false, have_next = false;
    int next_raw = 0;
    uint32_t p_stage = 0;
    int inflight = 0;

    auto issue_next = [&]() -> bool {
        if (p_left == 0) {
            if (p_done) return false;
            int rid;
            if (p_first) {
                rid = worker;
                p_first = false;
            } else {
                if (!have_next && lane == 0) next_raw = atomicAdd(p.status + kSchedNext, 1);
                rid = n_workers + __shfl_sync(0xffffffffu, next_raw, 0);
                have_next = false;
            }
            if (rid >= pl.n_ranges) {
                p_done = true;
                return false;
            }
            long long start;
            range_bounds(pl, rid, start, p_left);
            prod = locate(cum, p.B, p.Hkv, start);
            p_rid = rid;
        }
        int pid = page_id(pt, p, prod.b, prod.page, lane);
        if (pid < 0 || pid >= p.num_pages) {
            if (lane == 0) latch_status(p.status, kDevBadPage, prod.b, pid);
            pid = 0;
        }
        if (lane == 0) {
            my_stage_range[p_stage] = p_rid;
            const uint32_t bar = bar0 + p_stage * 8;
            mbar_arrive_expect_tx(bar, BLOCK);
            bulk_load(ring + p_stage * BLOCK, p.kv4 + (static_cast<size_t>(pid) * p.Hkv + prod.kvh) * BLOCK, BLOCK, bar);
        }
        advance(prod, cum, p.B, p.Hkv);
        --p_left;
        if (p_left <= kClaimAhead && !have_next && !p_first) {
            if (lane == 0) next_raw = atomicAdd(p.status + kSchedNext, 1);
            have_next = true;
        }
        if (++p_stage == STAGES) p_stage = 0;
        ++inflight;
        __syncwarp();
        return true;
    };

    while (inflight < STAGES && issue_next()) {}

    Cursor cons;
    cons.b = 0; cons.kvh = 0; cons.page = 0; cons.np = 1;
    int c_rid = -1, c_left = 0;
    uint32_t stage = 0, parity = 0;
    bool alive = true, seg_open = false;
    int seg_page0 = 0, L = 0;
    // Q^T as the fp16 B operand, head quad_row: register j of piece c holds d = 32 c + 8 t + j and + 4 (odd j: / 16)
    uint32_t qb[PIECES][4];
    // heads quad_col and quad_col + 1 (a, b): unit of the code products in log2 logits, and scale_log2 * sum(q) by group
    float unit_a = 0.f, unit_b = 0.f, qs_a[GROUPS], qs_b[GROUPS];
    // O^T, piece c, j: rows d = 32 c + 4 g + 2 j (registers 0, 1 for heads a, b) and + 1 (registers 2, 3, 16 times larger)
    float O[PIECES][2][4];
    float Ma[GROUPS], Mb[GROUPS];  // this lane's slots' share of sum p * v_min
    float m_a = -INFINITY, m_b = -INFINITY, l_a = 0.f, l_b = 0.f;
    float f_a = 1.f, f_b = 1.f;    // weights go to the tensor core as p * v_scale * f

    while (inflight > 0) {
        if (c_left == 0) {
            c_rid = my_stage_range[stage];
            long long start;
            range_bounds(pl, c_rid, start, c_left);
            cons = locate(cum, p.B, p.Hkv, start);
        }
        if (!seg_open) {
            seg_open = true;
            seg_page0 = cons.page;
            L = clamp_len(__ldg(p.ctx_lens + cons.b), p.MP);
            const __nv_bfloat16 *qrow = p.q + (static_cast<size_t>(cons.b) * p.Hq + cons.kvh * G + quad_row) * D;
            uint4 x[PIECES];
            float amax = 0.f, sum[GROUPS];
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) sum[g] = 0.f;
#pragma unroll
            for (int c = 0; c < PIECES; ++c) {
                x[c] = make_uint4(0u, 0u, 0u, 0u);
                if (quad_row < G) x[c] = __ldg(reinterpret_cast<const uint4 *>(qrow + c * 32 + quad_t * 8));
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
                qb[c][0] = half2_bits(bf16_lo(x[c].x) * up, bf16_lo(x[c].z) * up);
                qb[c][1] = half2_bits(bf16_hi(x[c].x) * up16, bf16_hi(x[c].z) * up16);
                qb[c][2] = half2_bits(bf16_lo(x[c].y) * up, bf16_lo(x[c].w) * up);
                qb[c][3] = half2_bits(bf16_hi(x[c].y) * up16, bf16_hi(x[c].w) * up16);
            }
            // what belongs to a head is wanted by the lanes whose accumulator columns it is
            const int e_a = __shfl_sync(0xffffffffu, e, quad_col * 4), e_b = __shfl_sync(0xffffffffu, e, quad_col * 4 + 4);
            unit_a = p.scale_log2 * pow2_int(24 - e_a);
            unit_b = p.scale_log2 * pow2_int(24 - e_b);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                qs_a[g] = p.scale_log2 * __shfl_sync(0xffffffffu, sum[g], quad_col * 4);
                qs_b[g] = p.scale_log2 * __shfl_sync(0xffffffffu, sum[g], quad_col * 4 + 4);
                Ma[g] = 0.f;
                Mb[g] = 0.f;
            }
#pragma unroll
            for (int c = 0; c < PIECES; ++c)
#pragma unroll
                for (int j = 0; j < 2; ++j) { O[c][j][0] = 0.f; O[c][j][1] = 0.f; O[c][j][2] = 0.f; O[c][j][3] = 0.f; }
            m_a = -INFINITY; m_b = -INFINITY;
            l_a = 0.f; l_b = 0.f;
            f_a = 1.f; f_b = 1.f;
        }

        const uint32_t kbase = ring + stage * BLOCK, vbase = kbase + 8 * D;
        const int valid = L - cons.page * kPageSize;
        if (!__all_sync(0xffffffffu, mbar_wait(bar0 + stage * 8, parity))) { alive = false; break; }

        // records of slots g and g + 8: per group {k_scale, k_min}, {v_scale, v_min}
        float ks0[GROUPS], km0[GROUPS], vs0[GROUPS], vm0[GROUPS], ks1[GROUPS], km1[GROUPS], vs1[GROUPS], vm1[GROUPS];
        const uint8_t *recs = aligned + (kbase - ring0) + 16 * D;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const uint2 r0 = *reinterpret_cast<const uint2 *>(recs + quad_row * (D / 8) + g * 8);
            const uint2 r1 = *reinterpret_cast<const uint2 *>(recs + (quad_row + 8) * (D / 8) + g * 8);
            ks0[g] = bf16_lo(r0.x); km0[g] = bf16_hi(r0.x); vs0[g] = bf16_lo(r0.y); vm0[g] = bf16_hi(r0.y);
            ks1[g] = bf16_lo(r1.x); km1[g] = bf16_hi(r1.x); vs1[g] = bf16_lo(r1.y); vm1[g] = bf16_hi(r1.y);
        }

        // code products K Q^T by group; the accumulators of a group hold the sum over its 64 values
        float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f, r0s = 0.f, r1s = 0.f, r2s = 0.f, r3s = 0.f;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            uint32_t w[4];  // (slots 0-7, 8-15) of piece 2 g, then of piece 2 g + 1
            ldmatrix_x4(w[0], w[1], w[2], w[3], kbase + ld_row + q4_piece_pos<D>(2 * g + ld_piece, ld_slot) * 16);
            float A[4] = {0.f, 0.f, 0.f, 0.f}, B[4] = {0.f, 0.f, 0.f, 0.f};
            mma_f16_16816(A, w[0] & kNib0, w[1] & kNib0, w[0] & kNib1, w[1] & kNib1, qb[2 * g][0], qb[2 * g][1]);
            mma_f16_16816(B, w[2] & kNib0, w[3] & kNib0, w[2] & kNib1, w[3] & kNib1, qb[2 * g + 1][0], qb[2 * g + 1][1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] >>= 8;
            mma_f16_16816(A, w[0] & kNib0, w[1] & kNib0, w[0] & kNib1, w[1] & kNib1, qb[2 * g][2], qb[2 * g][3]);
            mma_f16_16816(B, w[2] & kNib0, w[3] & kNib0, w[2] & kNib1, w[3] & kNib1, qb[2 * g + 1][2], qb[2 * g + 1][3]);
            s0 += (A[0] + B[0]) * ks0[g]; s1 += (A[1] + B[1]) * ks0[g];
            s2 += (A[2] + B[2]) * ks1[g]; s3 += (A[3] + B[3]) * ks1[g];
            r0s += km0[g] * qs_a[g]; r1s += km0[g] * qs_b[g];
            r2s += km1[g] * qs_a[g]; r3s += km1[g] * qs_b[g];
        }
        s0 = s0 * unit_a + r0s; s1 = s1 * unit_b + r1s;
        s2 = s2 * unit_a + r2s; s3 = s3 * unit_b + r3s;
        if (valid < kPageSize) {  // codes of empty slots are harmless numbers, their records may be anything
            if (quad_row >= valid) {
                s0 = -INFINITY; s1 = -INFINITY;
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) { vs0[g] = 0.f; vm0[g] = 0.f; }
            }
            if (quad_row + 8 >= valid) {
                s2 = -INFINITY; s3 = -INFINITY;
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) { vs1[g] = 0.f; vm1[g] = 0.f; }
            }
        }

        float mx_a = fmaxf(s0, s2), mx_b = fmaxf(s1, s3);
        float alpha_a = 1.f, alpha_b = 1.f;
        const bool raise = __any_sync(0xffffffffu, mx_a > m_a + kRescaleSlack || mx_b > m_b + kRescaleSlack);
        if (raise) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                mx_a = fmaxf(mx_a, __shfl_xor_sync(0xffffffffu, mx_a, o));
                mx_b = fmaxf(mx_b, __shfl_xor_sync(0xffffffffu, mx_b, o));
            }
            const float new_a = fmaxf(m_a, mx_a), new_b = fmaxf(m_b, mx_b);
            alpha_a = fast_exp2(m_a - new_a);
            alpha_b = fast_exp2(m_b - new_b);
            l_a *= alpha_a;
            l_b *= alpha_b;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) { Ma[g] *= alpha_a; Mb[g] *= alpha_b; }
            m_a = new_a;
            m_b = new_b;
        }
        const float p0 = fast_exp2(s0 - m_a), p1 = fast_exp2(s1 - m_b);
        const float p2 = fast_exp2(s2 - m_a), p3 = fast_exp2(s3 - m_b);
        l_a += p0 + p2;
        l_b += p1 + p3;
        float w_a = 0.f, w_b = 0.f;  // largest weight of this lane's slots
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            Ma[g] += p0 * vm0[g] + p2 * vm1[g];
            Mb[g] += p1 * vm0[g] + p3 * vm1[g];
            w_a = fmaxf(w_a, fmaxf(p0 * vs0[g], p2 * vs1[g]));
            w_b = fmaxf(w_b, fmaxf(p1 * vs0[g], p3 * vs1[g]));
        }
        if (__any_sync(0xffffffffu, raise || w_a * f_a > kWeightMax || w_b * f_b > kWeightMax)) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                w_a = fmaxf(w_a, __shfl_xor_sync(0xffffffffu, w_a, o));
                w_b = fmaxf(w_b, __shfl_xor_sync(0xffffffffu, w_b, o));
            }
            // this page's largest weight to [2^2, 2^3), unless older weights, shrunk by alpha, are larger: O never grows
            auto retarget = [](float w, float alpha, float &f, float &scale_o) {
                float nf = pow2_int(max(-100, min(100, 2 - exponent_of(w))));
                const float keep = f / alpha;  // alpha = 0 (first page, or nothing left of the past): +inf
                int ke = exponent_of(keep);
                if (ke < 100 && pow2_int(max(ke, -126)) < nf) nf = pow2_int(max(ke, -100));
                scale_o = alpha * (nf / f);
                if (!(alpha > 0.f)) scale_o = 0.f;
                f = nf;
            };
            float so_a, so_b;
            retarget(w_a, alpha_a, f_a, so_a);
            retarget(w_b, alpha_b, f_b, so_b);
#pragma unroll
            for (int c = 0; c < PIECES; ++c)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    O[c][j][0] *= so_a; O[c][j][2] *= so_a;
                    O[c][j][1] *= so_b; O[c][j][3] *= so_b;
                }
        }

        // O^T += V^T (P v_scale f)^T; the weights differ by group
        const float p0f = p0 * f_a, p1f = p1 * f_b, p2f = p2 * f_a, p3f = p3 * f_b;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const uint32_t pb0 = movmatrix_trans(half2_bits(p0f * vs0[g], p1f * vs0[g]));
            const uint32_t pb1 = movmatrix_trans(half2_bits(p2f * vs1[g], p3f * vs1[g]));
            uint32_t w[4];
            ldmatrix_x4_trans(w[0], w[1], w[2], w[3], vbase + ld_row + q4_piece_pos<D>(2 * g + ld_piece, ld_slot) * 16);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t x = w[2 * h], y = w[2 * h + 1];  // slots 2t, 2t+1 and 2t+8, 2t+9; four consecutive d each
                mma_f16_16816(O[2 * g + h][0], x & kNib0, x & kNib1, y & kNib0, y & kNib1, pb0, pb1);
                x >>= 8;
                y >>= 8;
                mma_f16_16816(O[2 * g + h][1], x & kNib0, x & kNib1, y & kNib0, y & kNib1, pb0, pb1);
            }
        }
        __syncwarp();
        --inflight;
        issue_next();
        if (++stage == STAGES) { stage = 0; parity ^= 1u; }

        --c_left;
        const bool pair_end = cons.page + 1 == cons.np;
        if (c_left == 0 || pair_end) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                l_a += __shfl_xor_sync(0xffffffffu, l_a, o);
                l_b += __shfl_xor_sync(0xffffffffu, l_b, o);
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    Ma[g] += __shfl_xor_sync(0xffffffffu, Ma[g], o);
                    Mb[g] += __shfl_xor_sync(0xffffffffu, Mb[g], o);
                }
            }
            const size_t row0 = static_cast<size_t>(cons.b) * p.Hq + cons.kvh * G + quad_col;
            const bool has_a = quad_col < G, has_b = quad_col + 1 < G;
            // codes came in as code * 2^-24 (and 16 times that in registers 2, 3)
            const float ka = 16777216.f / f_a, kb = 16777216.f / f_b;
            if (seg_page0 == 0 && pair_end) {
                const float inv_a = 1.f / l_a, inv_b = 1.f / l_b;
                __nv_bfloat16 *oa = p.out + row0 * D + 4 * quad_row, *ob = oa + D;
#pragma unroll
                for (int c = 0; c < PIECES; ++c) {
                    const float ma = Ma[c * GROUPS / PIECES], mb = Mb[c * GROUPS / PIECES];
                    const float *x = O[c][0], *y = O[c][1];
                    if (has_a)
                        *reinterpret_cast<uint2 *>(oa + 32 * c) =
                            make_uint2(pack_bf16x2((x[0] * ka + ma) * inv_a, (x[2] * (ka * 0.0625f) + ma) * inv_a),
                                       pack_bf16x2((y[0] * ka + ma) * inv_a, (y[2] * (ka * 0.0625f) + ma) * inv_a));
                    if (has_b)
                        *reinterpret_cast<uint2 *>(ob + 32 * c) =
                            make_uint2(pack_bf16x2((x[1] * kb + mb) * inv_b, (x[3] * (kb * 0.0625f) + mb) * inv_b),
                                       pack_bf16x2((y[1] * kb + mb) * inv_b, (y[3] * (kb * 0.0625f) + mb) * inv_b));
                }
                if (p.lse != nullptr && quad_row == 0) {
                    if (has_a) p.lse[row0] = (m_a + log2f(l_a)) * kLn2;
                    if (has_b) p.lse[row0 + 1] = (m_b + log2f(l_b)) * kLn2;
                }
            } else {
                const size_t slot = static_cast<size_t>(c_rid) + static_cast<size_t>(cons.b) * p.Hkv + cons.kvh;
                float *oa = p.part_o + (slot * G + quad_col) * D + 4 * quad_row, *ob = oa + D;
#pragma unroll
                for (int c = 0; c < PIECES; ++c) {
                    const float ma = Ma[c * GROUPS / PIECES], mb = Mb[c * GROUPS / PIECES];
                    const float *x = O[c][0], *y = O[c][1];
                    if (has_a)
                        *reinterpret_cast<float4 *>(oa + 32 * c) = make_float4(x[0] * ka + ma, x[2] * (ka * 0.0625f) + ma,
                                                                              y[0] * ka + ma, y[2] * (ka * 0.0625f) + ma);
                    if (has_b)
                        *reinterpret_cast<float4 *>(ob + 32 * c) = make_float4(x[1] * kb + mb, x[3] * (kb * 0.0625f) + mb,
                                                                              y[1] * kb + mb, y[3] * (kb * 0.0625f) + mb);
                }
                if (quad_row == 0) {
                    if (has_a) p.part_ml[slot * G + quad_col] = make_float2(m_a, l_a);
                    if (has_b) p.part_ml[slot * G + quad_col + 1] = make_float2(m_b, l_b);
                }
            }
            seg_open = false;
        }
        advance(cons, cum, p.B, p.Hkv);
    }

    if (lane == 0) {
        if (!alive) latch_status(p.status, kDevTimeout, -1, worker);
        if (atomicAdd(p.status + kSchedDone, 1) == n_workers - 1) {  // the last worker re-arms the claim counter
            p.status[kSchedNext] = 0;
            p.status[kSchedDone] = 0;
        }
    }
}

template <int D, int WARPS, int STAGES>
constexpr size_t q4_smem_bytes() {
    return static_cast<size_t>(WARPS) * STAGES * q4_block_bytes<D>() + 128 + WARPS * STAGES * 8 + sizeof(Plan) +
           WARPS * STAGES * 4 + 32 * 4 + (kMaxBatch + 1) * 4;
}

template <typename F>
cudaError_t with_q4_kernel(int head_dim, F &&f) {
    if (head_dim == 64) return f(decode_attn_split_q4_kernel<64, 16, 10>, q4_smem_bytes<64, 16, 10>(), 16);
    return f(decode_attn_split_q4_kernel<128, 16, 5>, q4_smem_bytes<128, 16, 5>(), 16);
}

}  // namespace

cudaError_t prepare_decode_attn_q4(int head_dim) {
    auto set = [](auto *k, size_t bytes, int) {
        return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
    };
    return with_q4_kernel(head_dim, set);
}

cudaError_t launch_decode_attn_q4(int head_dim, const AttnParams &p, int num_ctas, cudaStream_t stream) {
    auto go = [&](auto *k, size_t bytes, int warps) {
        return launch_pdl(k, dim3(num_ctas), dim3(warps * 32), bytes, stream, p.pdl != 0, p);
    };
    return with_q4_kernel(head_dim, go);
}

}  // namespace pd
