// Append-prefill attention in the expanded form of a cache of shared latent vectors: queries of 192 values, 128 against the
// head's own expanded keys, 64 against the rotated key part all heads share; values of 128.
//
// The scheme is that of pd_prefill_attn_d128.cu: one CTA per SM owns two tiles of 128 query rows (here 256 consecutive new
// tokens of one head) that share every K and V tile, walks the context in blocks of 128 tokens, and issues
// O0(j) S0(j+1) O1(j) S1(j+1) so that the tensor pipe runs one tile's products while the other tile's warpgroup does its softmax.
// What differs and why:
// - S is a product over 192: 12 MMAs of 128 x 128 x 16 a tile and block beside 8 of O, 2560 tensor cycles a block for both tiles,
//   and 2048 cycles of exponentials (16 per clock): the tensor pipe is the bound, not the softmax.
// - Q takes 96 KB, which leaves eight pieces of 16 KB. K goes in pieces of 64 columns (two from the head's own pages, one from
//   the rotated part of the latent pages), five in flight; V in halves of 64 tokens, three in flight. A piece is handed
//   back by its last product, not with its block, so the piece a block is short of is under way 1300-1500 cycles before it is needed.
// - Each tile has its own number of blocks: the first skips those that only the second one sees, and a turn of at most 128 tokens
//   runs one tile.
// - The issuing thread is chosen by elect.sync: the products then issue in half the time they take to run.
// Tensor memory: S0 | S1 | O0 | O1, 128 columns each; P_t as bf16 over the first 64 columns of S_t. Every wait is bounded.
#include "pd_kernels.cuh"
#include "pd_ptx.cuh"
#include "pd_tcgen05.cuh"

#include <type_traits>

namespace pd {

namespace {

constexpr float kLn2f = 0.6931471805599453f;
constexpr float kRaise = 32.f;                  // log2 units a logit may exceed its row's reference
constexpr int kRows = 128;                      // query rows per tile (MMA M), one softmax thread each
constexpr int kTiles = 2;
constexpr int kBlock = 128;                     // context tokens per step
constexpr int kBlockPages = kBlock / kPageSize;
constexpr int kQDim = kLatentHead + kLatentRope;
constexpr int kPiece = 16384;                   // 128 rows of 64 columns, or 64 tokens of 128 columns
constexpr int kKPieces = kQDim / 64;            // per block
constexpr int kKSlots = 5, kVSlots = 3;
constexpr int kParts = 2, kPart = kBlock / kParts;  // P and the O product go in two parts of 64 tokens
constexpr int kSoftmaxWarps = kTiles * kRows / 32;
constexpr int kThreads = 32 * (kSoftmaxWarps + 4);  // + MMA warp, K loader, V loader, one spare
constexpr int kQTileBytes = kKPieces * kPiece;
constexpr int kTmemCols = 512;
constexpr int kColS = 0, kColO = 256;
constexpr int kNumBars = 2 * kKSlots + 2 * kVSlots + 2 + 4 + 4 + 1 + 2;
constexpr size_t kSmemBytes = 1024 + kTiles * kQTileBytes + (kKSlots + kVSlots) * kPiece + kNumBars * 8;

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ void latch(int32_t *status, int code, int seq, int detail) {
    if (atomicCAS(status, kDevOk, code) == kDevOk) {
        status[1] = seq;
        status[2] = detail;
    }
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

__global__ void __launch_bounds__(kThreads, 1)
prefill_attn_latent_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                           const __grid_constant__ CUtensorMap tm_r, const LatentPrefillParams lp) {
    const PrefillParams &p = lp.a;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_slot;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int head = blockIdx.y;
    constexpr int CTA_TOK = kTiles * kRows;

    grid_dependency_wait();
    launch_dependents();
    const int b = p.order != nullptr ? p.order[blockIdx.z] : static_cast<int>(blockIdx.z);  // heaviest sequences first
    const int q0 = p.q_indptr[b], q_len = p.q_indptr[b + 1] - q0;
    // CTAs are scheduled in index order: start a sequence's last tokens (the longest contexts) first
    const int cta_start = static_cast<int>(gridDim.x - 1 - blockIdx.x) * CTA_TOK;
    if (cta_start >= q_len) return;  // before any allocation
    const int L = min(max(p.ctx_lens[b], 0), p.MP * kPageSize);
    if (L < q_len) {  // the cache must already hold the new tokens
        if (tid == 0) latch(p.status, kDevBadLength, b, L);
        return;
    }
    const int n_tok = min(CTA_TOK, q_len - cta_start);           // valid tokens of this CTA, over both tiles
    const int pos0 = L - q_len + cta_start;                      // absolute position of the CTA's first token
    const int nb0 = (pos0 + min(n_tok, kRows) - 1) / kBlock + 1;  // context blocks each tile's last token can see
    const int nb1 = n_tok > kRows ? (pos0 + n_tok - 1) / kBlock + 1 : 0;
    const int nb = max(nb0, nb1);
    const int n_pages = (L + kPageSize - 1) / kPageSize;

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *aligned = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t q_s = base;
    const uint32_t k_ring = base + kTiles * kQTileBytes, v_ring = k_ring + kKSlots * kPiece;
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + kTiles * kQTileBytes + (kKSlots + kVSlots) * kPiece);
    const uint32_t bar_k = smem_u32(bars), bar_kfree = bar_k + kKSlots * 8;          // a piece of K landed / is free again
    const uint32_t bar_v = bar_kfree + kKSlots * 8, bar_vfree = bar_v + kVSlots * 8;
    const uint32_t bar_s = bar_vfree + kVSlots * 8;  // [2] S_t of the current block complete (and every product before it)
    const uint32_t bar_p = bar_s + 16;               // [2 tiles][2 parts] that part of P_t is written (4 warps each)
    const uint32_t bar_o = bar_p + 32;               // [2] last O_t product complete; [2] first part's O_t product of the block complete
    const uint32_t bar_drain = bar_o + 32;
    const uint32_t bar_q = bar_drain + 8;            // [2] tile t's queries are in shared memory (4 warps each)

    if (tid == 0) {
        for (int i = 0; i < kNumBars; ++i) {
            const uint32_t bar = bar_k + i * 8;
            mbar_init(bar, bar >= bar_q || (bar >= bar_p && bar < bar_o) ? kRows / 32 : 1);
        }
        mbar_init_fence();
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
        prefetch_tensormap(&tm_r);
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(&tmem_slot), kTmemCols);
        tmem_relinquish_alloc_permit();
    }
    const int tile = tid / kRows, row = tid & (kRows - 1);  // of a softmax thread
    const int tok = tile * kRows + row;                 // token index inside the CTA
    const bool row_valid = tid < kTiles * kRows && tok < n_tok;
    const int my_pos = pos0 + min(tok, n_tok - 1);      // padding rows mirror the last token
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tm = tmem_slot;
    bool ok = true;

    if (warp == kSoftmaxWarps) {
        // ================= MMA warp: one elected thread issues every product =================
        if (elect_one()) {
            constexpr uint32_t idesc_s = umma_idesc_bf16(kRows, kBlock, false);
            constexpr uint32_t idesc_o = umma_idesc_bf16(kRows, kLatentHead, true);
            const uint64_t q_desc = umma_smem_desc(q_s, 16, 1024), k_desc = umma_smem_desc(k_ring, 16, 1024);
            const uint64_t v_desc = umma_smem_desc(v_ring, kPart * 128, 1024);
            auto issue_s = [&](int t, int j, bool wait, bool release) {  // S_t(j) = Q_t K_j^T
#pragma unroll
                for (int c = 0; c < kKPieces; ++c) {
                    const int i = j * kKPieces + c, slot = i % kKSlots;
                    if (wait) {
                        ok = ok && mbar_wait(bar_k + slot * 8, (i / kKSlots) & 1);
                        if (!ok) return;
                        tc_fence_after_sync();
                    }
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        umma_ss(tm + kColS + t * kBlock, q_desc + ((t * kQTileBytes + c * kPiece) >> 4) + ks * 2,
                                k_desc + slot * (kPiece >> 4) + ks * 2, idesc_s, (c | ks) != 0);
                    if (release) umma_commit(bar_kfree + slot * 8);
                }
                umma_commit(bar_s + t * 8);
            };
            auto issue_o = [&](int t, int j, int part, bool wait, bool release, bool last) {  // O_t += P_t(j)[:, part] V_j[part]
                const int i = j * kParts + part, slot = i % kVSlots;
                ok = ok && mbar_wait(bar_p + (t * 2 + part) * 8, j & 1);
                if (wait) ok = ok && mbar_wait(bar_v + slot * 8, (i / kVSlots) & 1);
                if (!ok) return;
                tc_fence_after_sync();
#pragma unroll
                for (int ks = 0; ks < kPart / 16; ++ks)
                    umma_ts(tm + kColO + t * kLatentHead, tm + kColS + t * kBlock + (part * (kPart / 16) + ks) * 8,
                            v_desc + slot * (kPiece >> 4) + ks * (2048 >> 4), idesc_o, (j | part | ks) != 0);
                if (release) umma_commit(bar_vfree + slot * 8);
                if (part == 0) umma_commit(bar_o + (2 + t) * 8);  // lets a row thread rescale O_t between the two parts (rare)
                else if (last) umma_commit(bar_o + t * 8);
            };
            ok = mbar_wait(bar_q, 0);
            if (ok) issue_s(0, 0, true, nb1 == 0);
            if (nb1 > 0) ok = ok && mbar_wait(bar_q + 8, 0);
            if (ok && nb1 > 0) issue_s(1, 0, false, true);
            // the tile that meets a piece first waits for it, the one that meets it last hands it back
            for (int j = 0; j < nb && ok; ++j) {
                const bool u0 = j < nb0, u1 = j < nb1, n0 = j + 1 < nb0, n1 = j + 1 < nb1;
                if (u0) {
                    issue_o(0, j, 0, true, !u1, j == nb0 - 1);
                    if (ok) issue_o(0, j, 1, true, !u1, j == nb0 - 1);
                }
                if (ok && n0) issue_s(0, j + 1, true, !n1);
                if (ok && u1) {
                    issue_o(1, j, 0, !u0, true, j == nb1 - 1);
                    if (ok) issue_o(1, j, 1, !u0, true, j == nb1 - 1);
                }
                if (ok && n1) issue_s(1, j + 1, !n0, true);
            }
            if (!ok) latch(p.status, kDevTimeout, b, blockIdx.x);
            umma_commit(bar_drain);  // nothing may be in flight when the tensor memory is freed
            mbar_wait(bar_drain, 0);
        }
    } else if (warp == kSoftmaxWarps + 1 || warp == kSoftmaxWarps + 2) {
        // ================= two TMA warps (one streams K, the other V): one box per lane, eight per piece =================
        const uint64_t policy = l2_policy_evict_first();
        const bool is_k = warp == kSoftmaxWarps + 1;
        const int32_t oob_kv = lp.kv_num_pages * p.Hq * kPageSize, oob_r = p.num_pages * kPageSize;  // boxes there are zero fill
        const int32_t *kv_row = lp.kv_table + static_cast<size_t>(b) * p.MP, *r_row = p.page_table + static_cast<size_t>(b) * p.MP;
        int issued = 0;
        auto page_y = [&](const int32_t *table_row, int lp_page, int limit, int scale, int add, int32_t oob) {
            if (lp_page >= n_pages) return oob;
            int pid = __ldg(table_row + lp_page);
            if (pid < 0 || pid >= limit) {
                latch(p.status, kDevBadPage, b, pid);
                pid = 0;
            }
            return (pid * scale + add) * kPageSize;
        };
        if (is_k) {
            int32_t y_next = lane < 16 ? (lane < 8 ? page_y(kv_row, lane, lp.kv_num_pages, p.Hq, head, oob_kv)
                                                   : page_y(r_row, lane - 8, p.num_pages, 1, 0, oob_r)) : 0;
            for (int j = 0; j < nb && ok; ++j) {
                const int32_t y = y_next;  // lanes 0..7: the block's pages of K, lanes 8..15: of the rotated part
                if (j + 1 < nb && lane < 16)
                    y_next = lane < 8 ? page_y(kv_row, (j + 1) * kBlockPages + lane, lp.kv_num_pages, p.Hq, head, oob_kv)
                                      : page_y(r_row, (j + 1) * kBlockPages + lane - 8, p.num_pages, 1, 0, oob_r);
                for (int c = 0; c < kKPieces; ++c) {
                    const int i = j * kKPieces + c, slot = i % kKSlots, fill = i / kKSlots;
                    if (fill > 0) ok = __all_sync(0xffffffffu, mbar_wait(bar_kfree + slot * 8, (fill - 1) & 1));
                    if (!ok) break;
                    if (lane == 0) mbar_arrive_expect_tx(bar_k + slot * 8, kPiece);
                    __syncwarp();
                    const uint32_t dst = k_ring + slot * kPiece + (lane & 7) * (kPageSize * 128);
                    if (c < 2 && lane < 8) tma_load_2d(dst, &tm_k, c * 64, y, bar_k + slot * 8, policy);
                    if (c == 2 && lane >= 8 && lane < 16) tma_load_2d(dst, &tm_r, kLatentDim, y, bar_k + slot * 8, policy);
                    issued = i + 1;
                }
            }
        } else {
            int32_t y_next = lane < 8 ? page_y(kv_row, lane, lp.kv_num_pages, p.Hq, head, oob_kv) : 0;
            for (int j = 0; j < nb && ok; ++j) {
                const int32_t y = y_next;
                if (j + 1 < nb && lane < 8) y_next = page_y(kv_row, (j + 1) * kBlockPages + lane, lp.kv_num_pages, p.Hq, head, oob_kv);
                for (int part = 0; part < kParts; ++part) {
                    const int i = j * kParts + part, slot = i % kVSlots, fill = i / kVSlots;
                    if (fill > 0) ok = __all_sync(0xffffffffu, mbar_wait(bar_vfree + slot * 8, (fill - 1) & 1));
                    if (!ok) break;
                    if (lane == 0) mbar_arrive_expect_tx(bar_v + slot * 8, kPiece);
                    __syncwarp();
                    const int32_t yy = __shfl_sync(0xffffffffu, y, part * 4 + ((lane >> 1) & 3));
                    if (lane < 8)
                        tma_load_2d(v_ring + slot * kPiece + (lane & 1) * (kPart * 128) + (lane >> 1) * (kPageSize * 128), &tm_v, (lane & 1) * 64, yy,
                                    bar_v + slot * 8, policy);
                    issued = i + 1;
                }
            }
        }
        if (!ok) {  // copies in flight have to land before the block's memory goes
            if (lane == 0) latch(p.status, kDevTimeout, b, blockIdx.x);
            const int slots = is_k ? kKSlots : kVSlots;
            for (int i = max(0, issued - slots); i < issued; ++i) mbar_wait((is_k ? bar_k : bar_v) + (i % slots) * 8, (i / slots) & 1);
        }
    } else if (warp < kSoftmaxWarps && (tile == 0 || nb1 > 0)) {
        // ================= softmax warpgroups: warpgroup t owns tile t, one thread per query row =================
        const int t = tile, my_nb = t == 0 ? nb0 : nb1;
        const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_buf = tm + lane_base + kColS + t * kBlock;
        const uint32_t o_buf = tm + lane_base + kColO + t * kLatentHead;
        // ---- the tile's queries: neighbouring threads copy neighbouring 16 bytes, all in flight at once
        {
            constexpr int kChunks = kQDim / 8;  // 128 rows x 24 pieces over 128 threads
            const __nv_bfloat16 *src = p.q + (static_cast<size_t>(q0 + cta_start + tile * kRows) * p.Hq + head) * kQDim;
            const int rows = min(kRows, n_tok - tile * kRows);
#pragma unroll
            for (int i = 0; i < kChunks; ++i) {
                const int x = i * kRows + row, r = x / kChunks, c = x - r * kChunks;
                const uint32_t a = q_s + tile * kQTileBytes + (c >> 3) * kPiece + sw128_offset(r, c & 7);
                cp_async16(a, src + static_cast<size_t>(min(r, rows - 1)) * p.Hq * kQDim + c * 8, r < rows ? 16 : 0);  // rows past the last are zeros
            }
            cp_async_wait_all();
            fence_proxy_async();  // written through the generic proxy, read by the tensor core through the async one
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_q + t * 8);
        }
        float m_run = 0.f, l_run = 0.f;
        for (int j = 0; j < my_nb && ok; ++j) {
            ok = mbar_wait(bar_s + t * 8, j & 1);
            tc_fence_after_sync();
            if (!ok) break;
            const int t0 = j * kBlock;
            const bool masked = t0 + kBlock - 1 > my_pos;  // the block reaches past this row's position
            // V rows past the context inside the last page may hold NaN; 0 * NaN is NaN, so the warpgroup whose products of
            // this block come first clears them
            const int valid_rows = L - t0;
            if (valid_rows < kBlock && (t == 0 || j >= nb0)) {
                const int last = min(kBlock, (valid_rows + kPageSize - 1) / kPageSize * kPageSize);
                for (int part = 0; part < kParts; ++part) {  // the parts must have landed
                    const int i = j * kParts + part;
                    ok = ok && mbar_wait(bar_v + (i % kVSlots) * 8, (i / kVSlots) & 1);
                }
                if (!ok) break;
                for (int i = row; i < (last - valid_rows) * (kLatentHead / 8); i += kRows) {
                    const int r = valid_rows + i / (kLatentHead / 8), c = i % (kLatentHead / 8);
                    const int slot = (j * kParts + r / kPart) % kVSlots;
                    st_shared_zero16(v_ring + slot * kPiece + (c >> 3) * (kPart * 128) + (r % kPart) * 128 + (c & 7) * 16);
                }
                fence_proxy_async();
            }
            auto load = [&](int part, uint32_t (&v)[kPart]) {
#pragma unroll
                for (int c = 0; c < kPart; c += 32) tmem_ld32(s_buf + part * kPart + c, *reinterpret_cast<uint32_t(*)[32]>(v + c));
            };
            // one part of 64 tokens: x = s * scale - m against the reference as it stands, P = 2^x and its sum at once, so that the
            // special-function unit starts with the first logits; the largest x is looked at behind them
            auto weigh = [&](auto masked_c, int part, uint32_t (&v)[kPart], uint32_t (&pk)[kPart / 2], float &sum) {
                if (decltype(masked_c)::value) {  // mask by select: masked logits become -inf, their exponentials exact zeros
                    const int visible = my_pos - (t0 + part * kPart) + 1;
#pragma unroll
                    for (int c = 0; c < kPart; ++c)
                        if (c >= visible) v[c] = 0xff800000u;
                }
                const float2 sc2 = make_float2(p.scale_log2, p.scale_log2), nm2 = make_float2(-m_run, -m_run);
                float xm[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                float2 a[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int c = 0; c < kPart; c += 4) {
                    const float2 x = __ffma2_rn(make_float2(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), sc2, nm2);
                    const float2 y = __ffma2_rn(make_float2(__uint_as_float(v[c + 2]), __uint_as_float(v[c + 3])), sc2, nm2);
                    xm[(c >> 2) & 1] = max3(xm[(c >> 2) & 1], x.x, x.y);
                    xm[2 + ((c >> 2) & 1)] = max3(xm[2 + ((c >> 2) & 1)], y.x, y.y);
                    const float2 e = make_float2(fast_exp2(x.x), fast_exp2(x.y)), f = make_float2(fast_exp2(y.x), fast_exp2(y.y));
                    a[0] = __fadd2_rn(a[0], e);
                    a[1] = __fadd2_rn(a[1], f);
                    pk[c >> 1] = pack_bf16x2(e.x, e.y);
                    pk[(c >> 1) + 1] = pack_bf16x2(f.x, f.y);
                }
                sum = (a[0].x + a[0].y) + (a[1].x + a[1].y);
                return fmaxf(fmaxf(xm[0], xm[1]), fmaxf(xm[2], xm[3]));
            };
            auto hand_over = [&](auto masked_c, int part, float xmax, uint32_t (&pk)[kPart / 2], float sum) {
                if (__any_sync(0xffffffffu, xmax > kRaise)) {
                    // rare: the row's reference rises by its largest x, what it has accumulated is rescaled, and the part is weighed again
                    // (its logits still stand in tensor memory)
                    const float shift = xmax > kRaise ? xmax : 0.f, alpha = fast_exp2(-shift);
                    m_run += shift;
                    if (j > 0 || part > 0) {
                        if (part > 0) {  // the first part's product of this block must be over before O_t is touched
                            ok = ok && mbar_wait(bar_o + (2 + t) * 8, j & 1);
                            tc_fence_after_sync();
                        }  // (the commit that announced S_t(j) also covers O_t(j-1))
#pragma unroll 1
                        for (int c = 0; c < kLatentHead; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(o_buf + c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                            tmem_st16(o_buf + c, o);
                        }
                        tmem_wait_st();
                        l_run *= alpha;
                    }
                    uint32_t v[kPart];
                    load(part, v);
                    tmem_wait_ld();
                    weigh(masked_c, part, v, pk, sum);
                }
                l_run += sum;
                // P over the first 64 columns of the tile's logit buffer (columns this thread has already consumed)
#pragma unroll
                for (int c = 0; c < kPart / 2; c += 16) tmem_st16(s_buf + part * (kPart / 2) + c, *reinterpret_cast<uint32_t(*)[16]>(pk + c));
                tmem_wait_st();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_p + (t * 2 + part) * 8);
            };
            auto do_block = [&](auto masked_c) {
                uint32_t va[kPart], vb[kPart], pk[kPart / 2];
                float sum;
                load(0, va);
                tmem_wait_ld();
                if (j == 0) {  // the reference: the row's largest logit of the first part, finite because position 0 is visible
                    float top = -INFINITY;
                    const int visible = my_pos + 1;
#pragma unroll
                    for (int c = 0; c < kPart; ++c) top = c < visible ? fmaxf(top, __uint_as_float(va[c])) : top;
                    m_run = top * p.scale_log2;
                }
                load(1, vb);  // on their way while the first part's exponentials run
                float xmax = weigh(masked_c, 0, va, pk, sum);
                tmem_wait_ld();
                hand_over(masked_c, 0, xmax, pk, sum);
                xmax = weigh(masked_c, 1, vb, pk, sum);
                hand_over(masked_c, 1, xmax, pk, sum);
            };
            if (__any_sync(0xffffffffu, masked)) do_block(std::true_type{});
            else do_block(std::false_type{});
        }

        // ---- epilogue: O_t / l -> bf16 rows
        ok = ok && mbar_wait(bar_o + t * 8, 0);
        tc_fence_after_sync();
        const float inv = 1.f / l_run;
        const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0;
        __nv_bfloat16 *orow = p.out + (static_cast<size_t>(q0 + cta_start + min(tok, n_tok - 1)) * p.Hq + head) * kLatentHead;
#pragma unroll
        for (int c = 0; c < kLatentHead; c += 32) {
            uint32_t o[32];
            tmem_ld32(o_buf + c, o);
            tmem_wait_ld();
            if (row_valid && ok) {
#pragma unroll
                for (int i = 0; i < 32; i += 16) {
                    uint32_t v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = pack_bf16x2(__uint_as_float(o[i + 2 * k]) * inv, __uint_as_float(o[i + 2 * k + 1]) * inv);
                    if (wide) {
                        store32(orow + c + i, v);
                    } else {
                        *reinterpret_cast<uint4 *>(orow + c + i) = make_uint4(v[0], v[1], v[2], v[3]);
                        *reinterpret_cast<uint4 *>(orow + c + i + 8) = make_uint4(v[4], v[5], v[6], v[7]);
                    }
                }
            }
        }
        if (p.lse != nullptr && row_valid && ok)
            p.lse[static_cast<size_t>(q0 + cta_start + tok) * p.Hq + head] = (m_run + log2f(l_run)) * kLn2f;
        if (!ok && lane == 0) latch(p.status, kDevTimeout, b, blockIdx.x);
    }
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tm, kTmemCols);
}

}  // namespace

cudaError_t prepare_prefill_attn_latent() {
    return cudaFuncSetAttribute(prefill_attn_latent_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmemBytes));
}

cudaError_t launch_prefill_attn_latent(const CUtensorMap &tm_k, const CUtensorMap &tm_v, const CUtensorMap &tm_r,
                                       const LatentPrefillParams &p, int max_q_len, cudaStream_t stream) {
    if (p.a.order != nullptr) {
        const cudaError_t e = launch_prefill_order(p.a, stream);
        if (e != cudaSuccess) return e;
    }
    const dim3 grid((max_q_len + kTiles * kRows - 1) / (kTiles * kRows), p.a.Hq, p.a.B);
    return launch_pdl(prefill_attn_latent_kernel, grid, dim3(kThreads), kSmemBytes, stream, p.a.pdl != 0, tm_k, tm_v, tm_r, p);
}

}  // namespace pd
