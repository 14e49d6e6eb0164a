// Append-prefill attention in the expanded form of a cache of shared latent vectors: queries of 192 values, 128 against the
// head's own expanded keys, 64 against the rotated key part all heads share; values of 128.
//
// One CTA per SM owns two tiles of 128 query rows (256 consecutive new tokens of one head) that share every K and V tile, as in
// pd_prefill_attn_d128.cu, and walks the context in blocks of 80 tokens (5 pages):
//   tcgen05  S_t = Q_t K^T (12 MMAs of 128 x 80 x 16, Q and K from shared memory), O_t += P_t V (5 of 128 x 128 x 16, P_t from
//            tensor memory), in the order S0(j+1) O0(j) S1(j+1) O1(j)
//   softmax  one warpgroup per tile, one thread per row
// Why 80: tensor memory has 128 columns a tile beside its 128 of O. With blocks of 128 P has to lie where S lay, so S(j+1) waits
// for the softmax of block j, for its O product and for four hand-overs: 3630 cycles per 128 tokens (both tiles), where the
// products take 2560. With 80 columns of S and 40 of P beside them, S(j+1) waits only until the row threads hold the
// logits of block j in registers, and runs during their softmax. What bounds it now is shared memory: an S product reads 4 KB of Q and 2.5 KB of
// K in 51 cycles (128 bytes each), 1864 cycles a block with O, and the copies write 50 KB (400 cycles) beside that.
// A page's 128 columns come as one box in the order [8-row group][64-column half][8 rows]: row groups follow one another
// at the same distance across pages, as both operand forms want it.
// Each tile has its own number of blocks: the first skips those that only the second one sees, and a turn of at most 128 tokens
// runs one tile. Tensor memory: (S0 80, P0 40) (S1, P1) O0 O1, 128 columns each. Every wait is bounded.
#include "pd_kernels.cuh"
#include "pd_ptx.cuh"
#include "pd_tcgen05.cuh"

namespace pd {

namespace {

constexpr float kLn2f = 0.6931471805599453f;
constexpr float kRaise = 32.f;                  // log2 units a logit may exceed its row's reference
constexpr int kRows = 128;                      // query rows per tile (MMA M), one softmax thread each
constexpr int kTiles = 2;
constexpr int kBlock = 80;                      // context tokens per step
constexpr int kBlockPages = kBlock / kPageSize;
constexpr int kQDim = kLatentHead + kLatentRope;
constexpr int kQPiece = kRows * 128;            // 64 columns of a Q tile
constexpr int kQTileBytes = kQDim / 64 * kQPiece;
constexpr int kKvBytes = kBlock * kLatentHead * 2;   // a block's K or V
constexpr int kRopeBytes = kBlock * kLatentRope * 2;
constexpr int kKSlots = 2, kVSlots = 3;
constexpr int kSoftmaxWarps = kTiles * kRows / 32;
constexpr int kThreads = 32 * (kSoftmaxWarps + 4);  // + MMA warp, K loader, V loader, one spare
constexpr int kTmemCols = 512;
constexpr int kColS = 0, kColP = kBlock, kColO = 256;  // S_t, P_t at 128 t + .., O_t at kColO + 128 t
// Registers per thread: the softmax keeps a row's 80 logits and 40 packed weights, which do not fit the launch's 168 without spills.
// 128 * 104 + 256 * 200 = 384 * 168.
constexpr int kOtherRegs = 104, kSoftmaxRegs = 200;
constexpr int kNumBars = 4 * kKSlots + 2 * kVSlots + 5 * kTiles + 1;
constexpr size_t kSmemBytes = 1024 + kTiles * kQTileBytes + kKSlots * (kKvBytes + kRopeBytes) + kVSlots * kKvBytes + kNumBars * 8;

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
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void *tmap, int32_t w, uint32_t bar, uint64_t l2_policy) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
                 " [%0], [%1, {%2, %2, %2, %3}], [%4], %5;"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(0), "r"(w), "r"(bar), "l"(l2_policy) : "memory");
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
    // heaviest sequences first: up to 32 sequences every warp ranks them by itself, beyond that a small kernel did
    int b, q0, q_len, len;
    if (p.order == nullptr) {
        const int mine = min(lane, p.B - 1);
        const int from = p.q_indptr[mine], n = p.q_indptr[mine + 1] - from, L0 = p.ctx_lens[mine];
        const long long work = static_cast<long long>(n) * (2ll * L0 - n);
        int rank = 0;
        for (int i = 0; i < p.B; ++i) {
            const long long w = __shfl_sync(0xffffffffu, work, i);
            rank += w > work || (w == work && i < lane) ? 1 : 0;
        }
        b = __ffs(__ballot_sync(0xffffffffu, lane < p.B && rank == static_cast<int>(blockIdx.z))) - 1;
        q0 = __shfl_sync(0xffffffffu, from, b);
        q_len = __shfl_sync(0xffffffffu, n, b);
        len = __shfl_sync(0xffffffffu, L0, b);
    } else {
        b = p.order[blockIdx.z];
        q0 = p.q_indptr[b];
        q_len = p.q_indptr[b + 1] - q0;
        len = p.ctx_lens[b];
    }
    // CTAs are scheduled in index order: start a sequence's last tokens (the longest contexts) first
    const int cta_start = static_cast<int>(gridDim.x - 1 - blockIdx.x) * CTA_TOK;
    if (cta_start >= q_len) return;  // before any allocation
    const int L = min(max(len, 0), p.MP * kPageSize);
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
    const uint32_t q_s = base, k_ring = q_s + kTiles * kQTileBytes, r_ring = k_ring + kKSlots * kKvBytes;
    const uint32_t v_ring = r_ring + kKSlots * kRopeBytes;
    const uint32_t bar_k = v_ring + kVSlots * kKvBytes, bar_kfree = bar_k + kKSlots * 8;  // a block of K landed / is free again
    const uint32_t bar_r = bar_kfree + kKSlots * 8, bar_rfree = bar_r + kKSlots * 8;      // the same of the rotated part
    const uint32_t bar_v = bar_rfree + kKSlots * 8, bar_vfree = bar_v + kVSlots * 8;
    const uint32_t bar_s = bar_vfree + kVSlots * 8;  // [2] S_t of the block complete
    const uint32_t bar_o = bar_s + kTiles * 8;       // [2] O_t product of the block complete
    const uint32_t bar_drain = bar_o + kTiles * 8;
    const uint32_t bar_sfree = bar_drain + 8;        // [2] the rows hold S_t of the block in registers (4 warps each, like the next two)
    const uint32_t bar_p = bar_sfree + kTiles * 8;   // [2] P_t is written
    const uint32_t bar_q = bar_p + kTiles * 8;       // [2] tile t's queries are in shared memory

    if (tid == 0) {
        for (int i = 0; i < kNumBars; ++i) {
            const uint32_t bar = bar_k + i * 8;
            mbar_init(bar, bar >= bar_sfree ? kRows / 32 : 1);
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

    if (warp >= kSoftmaxWarps) {
        setmaxnreg_dec<kOtherRegs>();
        if (warp == kSoftmaxWarps) {
            // ================= MMA warp: one elected thread issues every product =================
            if (elect_one()) {
                constexpr uint32_t idesc_s = umma_idesc_bf16(kRows, kBlock, false);
                constexpr uint32_t idesc_o = umma_idesc_bf16(kRows, kLatentHead, true);
                const uint64_t q_desc = umma_smem_desc(q_s, 16, 1024), k_desc = umma_smem_desc(k_ring, 16, 2048);
                const uint64_t r_desc = umma_smem_desc(r_ring, 16, 1024), v_desc = umma_smem_desc(v_ring, 1024, 2048);
                auto issue_s = [&](int t, int j, bool wait, bool release) {  // S_t(j) = Q_t K_j^T
                    const int slot = j % kKSlots;
                    const uint32_t d = tm + kColS + t * 128, parity = (j / kKSlots) & 1;
                    const uint64_t q = q_desc + (t * kQTileBytes >> 4);
                    if (wait) ok = ok && mbar_wait(bar_k + slot * 8, parity);
                    if (!ok) return;
                    tc_fence_after_sync();
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            umma_ss(d, q + (c * kQPiece >> 4) + ks * 2, k_desc + slot * (kKvBytes >> 4) + c * (1024 >> 4) + ks * 2, idesc_s, (c | ks) != 0);
                    if (release) umma_commit(bar_kfree + slot * 8);
                    if (wait) ok = mbar_wait(bar_r + slot * 8, parity);
                    if (!ok) return;
                    tc_fence_after_sync();
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        umma_ss(d, q + (2 * kQPiece >> 4) + ks * 2, r_desc + slot * (kRopeBytes >> 4) + ks * 2, idesc_s, true);
                    if (release) umma_commit(bar_rfree + slot * 8);
                    umma_commit(bar_s + t * 8);
                };
                auto issue_o = [&](int t, int j, bool wait, bool release) {  // O_t += P_t(j) V_j
                    const int slot = j % kVSlots;
                    ok = mbar_wait(bar_p + t * 8, j & 1);
                    if (wait) ok = ok && mbar_wait(bar_v + slot * 8, (j / kVSlots) & 1);
                    if (!ok) return;
                    tc_fence_after_sync();
#pragma unroll
                    for (int ks = 0; ks < kBlock / 16; ++ks)
                        umma_ts(tm + kColO + t * kLatentHead, tm + t * 128 + kColP + ks * 8, v_desc + slot * (kKvBytes >> 4) + ks * (4096 >> 4), idesc_o,
                                (j | ks) != 0);
                    if (release) umma_commit(bar_vfree + slot * 8);
                    umma_commit(bar_o + t * 8);
                };
                ok = mbar_wait(bar_q, 0);
                if (ok) issue_s(0, 0, true, nb1 == 0);
                if (nb1 > 0) ok = ok && mbar_wait(bar_q + 8, 0);
                if (ok && nb1 > 0) issue_s(1, 0, false, true);
                // the tile that meets a block first waits for it, the one that meets it last hands it back
                for (int j = 0; j < nb && ok; ++j) {
                    const bool u0 = j < nb0, u1 = j < nb1, n0 = j + 1 < nb0, n1 = j + 1 < nb1;
                    if (n0) ok = mbar_wait(bar_sfree, j & 1);
                    if (ok && n0) issue_s(0, j + 1, true, !n1);
                    if (ok && u0) issue_o(0, j, true, !u1);
                    if (ok && n1) ok = mbar_wait(bar_sfree + 8, j & 1);
                    if (ok && n1) issue_s(1, j + 1, !n0, true);
                    if (ok && u1) issue_o(1, j, !u0, true);
                }
                if (!ok) latch(p.status, kDevTimeout, b, blockIdx.x);
                umma_commit(bar_drain);  // nothing may be in flight when the tensor memory is freed
                mbar_wait(bar_drain, 0);
            }
        } else if (warp == kSoftmaxWarps + 1 || warp == kSoftmaxWarps + 2) {
            // ================= two TMA warps (K and the rotated part, V), one elected thread each =================
            if (elect_one()) {
                const uint64_t policy = l2_policy_evict_first();
                const bool is_k = warp == kSoftmaxWarps + 1;
                const int32_t *kv_row = lp.kv_table + static_cast<size_t>(b) * p.MP, *r_row = p.page_table + static_cast<size_t>(b) * p.MP;
                int issued = 0, issued_r = 0;
                int32_t kv_id[kBlockPages], r_id[kBlockPages];  // the next block's pages
                auto load_ids = [&](int j) {
#pragma unroll
                    for (int g = 0; g < kBlockPages; ++g) {
                        const int page = j * kBlockPages + g;
                        kv_id[g] = page < n_pages ? __ldg(kv_row + page) : 0;
                        if (is_k) r_id[g] = page < n_pages ? __ldg(r_row + page) : 0;
                    }
                };
                auto checked = [&](int32_t pid, int page, int limit) {  // `limit`: a page past the pool is zero fill
                    if (page >= n_pages) return limit;
                    if (pid >= 0 && pid < limit) return pid;
                    latch(p.status, kDevBadPage, b, pid);
                    return 0;
                };
                load_ids(0);
                for (int j = 0; j < nb && ok; ++j) {
                    int32_t kv_page[kBlockPages], r_page[kBlockPages];
#pragma unroll
                    for (int g = 0; g < kBlockPages; ++g) {
                        kv_page[g] = checked(kv_id[g], j * kBlockPages + g, lp.kv_num_pages);
                        r_page[g] = is_k ? checked(r_id[g], j * kBlockPages + g, p.num_pages) : 0;
                    }
                    if (j + 1 < nb) load_ids(j + 1);
                    const int slots = is_k ? kKSlots : kVSlots, slot = j % slots, fill = j / slots;
                    const uint32_t full = (is_k ? bar_k : bar_v) + slot * 8, dst = (is_k ? k_ring : v_ring) + slot * kKvBytes;
                    if (fill > 0) ok = mbar_wait((is_k ? bar_kfree : bar_vfree) + slot * 8, (fill - 1) & 1);
                    if (!ok) break;
                    mbar_arrive_expect_tx(full, kKvBytes);
#pragma unroll
                    for (int g = 0; g < kBlockPages; ++g) tma_load_4d(dst + g * 4096, is_k ? &tm_k : &tm_v, (kv_page[g] * p.Hq + (kv_page[g] < lp.kv_num_pages ? head : 0)) * 2, full, policy);
                    issued = j + 1;
                    if (is_k) {
                        if (fill > 0) ok = mbar_wait(bar_rfree + slot * 8, (fill - 1) & 1);
                        if (!ok) break;
                        mbar_arrive_expect_tx(bar_r + slot * 8, kRopeBytes);
#pragma unroll
                        for (int g = 0; g < kBlockPages; ++g)
                            tma_load_2d(r_ring + slot * kRopeBytes + g * (kPageSize * 128), &tm_r, kLatentDim, r_page[g] * kPageSize, bar_r + slot * 8, policy);
                        issued_r = j + 1;
                    }
                }
                if (!ok) {  // copies in flight have to land before the block's memory goes
                    latch(p.status, kDevTimeout, b, blockIdx.x);
                    const int slots = is_k ? kKSlots : kVSlots;
                    for (int i = max(0, issued - slots); i < issued; ++i) mbar_wait((is_k ? bar_k : bar_v) + (i % slots) * 8, (i / slots) & 1);
                    for (int i = max(0, issued_r - kKSlots); i < issued_r; ++i) mbar_wait(bar_r + (i % kKSlots) * 8, (i / kKSlots) & 1);
                }
            }
        }
    } else {
        setmaxnreg_inc<kSoftmaxRegs>();
        if (tile == 0 || nb1 > 0) {
            // ================= softmax warpgroups: warpgroup t owns tile t, one thread per query row =================
            const int t = tile, my_nb = t == 0 ? nb0 : nb1;
            const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
            const uint32_t s_buf = tm + lane_base + kColS + t * 128, p_buf = tm + lane_base + kColP + t * 128;
            const uint32_t o_buf = tm + lane_base + kColO + t * kLatentHead;
            // ---- the tile's queries: neighbouring threads copy neighbouring 16 bytes, all in flight at once
            {
                constexpr int kChunks = kQDim / 8;  // 128 rows x 24 pieces over 128 threads
                const __nv_bfloat16 *src = p.q + (static_cast<size_t>(q0 + cta_start + tile * kRows) * p.Hq + head) * kQDim;
                const int rows = min(kRows, n_tok - tile * kRows);
#pragma unroll
                for (int i = 0; i < kChunks; ++i) {
                    const int x = i * kRows + row, r = x / kChunks, c = x - r * kChunks;
                    const uint32_t a = q_s + tile * kQTileBytes + (c >> 3) * kQPiece + sw128_offset(r, c & 7);
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
                    ok = mbar_wait(bar_v + (j % kVSlots) * 8, (j / kVSlots) & 1);  // it must have landed
                    if (!ok) break;
                    for (int i = row; i < (last - valid_rows) * (kLatentHead / 8); i += kRows) {
                        const int r = valid_rows + i / (kLatentHead / 8), c = i % (kLatentHead / 8);
                        st_shared_zero16(v_ring + (j % kVSlots) * kKvBytes + (r >> 3) * 2048 + (c >> 3) * 1024 + (r & 7) * 128 + (c & 7) * 16);
                    }
                    fence_proxy_async();
                }
                uint32_t v[kBlock], pk[kBlock / 2];
                tmem_ld32(s_buf, *reinterpret_cast<uint32_t(*)[32]>(v));
                tmem_ld32(s_buf + 32, *reinterpret_cast<uint32_t(*)[32]>(v + 32));
                tmem_ld16(s_buf + 64, *reinterpret_cast<uint32_t(*)[16]>(v + 64));
                tmem_wait_ld();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_sfree + t * 8);  // S_t(j+1) may come
                float sum = 0.f;
                // x = s * scale - m against the reference as it stands, P = 2^x and its sum at once, so that the special-function unit
                // starts with the first logits; the largest x is looked at behind them
                auto weigh = [&]() {
                    const float2 sc2 = make_float2(p.scale_log2, p.scale_log2), nm2 = make_float2(-m_run, -m_run);
                    float xm[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    float2 a[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                    for (int c = 0; c < kBlock; c += 4) {
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
                if (__any_sync(0xffffffffu, masked)) {  // masked logits become -inf, their exponentials exact zeros
                    const int visible = my_pos - t0 + 1;
#pragma unroll
                    for (int c = 0; c < kBlock; ++c)
                        if (c >= visible) v[c] = 0xff800000u;
                }
                if (j == 0) {  // the reference: the row's largest logit of the block, finite because position 0 is visible
                    float top = -INFINITY;
#pragma unroll
                    for (int c = 0; c < kBlock; c += 2) top = max3(top, __uint_as_float(v[c]), __uint_as_float(v[c + 1]));
                    m_run = top * p.scale_log2;
                }
                const float xmax = weigh();
                if (__any_sync(0xffffffffu, xmax > kRaise)) {
                    // rare: the row's reference rises by its largest x, what it has accumulated is rescaled, and the block is weighed again
                    const float shift = xmax > kRaise ? xmax : 0.f, alpha = fast_exp2(-shift);
                    m_run += shift;
                    if (j > 0) {
                        ok = mbar_wait(bar_o + t * 8, (j - 1) & 1);
                        tc_fence_after_sync();
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
                    weigh();
                }
                l_run += sum;
                if (j > 0) {  // P_t has been used by the last block's product
                    ok = ok && mbar_wait(bar_o + t * 8, (j - 1) & 1);
                    if (!ok) break;
                    tc_fence_after_sync();
                }
                tmem_st16(p_buf, *reinterpret_cast<uint32_t(*)[16]>(pk));
                tmem_st16(p_buf + 16, *reinterpret_cast<uint32_t(*)[16]>(pk + 16));
                tmem_st8(p_buf + 32, *reinterpret_cast<uint32_t(*)[8]>(pk + 32));
                tmem_wait_st();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_p + t * 8);
            }

            // ---- epilogue: O_t / l -> bf16 rows
            ok = ok && mbar_wait(bar_o + t * 8, (my_nb - 1) & 1);
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
                                       const LatentPrefillParams &base, int max_q_len, int *launched, cudaStream_t stream) {
    LatentPrefillParams p = base;
    *launched = 0;
    if (p.a.B <= 32) p.a.order = nullptr;
    if (p.a.order != nullptr) {
        const cudaError_t e = launch_prefill_order(p.a, stream);
        if (e != cudaSuccess) return e;
        *launched = 1;
    }
    *launched += 1;
    const dim3 grid((max_q_len + kTiles * kRows - 1) / (kTiles * kRows), p.a.Hq, p.a.B);
    return launch_pdl(prefill_attn_latent_kernel, grid, dim3(kThreads), kSmemBytes, stream, p.a.pdl != 0, tm_k, tm_v, tm_r, p);
}

}  // namespace pd
