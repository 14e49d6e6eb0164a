// K and V of every head from cached latents: K_h = W_h[0:128] c, V_h = W_h[128:256] c, for the tokens of a batch of contexts,
// from latent pages into pages of bf16 K and V. A matrix product [tokens x 512] x [512 x 256 per head] whose rows are gathered
// by page and whose results are scattered by page.
//
// A unit is (two tiles of 128 tokens, head): 32 MMAs of 256 x 256 x 16 over a pair of CTAs (a cluster), a tile in each, 4096
// cycles, for 256 KB of latents, 256 KB of W (from L2) and 128 KB of results. Each CTA holds half of W_h, K's rows in the first
// and V's in the second, so W crosses from L2 once per 256 tokens. With a product per CTA (128 tokens) it crosses twice as often: 64 bytes
// a cycle into each SM, and 76K tokens x 32 heads took 579 us, 393 of them without the stores of the results.
// A pair walks a run of units, heads innermost: a tile's latents (8 blocks of 64 columns) stay in shared memory over its heads, W
// streams through a ring of 16 KB blocks, and each block of the next tile is fetched as soon as the last head's product has
// passed it. Two accumulators of 256 columns fill tensor memory, so the products of one unit run while the results of the last
// are stored: a thread turns 64 columns of a token's row into bf16, a warp lays the halves of its two pages out in shared memory, and
// each goes out as one box (a page that is only partly wanted, by plain stores). With plain stores of 32 bytes a thread throughout
// the same work took 474 us, 358 of them without any stores.
// The first CTA issues the products; the copies of both complete on its barriers.
#include "pd_decode_plan.cuh"
#include "pd_kernels.cuh"
#include "pd_ptx.cuh"
#include "pd_tcgen05.cuh"

namespace pd {

namespace {

constexpr int kTile = 128, kTilePages = kTile / kPageSize;
constexpr int kCols = 2 * kLatentHead;           // K and V of a head
constexpr int kChunks = kLatentDim / 64;
constexpr int kABytes = kTile * 128;             // 64 columns of the tile
constexpr int kBBytes = kLatentHead * 128;       // 64 columns of a CTA's half of W_h
constexpr int kStages = 4;
constexpr int kStoreWarps = 8;                   // four for K, four for V
constexpr int kThreads = 32 * kStoreWarps + 64;  // + TMA warp + MMA warp (idle in the second CTA)
constexpr int kTmemCols = 512;
constexpr int kStageBytes = 32 * 128;            // of a store warp: 64 columns of its 32 tokens
constexpr int kNumBars = 2 * kChunks + 2 * kStages + 4 + 1;
constexpr size_t kSmemBytes = 1024 + kChunks * kABytes + kStages * kBBytes + kStoreWarps * kStageBytes + kNumBars * 8;

// The tokens of a sequence that are wanted, and the tiles they take: from the page of the first one on.
struct Span {
    int first, len, page0, tiles;
};
__device__ __forceinline__ Span span_of(const LatentExpandParams &p, int b) {
    Span s;
    s.first = p.first_token != nullptr ? __ldg(p.first_token + b) : 0;
    s.len = __ldg(p.ctx_lens + b);
    if (s.first < 0 || s.len < 0 || s.len > p.MP * kPageSize || s.first >= s.len) s.first = s.len = 0;
    s.page0 = s.first / kPageSize;
    s.tiles = (s.len - s.page0 * kPageSize + kTile - 1) / kTile;
    return s;
}

// Where a CTA stands: its tile (none behind the last one) and the head.
struct Walk {
    int b, tile, head;
    Span s;
};
__device__ __forceinline__ void next_tile(Walk &w, const LatentExpandParams &p) {
    if (w.b >= p.B || ++w.tile < w.s.tiles) return;
    w.tile = 0;
    do {
        w.s.first = w.s.len = w.s.page0 = w.s.tiles = 0;
        if (++w.b >= p.B) return;
        w.s = span_of(p, w.b);
    } while (w.s.tiles == 0);
}
__device__ __forceinline__ void step(Walk &w, const LatentExpandParams &p) {
    if (++w.head < p.Hq) return;
    w.head = 0;
    next_tile(w, p);  // the pair's other tile
    next_tile(w, p);
}

__global__ void __launch_bounds__(kThreads, 1)
kv_expand_latent_kernel(const __grid_constant__ CUtensorMap tm_kv, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_k,
                        const __grid_constant__ CUtensorMap tm_v, const LatentExpandParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ int32_t warp_sums[kThreads / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *aligned = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t a_s = base, b_ring = base + kChunks * kABytes, stage_s = b_ring + kStages * kBBytes;
    const uint32_t bar_a = stage_s + kStoreWarps * kStageBytes, bar_afree = bar_a + kChunks * 8;
    const uint32_t bar_b = bar_afree + kChunks * 8, bar_bfree = bar_b + kStages * 8;
    const uint32_t bar_d = bar_bfree + kStages * 8, bar_dfree = bar_d + 16, bar_drain = bar_dfree + 16;
    const uint32_t rank = cluster_rank(), pairs = gridDim.x / 2, pair = blockIdx.x / 2;
    if (tid == 0) {
        for (int i = 0; i < kNumBars; ++i) mbar_init(bar_a + i * 8, bar_a + i * 8 == bar_dfree || bar_a + i * 8 == bar_dfree + 8 ? 2 * kStoreWarps : 1);
        mbar_init_fence();
        prefetch_tensormap(&tm_kv);
        prefetch_tensormap(&tm_w);
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
    }
    if (warp == 0) {
        tmem_alloc_pair(smem_u32(&tmem_slot), kTmemCols);
        tmem_relinquish_alloc_permit_pair();
    }
    grid_dependency_wait();
    launch_dependents();

    // ---- prefix sums of the tiles, in memory that no copy uses yet
    int32_t *cum = reinterpret_cast<int32_t *>(aligned);
    {
        const int items = (p.B + kThreads - 1) / kThreads, begin = min(p.B, tid * items), end = min(p.B, begin + items);
        int sum = 0;
        for (int i = begin; i < end; ++i) {
            const int len = __ldg(p.ctx_lens + i), first = p.first_token != nullptr ? __ldg(p.first_token + i) : 0;
            if (blockIdx.x == 0 && (len < 0 || len > p.MP * kPageSize || first < 0)) latch_status(p.status, kDevBadLength, i, first < 0 ? first : len);
            const int tiles = span_of(p, i).tiles;
            cum[i] = tiles;
            sum += tiles;
        }
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        if (lane == 31) warp_sums[warp] = incl;
        __syncthreads();
        int run = incl - sum;
        for (int w = 0; w < warp; ++w) run += warp_sums[w];
        for (int i = begin; i < end; ++i) {
            const int tiles = cum[i];
            cum[i] = run;
            run += tiles;
        }
        if (tid == kThreads - 1) cum[p.B] = run;
        __syncthreads();
    }
    const int n_tiles = cum[p.B];
    const long long total = static_cast<long long>((n_tiles + 1) / 2) * p.Hq;
    const long long u0 = total * pair / pairs;
    const int units = static_cast<int>(total * (pair + 1) / pairs - u0);
    Walk w{};
    if (units > 0) {
        const long long tile_pair = div_positive(u0, p.Hq);
        const int tile = static_cast<int>(2 * tile_pair) + static_cast<int>(rank);
        w.head = static_cast<int>(u0 - tile_pair * p.Hq);
        w.b = p.B;
        if (tile < n_tiles) {
            const Cursor c = locate(cum, p.B, 1, tile);
            w.b = c.b;
            w.tile = c.page;
            w.s = span_of(p, c.b);
        }
    }
    fence_proxy_async();  // the copies that follow overwrite what was read here
    tc_fence_before_sync();
    cluster_sync();  // (the other CTA's barriers are initialised too)
    tc_fence_after_sync();
    const uint32_t tm = tmem_slot;
    bool ok = true;

    if (units > 0 && warp == kStoreWarps) {
        // ================= TMA warp: one elected thread =================
        if (elect_one()) {
            const uint64_t policy = l2_policy_evict_first(), keep = l2_policy_evict_last();
            const int32_t oob_row = p.num_pages * kPageSize;  // a box that starts here is all zero fill
            const uint32_t a_full = cluster_address(bar_a, 0), b_full = cluster_address(bar_b, 0);
            int ac = 0, bc = 0;  // blocks of latents and of W issued
            for (int u = 0; u < units && ok; ++u) {
                const bool new_tile = u == 0 || w.head == 0;
                int32_t y[kTilePages];
                if (new_tile) {
#pragma unroll
                    for (int g = 0; g < kTilePages; ++g) {
                        const int page = w.s.page0 + w.tile * kTilePages + g;
                        const int pid = w.b < p.B && page * kPageSize < w.s.len ? __ldg(p.page_table + static_cast<size_t>(w.b) * p.MP + page) : -1;
                        y[g] = pid >= 0 && pid < p.num_pages ? pid * kPageSize : oob_row;  // (the store warps latch bad ids)
                    }
                }
                for (int c = 0; c < kChunks && ok; ++c) {
                    if (new_tile) {
                        if (ac >= kChunks) ok = mbar_wait(bar_afree + c * 8, (ac / kChunks - 1) & 1);
                        if (!ok) break;
                        if (rank == 0) mbar_arrive_expect_tx(bar_a + c * 8, 2 * kABytes);
#pragma unroll
                        for (int g = 0; g < kTilePages; ++g)
                            tma_load_2d_pair(a_s + c * kABytes + g * (kPageSize * 128), &tm_kv, c * 64, y[g], a_full + c * 8, policy);
                        ++ac;
                    }
                    const int slot = bc % kStages, fill = bc / kStages;
                    if (fill > 0) ok = mbar_wait(bar_bfree + slot * 8, (fill - 1) & 1);
                    if (!ok) break;
                    if (rank == 0) mbar_arrive_expect_tx(bar_b + slot * 8, 2 * kBBytes);
                    tma_load_2d_pair(b_ring + slot * kBBytes, &tm_w, c * 64, w.head * kCols + static_cast<int>(rank) * kLatentHead, b_full + slot * 8, keep);
                    ++bc;
                }
                step(w, p);
            }
            if (!ok) {
                latch_status(p.status, kDevTimeout, w.b, blockIdx.x);
                if (rank == 0) {  // copies in flight, the other CTA's among them, have to land before the pair's memory goes
                    for (int i = max(0, bc - kStages); i < bc; ++i) mbar_wait(bar_b + (i % kStages) * 8, (i / kStages) & 1);
                    for (int i = max(0, ac - kChunks); i < ac; ++i) mbar_wait(bar_a + (i % kChunks) * 8, (i / kChunks) & 1);
                }
            }
        }
    } else if (units > 0 && warp == kStoreWarps + 1 && rank == 0) {
        // ================= MMA warp of the first CTA: one elected thread =================
        if (elect_one()) {
            constexpr uint32_t idesc = umma_idesc_bf16(2 * kTile, kCols, false);
            const uint64_t a_desc = umma_smem_desc(a_s, 16, 1024), b_desc = umma_smem_desc(b_ring, 16, 1024);
            int tiles = 0, bc = 0;
            for (int u = 0; u < units && ok; ++u) {
                const bool new_tile = u == 0 || w.head == 0, last_head = u == units - 1 || w.head == p.Hq - 1;
                if (new_tile) ++tiles;
                if (u >= 2) ok = mbar_wait_cluster(bar_dfree + (u & 1) * 8, ((u >> 1) - 1) & 1);
                const uint32_t d = tm + (u & 1) * kCols;
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const int slot = bc % kStages;
                    if (new_tile) ok = ok && mbar_wait_cluster(bar_a + c * 8, (tiles - 1) & 1);
                    ok = ok && mbar_wait_cluster(bar_b + slot * 8, (bc / kStages) & 1);
                    if (!ok) break;
                    tc_fence_after_sync();
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        umma_ss_pair(d, a_desc + (c * kABytes >> 4) + ks * 2, b_desc + slot * (kBBytes >> 4) + ks * 2, idesc, (c | ks) != 0);
                    umma_commit_pair(bar_bfree + slot * 8);
                    if (last_head) umma_commit_pair(bar_afree + c * 8);
                    ++bc;
                }
                if (!ok) break;
                umma_commit_pair(bar_d + (u & 1) * 8);
                step(w, p);
            }
            if (!ok) latch_status(p.status, kDevTimeout, w.b, blockIdx.x);
            umma_commit_pair(bar_drain);  // nothing may be in flight when the tensor memory is freed
            mbar_wait(bar_drain, 0);
        }
    } else if (units > 0 && warp < kStoreWarps) {
        // ================= store warps: thread = token of the tile, K (first four warps) or V =================
        const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const int half = warp >> 2, row = tid & (kTile - 1);
        const uint32_t dfree = cluster_address(bar_dfree, 0), stage = stage_s + warp * kStageBytes;
        __nv_bfloat16 *pool = half == 0 ? p.k_pages : p.v_pages;
        int to = -1;             // this token's page of the expanded pool, if it is to be written
        uint32_t whole = 0;      // bit g: all 16 tokens of the warp's page g are
        for (int u = 0; u < units && ok; ++u) {
            if (u == 0 || w.head == 0) {
                const int tok = (w.s.page0 + w.tile * kTilePages) * kPageSize + row, page = tok / kPageSize;
                to = -1;
                if (w.b < p.B && tok >= w.s.first && tok < w.s.len) {
                    const int from = __ldg(p.page_table + static_cast<size_t>(w.b) * p.MP + page);
                    to = __ldg(p.dst_table + static_cast<size_t>(w.b) * p.MP + page);
                    if (from < 0 || from >= p.num_pages || to < 0 || to >= p.dst_num_pages) {
                        latch_status(p.status, kDevBadPage, w.b, from < 0 || from >= p.num_pages ? from : to);
                        to = -1;
                    }
                }
                const uint32_t valid = __ballot_sync(0xffffffffu, to >= 0);
                whole = ((valid & 0xffffu) == 0xffffu ? 1u : 0u) | ((valid >> 16) == 0xffffu ? 2u : 0u);
            }
            ok = __all_sync(0xffffffffu, mbar_wait(bar_d + (u & 1) * 8, (u >> 1) & 1));
            if (!ok) break;
            tc_fence_after_sync();
            const int at = (to * p.Hq + w.head) * kPageSize;  // first row of this token's page and head
#pragma unroll
            for (int c = 0; c < 2; ++c) {  // 64 columns at a time
                uint32_t o[2][32], v[4][8];
                const uint32_t src = tm + lane_base + (u & 1) * kCols + half * kLatentHead + c * 64;
                tmem_ld32(src, o[0]);
                tmem_ld32(src + 32, o[1]);
                tmem_wait_ld();
                if (c == 1) {  // the accumulator has been read
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_relaxed(dfree + (u & 1) * 8);
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i >> 3][i & 7] = pack_bf16x2(__uint_as_float(o[i >> 4][2 * (i & 15)]), __uint_as_float(o[i >> 4][2 * (i & 15) + 1]));
                if (lane == 0) bulk_wait_group_read<0>();  // the staging is free
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(stage + sw128_offset(lane, i)), "r"(v[i >> 1][4 * (i & 1)]),
                                 "r"(v[i >> 1][4 * (i & 1) + 1]), "r"(v[i >> 1][4 * (i & 1) + 2]), "r"(v[i >> 1][4 * (i & 1) + 3]) : "memory");
                fence_proxy_async();
                __syncwarp();
                const int at1 = __shfl_sync(0xffffffffu, at, 16);
                if (lane == 0) {
                    const CUtensorMap *map = half == 0 ? &tm_k : &tm_v;
                    if (whole & 1u) tma_store_2d(map, c * 64, at, stage);
                    if (whole & 2u) tma_store_2d(map, c * 64, at1, stage + kPageSize * 128);
                    bulk_commit_group();
                }
                if (to >= 0 && !((whole >> (lane >> 4)) & 1u)) {
                    __nv_bfloat16 *dst = pool + (static_cast<size_t>(at) + row % kPageSize) * kLatentHead + c * 64;
#pragma unroll
                    for (int i = 0; i < 4; ++i) store32(dst + i * 16, v[i]);
                }
            }
            step(w, p);
        }
        if (lane == 0) bulk_wait_all();
        if (!ok && lane == 0) latch_status(p.status, kDevTimeout, w.b, blockIdx.x);
    }
    __syncwarp();
    tc_fence_before_sync();
    cluster_sync();  // neither CTA leaves while the other may still use its memory and barriers
    if (warp == 0) tmem_dealloc_pair(tm, kTmemCols);
}

}  // namespace

// The pairs that fit the device at once (a cluster needs two free SMs of one GPC); the launch is that many.
cudaError_t prepare_kv_expand_latent(int num_sms, int *num_pairs) {
    cudaError_t e = cudaFuncSetAttribute(kv_expand_latent_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmemBytes));
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(num_sms / 2 * 2);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemBytes;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(num_pairs, kv_expand_latent_kernel, &cfg);
    if (e == cudaSuccess && *num_pairs < 1) e = cudaErrorInvalidConfiguration;
    if (e == cudaSuccess && *num_pairs > num_sms / 2) *num_pairs = num_sms / 2;
    return e;
}

cudaError_t launch_kv_expand_latent(const CUtensorMap &tm_kv, const CUtensorMap &tm_w, const CUtensorMap &tm_k, const CUtensorMap &tm_v,
                                    const LatentExpandParams &p, int num_pairs, cudaStream_t stream) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(2 * num_pairs);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemBytes;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = p.pdl != 0 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kv_expand_latent_kernel, tm_kv, tm_w, tm_k, tm_v, p);
}

}  // namespace pd
