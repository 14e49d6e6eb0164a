// Append-prefill attention in the expanded form of a cache of shared latent vectors: queries of 192 values, 128 against the
// head's own expanded keys, 64 against the rotated key part all heads share; values of 128.
//
// An item of work is two tiles of 128 query rows (256 consecutive new tokens of one head) that share every K and V tile, as in
// pd_prefill_attn_d128.cu. One CTA per SM takes items from a counter and walks each one's context in blocks of 80 tokens (5 pages):
//   tcgen05  S_t = Q_t K^T (12 MMAs of 128 x 80 x 16, Q and K from shared memory), O_t += P_t V (5 of 128 x 128 x 16, P_t from
//            tensor memory), in the order S0(j+1) O0(j) S1(j+1) O1(j)
//   softmax  one warpgroup per tile, one thread per row
// Why 80: tensor memory has 128 columns a tile beside its 128 of O. With blocks of 128 P has to lie where S lay, so S(j+1) waits
// for the softmax of block j, for its O product and for four hand-overs: 3630 cycles per 128 tokens (both tiles), where the
// products take 2560. With 80 columns of S and 40 of P beside them, S(j+1) waits only until the row threads hold the logits of
// block j in registers, and runs during their softmax. What bounds it now is shared memory: an S product reads 4 KB of Q and
// 2.5 KB of K in 51 cycles (128 bytes each), 1864 cycles a block with O, and the copies write 50 KB (400 cycles) beside that;
// a block takes 2200. Eight turns, 9.6K new tokens on contexts of up to 18K, 32 heads: 1.79 to 1.87 ms, 1.18 to 1.23 PFLOP/s; 2.14 ms under
// sustained load, where the power limit lowers the clock.
// Probabilities are rounded to bf16, as tcgen05 takes its 16-bit operands (off by at most 2^-8 of themselves); their sum is taken before.
// Dividing by the sum of the rounded ones instead would take 1 % off the error (0.00224 from 0.00226, root of the mean squares) and costs 120
// instructions a row and block behind the stores of P: 37.3 from 34.2 us on nine odd turns, 2250 from 2130 on eight long ones.
// A page's 128 columns come as one box in the order [8-row group][64-column half][8 rows]: row groups follow one another
// at the same distance across pages, as both operand forms want it.
// Each tile has its own number of blocks: the first skips those that only the second one sees, and a turn of at most 128 tokens
// runs one tile. Tensor memory: (S0 80, P0 40) (S1, P1) O0 O1, 128 columns each. Every wait is bounded.
// Why a counter and not a block per item: the grid would have to be as wide as the longest turn for every sequence, and the next
// item's queries, keys and values come in during the last one's softmax and stores. Two turns of 2048 among 62 single tokens, 32
// heads: 233 us, 329 with a block per item; nine odd turns 34.0 from 36.6. The few more instructions of the walk cost long
// turns 2 %.
// Few tokens on a long context are few items: then an item is a stretch of the context, its unnormalised outputs go to the workspace in
// fp32, and the warp that counts the last stretch of its 32 rows joins them in their order (the same bits in every call). 128 tokens on
// 8000, 32 heads: 43 us, 95 whole; 512 on 30000, 8 heads: 91 and 464.
#include "pd_kernels.cuh"
#include "pd_ptx.cuh"
#include "pd_tcgen05.cuh"

#include <cfloat>

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
constexpr int kThreads = 32 * (kSoftmaxWarps + 4);  // + MMA warp, K loader, V loader, the warp that hands out items
constexpr int kTmemCols = 512;
constexpr int kColS = 0, kColP = kBlock, kColO = 256;  // S_t, P_t at 128 t + .., O_t at kColO + 128 t
// Registers per thread: the softmax keeps a row's 80 logits and 40 packed weights, which do not fit the launch's 168 without spills.
// 128 * 104 + 256 * 200 = 384 * 168.
constexpr int kOtherRegs = 104, kSoftmaxRegs = 200;
constexpr int kItemSlots = 4;
constexpr int kNumBars = 2 * kKSlots + 2 * kVSlots + 6 * kTiles + 2 + 2 * kItemSlots;
constexpr int kItemReaders = kSoftmaxWarps + 3;
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

// Natural logarithm of sum * 2^(reference * scale).
__device__ __forceinline__ float log_sum(float reference, float sum, float scale_log2) {
    return fmaf(reference, scale_log2 * kLn2f, log2f(sum) * kLn2f);
}

// Every item starts the rings at slot 0. Bit s: whether its nb blocks fill slot s an odd number of times.
template <int SLOTS>
__device__ __forceinline__ uint32_t fills(int nb) {
    uint32_t mask = 0;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) mask |= static_cast<uint32_t>((nb - s + SLOTS - 1) / SLOTS & 1) << s;
    return mask;
}

// Two tiles of one head over a stretch of their context.
struct Item {
    int row0, n_tok, pos0, len;  // first packed row, rows (0: no more items), position of the first one, tokens of the context
    int b, head, nb0, nb1;       // blocks of each tile in the stretch, as far as its last token sees
    int j0, parts, part, first;  // first block; stretches of these tiles, the partial result this one writes, the first one's
};
// A partial result: per tile [column / 4][row][4] unnormalised outputs, then [row] (reference, sum).
constexpr int kPartTile = kRows * kLatentHead;
constexpr size_t kPartFloats = kTiles * (kPartTile + 2 * kRows);
static_assert(kPartFloats * sizeof(float) == kLatentPrefillPartBytes, "the workspace is sized by it");

// SPLITS: contexts may be cut. A kernel of its own, as the code of that costs every item 0.4 us.
template <bool SPLITS>
__global__ void __launch_bounds__(kThreads, 1)
prefill_attn_latent_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                           const __grid_constant__ CUtensorMap tm_r, const LatentPrefillParams lp) {
    const PrefillParams &p = lp.a;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ Item items[kItemSlots];
    __shared__ int32_t arrived_set;  // where this call counts stretches
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int kItemTok = kTiles * kRows;

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_s = base, k_ring = q_s + kTiles * kQTileBytes, r_ring = k_ring + kKSlots * kKvBytes;
    const uint32_t v_ring = r_ring + kKSlots * kRopeBytes;
    const uint32_t bar_k = v_ring + kVSlots * kKvBytes, bar_kfree = bar_k + kKSlots * 8;  // K and rotated part landed / are free again
    const uint32_t bar_v = bar_kfree + kKSlots * 8, bar_vfree = bar_v + kVSlots * 8;
    const uint32_t bar_s = bar_vfree + kVSlots * 8;  // [2] S_t of the block complete
    const uint32_t bar_o = bar_s + kTiles * 8;       // [2] O_t product of the block complete
    const uint32_t bar_drain = bar_o + kTiles * 8;
    const uint32_t bar_claim = bar_drain + 8;        // the item's last keys are on their way: time to claim another
    const uint32_t bar_item = bar_claim + 8;         // [4] an item stands in its slot
    // from 4 warps each:
    const uint32_t bar_sfree = bar_item + kItemSlots * 8;  // [2] the rows hold S_t of the block in registers
    const uint32_t bar_p = bar_sfree + kTiles * 8;   // [2] P_t is written
    const uint32_t bar_q = bar_p + kTiles * 8;       // [2] tile t's queries of the item are in shared memory
    const uint32_t bar_done = bar_q + kTiles * 8;    // [2] the rows have read O_t of the item
    const uint32_t bar_taken = bar_done + kTiles * 8;  // [4] every reader is done with the item of that slot

    if (tid == 0) {
        for (int i = 0; i < kNumBars; ++i) {
            const uint32_t bar = bar_k + i * 8;
            mbar_init(bar, bar >= bar_taken ? kItemReaders : bar >= bar_sfree ? kRows / 32 : 1);
        }
        mbar_init_fence();
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
        prefetch_tensormap(&tm_r);
    }
    grid_dependency_wait();  // before the allocation: a predecessor's blocks may still be waiting for theirs
    if (warp == 0) {
        tmem_alloc(smem_u32(&tmem_slot), kTmemCols);
        tmem_relinquish_alloc_permit();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tm = tmem_slot;
    launch_dependents();
    bool ok = true;

    int taken = 0;  // items this thread has come to
    // The slot of the next item; the item behind the last one has no rows.
    auto next_item = [&]() -> const Item & {
        const int slot = taken % kItemSlots;
        ok = ok && mbar_wait(bar_item + slot * 8, (taken / kItemSlots) & 1);
        ++taken;
        return items[slot];
    };
    // ... copied, and its slot handed back, by a single thread
    auto take_item = [&](Item &it) {
        const Item &next = next_item();
        if (!ok) return false;
        it = next;
        mbar_arrive(bar_taken + (taken - 1) % kItemSlots * 8);
        return it.n_tok > 0;
    };

    if (warp >= kSoftmaxWarps) {
        setmaxnreg_dec<kOtherRegs>();
        if (warp == kSoftmaxWarps + 3) {
            // ================= hands out items: sequences by falling work, one head after the other, last tokens first =================
            // Lanes hold 32 sequences at a time and count their items up. Up to 32 are ranked here, more by a small kernel before.
            int b = 0, from = 0, n = 0, L = 0, per_head = 0, count = 0, incl = 0, chunk = 0;  // chunk: most blocks of a stretch, 0: any
            // blocks the two tiles from token `start` of a sequence's m new ones see, and the stretches they are cut into
            auto blocks_of = [&](int m, int len, int start) { return (len - m + min(start + kItemTok, m) - 1) / kBlock + 1; };
            auto parts_of = [&](int nb, int c) { return static_cast<int>((static_cast<float>(nb + c) - 0.5f) * (1.f / static_cast<float>(c))); };
            auto pieces_of = [&](int c) {
                int sum = 0;
                for (int start = 0; start < n; start += kItemTok) sum += parts_of(blocks_of(n, L, start), c);
                return sum;
            };
            auto window = [&](int w) {
                const int z = w * 32 + lane;
                if (p.order == nullptr) {
                    const int mine = min(lane, p.B - 1);
                    const int f = p.q_indptr[mine], m = p.q_indptr[mine + 1] - f, l = p.ctx_lens[mine];
                    const long long work = static_cast<long long>(m) * (2ll * l - m);
                    int rank = 0, src = 0;
                    for (int i = 0; i < p.B; ++i) {
                        const long long x = __shfl_sync(0xffffffffu, work, i);
                        rank += x > work || (x == work && i < lane) ? 1 : 0;
                    }
                    for (int i = 0; i < p.B; ++i)
                        if (__shfl_sync(0xffffffffu, rank, i) == lane) src = i;
                    b = src;
                    from = __shfl_sync(0xffffffffu, f, src);
                    n = __shfl_sync(0xffffffffu, m, src);
                    L = __shfl_sync(0xffffffffu, l, src);
                } else if (z < p.B) {
                    b = p.order[z];
                    from = p.q_indptr[b];
                    n = p.q_indptr[b + 1] - from;
                    L = p.ctx_lens[b];
                }
                const bool real = z < p.B && n > 0, fits = L >= n && L <= p.MP * kPageSize;  // the cache must hold the new tokens
                if (real && !fits && blockIdx.x == 0) latch(p.status, kDevBadLength, b, L);
                if (!real || !fits) n = L = 0;
                if (SPLITS) {
                    // Few items: a context is cut where whole ones would leave SMs idle. In blocks of 1.0 to 1.5 us: a stretch costs about 4
                    // more, joining one about 1, and where there are more stretches than SMs the last ones end half a stretch late.
                    int sum = 0, longest = 0;
                    for (int start = 0; start < n; start += kItemTok) {
                        const int nb = blocks_of(n, L, start);
                        sum += nb;
                        longest = max(longest, nb);
                    }
                    longest = __reduce_max_sync(0xffffffffu, longest);
                    if (longest >= 16) {
                        const int sms = lp.num_sms, fair = (__reduce_add_sync(0xffffffffu, sum) * p.Hq + sms - 1) / sms;
                        const int whole = __reduce_add_sync(0xffffffffu, (n + kItemTok - 1) / kItemTok) * p.Hq;
                        int best = whole <= sms ? longest : max(longest, fair + longest / 2);
                        for (int c = max(fair, 8); c < longest; c += (c + 3) / 4) {
                            const int pieces = __reduce_add_sync(0xffffffffu, pieces_of(c)) * p.Hq;
                            const int est = max(c, pieces <= sms ? 0 : fair + c / 2 + 4) + 4 + longest / c;
                            if (pieces <= lp.max_parts && est < best) best = est, chunk = c;
                            if (c > best) break;
                        }
                    }
                }
                per_head = !SPLITS || chunk == 0 ? (n + kItemTok - 1) / kItemTok : pieces_of(chunk);
                count = per_head * p.Hq;
                incl = count;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int x = __shfl_up_sync(0xffffffffu, incl, o);
                    if (lane >= o) incl += x;
                }
            };
            const int groups = lp.max_parts * kSoftmaxWarps;
            const int calls = SPLITS ? __ldcg(lp.arrived + 2 * groups) : 0;
            int idx = blockIdx.x, before = 0, w = 0;
            window(0);
            if (SPLITS) {
                const int set = calls & 1;
                for (int i = blockIdx.x * 32 + lane; i < groups; i += gridDim.x * 32) lp.arrived[(set ^ 1) * groups + i] = 0;
                if (lane == 0) arrived_set = set * groups;  // (read behind the first item)
            }
            for (int k = 0; ok; ++k) {
                while (w * 32 < p.B && idx >= before + __shfl_sync(0xffffffffu, incl, 31)) {
                    before += __shfl_sync(0xffffffffu, incl, 31);
                    if (++w * 32 < p.B) window(w);
                }
                Item it{};
                const bool more = w * 32 < p.B;
                if (more) {
                    const int src = __ffs(__ballot_sync(0xffffffffu, idx - before < incl)) - 1;
                    const int rel = idx - before - __shfl_sync(0xffffffffu, incl - count, src);
                    const int q_len = __shfl_sync(0xffffffffu, n, src);
                    it.b = __shfl_sync(0xffffffffu, b, src);
                    it.len = __shfl_sync(0xffffffffu, L, src);
                    int left, start = (q_len - 1) / kItemTok * kItemTok, parts = 1, nb;
                    if (!SPLITS || chunk == 0) {  // the tiles of one head after those of another: they read the same keys and values
                        const int tiles = __shfl_sync(0xffffffffu, per_head, src);
                        it.head = rel / tiles;
                        start -= (rel - it.head * tiles) * kItemTok;
                        left = 0;
                        nb = blocks_of(q_len, it.len, start);
                    } else {  // the longest contexts of all heads first
                        left = rel / p.Hq;
                        it.head = rel - left * p.Hq;
                        for (;; start -= kItemTok) {
                            nb = blocks_of(q_len, it.len, start);
                            parts = parts_of(nb, chunk);
                            if (left < parts || start == 0) break;
                            left -= parts;
                        }
                    }
                    const int size = parts == 1 ? nb : (nb + parts - 1) / parts;
                    it.row0 = __shfl_sync(0xffffffffu, from, src) + start;
                    it.n_tok = min(kItemTok, q_len - start);
                    it.pos0 = it.len - q_len + start;
                    if (SPLITS) it.j0 = left * size, it.parts = parts, it.part = idx, it.first = idx - left * p.Hq;
                    it.nb0 = min(max((it.pos0 + min(it.n_tok, kRows) - 1) / kBlock + 1 - left * size, 0), size);
                    it.nb1 = it.n_tok > kRows ? min(max(nb - left * size, 0), size) : 0;
                }
                if (k >= kItemSlots)
                    ok = __all_sync(0xffffffffu, mbar_wait(bar_taken + k % kItemSlots * 8, (k / kItemSlots - 1) & 1));
                if (!ok) break;
                if (lane == 0) {
                    items[k % kItemSlots] = it;
                    mbar_arrive(bar_item + k % kItemSlots * 8);
                }
                if (!more) break;
                ok = __all_sync(0xffffffffu, mbar_wait(bar_claim, k & 1));  // no earlier: claims far ahead leave idle blocks nothing
                int claim = 0;
                if (ok && lane == 0) claim = atomicAdd(p.status + kSchedNext, 1);
                idx = static_cast<int>(gridDim.x) + __shfl_sync(0xffffffffu, claim, 0);
            }
            if (lane == 0) {  // the last block to stop claiming sets the counters back
                if (!ok) latch(p.status, kDevTimeout, -1, blockIdx.x);
                __threadfence();
                if (atomicAdd(p.status + kSchedDone, 1) == static_cast<int>(gridDim.x) - 1) {
                    p.status[kSchedNext] = 0;
                    p.status[kSchedDone] = 0;
                    if (SPLITS) lp.arrived[2 * groups] = calls + 1;  // (every block has read it)
                }
            }
        } else if (warp == kSoftmaxWarps) {
            // ================= MMA warp: one elected thread issues every product =================
            if (elect_one()) {
                constexpr uint32_t idesc_s = umma_idesc_bf16(kRows, kBlock, false);
                constexpr uint32_t idesc_o = umma_idesc_bf16(kRows, kLatentHead, true);
                const uint64_t q_desc = umma_smem_desc(q_s, 16, 1024), k_desc = umma_smem_desc(k_ring, 16, 2048);
                const uint64_t r_desc = umma_smem_desc(r_ring, 16, 1024), v_desc = umma_smem_desc(v_ring, 1024, 2048);
                uint32_t k_mask = 0, v_mask = 0;                           // parity of each slot's fills by earlier items
                uint32_t done[kTiles] = {0, 0}, turns[kTiles] = {0, 0};  // parity of each tile's blocks and items so far
                auto issue_s = [&](int t, int j, bool wait, bool release) {  // S_t(j) = Q_t K_j^T
                    const int slot = j % kKSlots;
                    const uint32_t parity = (k_mask >> slot ^ j / kKSlots) & 1;
                    const uint32_t d = tm + kColS + t * 128;
                    const uint64_t q = q_desc + (t * kQTileBytes >> 4);
                    ok = ok && mbar_wait(bar_sfree + t * 8, (done[t] ^ j ^ 1) & 1);  // passes at once before the first block
                    if (wait) ok = ok && mbar_wait(bar_k + slot * 8, parity);
                    if (!ok) return;
                    tc_fence_after_sync();
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            umma_ss(d, q + (c * kQPiece >> 4) + ks * 2, k_desc + slot * (kKvBytes >> 4) + c * (1024 >> 4) + ks * 2, idesc_s,
                                    (c | ks) != 0);
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        umma_ss(d, q + (2 * kQPiece >> 4) + ks * 2, r_desc + slot * (kRopeBytes >> 4) + ks * 2, idesc_s, true);
                    if (release) umma_commit(bar_kfree + slot * 8);
                    umma_commit(bar_s + t * 8);
                };
                auto issue_o = [&](int t, int j, bool wait, bool release) {  // O_t += P_t(j) V_j
                    const int slot = j % kVSlots;
                    ok = ok && mbar_wait(bar_p + t * 8, (done[t] ^ j) & 1);
                    if (wait) ok = ok && mbar_wait(bar_v + slot * 8, (v_mask >> slot ^ j / kVSlots) & 1);
                    if (!ok) return;
                    tc_fence_after_sync();
#pragma unroll
                    for (int ks = 0; ks < kBlock / 16; ++ks)
                        umma_ts(tm + kColO + t * kLatentHead, tm + t * 128 + kColP + ks * 8,
                                v_desc + slot * (kKvBytes >> 4) + ks * (4096 >> 4), idesc_o, (j | ks) != 0);
                    if (release) umma_commit(bar_vfree + slot * 8);
                    umma_commit(bar_o + t * 8);
                };
                Item it{};
                while (take_item(it)) {
                    const int nb0 = it.nb0, nb1 = it.nb1, nb = max(nb0, nb1);
                    const bool two = nb1 > 0, one = !SPLITS || nb0 > 0;  // the first tile may see nothing of a stretch
                    if (one) ok = mbar_wait(bar_q, turns[0] & 1);
                    if (ok && one) issue_s(0, 0, true, !two);
                    if (two) ok = ok && mbar_wait(bar_q + 8, turns[1] & 1);
                    if (ok && two) issue_s(1, 0, !one, true);
                    // the rows have read what the tiles' last items left in O
                    if (one) ok = ok && mbar_wait(bar_done, (turns[0] & 1) ^ 1);
                    if (two) ok = ok && mbar_wait(bar_done + 8, (turns[1] & 1) ^ 1);
                    // the tile that meets a block first waits for it, the one that meets it last hands it back
                    for (int j = 0; j < nb && ok; ++j) {
                        const bool u0 = j < nb0, u1 = j < nb1, n0 = j + 1 < nb0, n1 = j + 1 < nb1;
                        if (n0) issue_s(0, j + 1, true, !n1);
                        if (ok && u0) issue_o(0, j, true, !u1);
                        if (ok && n1) issue_s(1, j + 1, !n0, true);
                        if (ok && u1) issue_o(1, j, !u0, true);
                    }
                    if (!ok) break;
                    k_mask ^= fills<kKSlots>(nb), v_mask ^= fills<kVSlots>(nb);
                    if (one) done[0] ^= nb0 & 1, turns[0] ^= 1;
                    if (two) done[1] ^= nb1 & 1, turns[1] ^= 1;
                }
                if (!ok) latch(p.status, kDevTimeout, it.b, blockIdx.x);
                umma_commit(bar_drain);  // nothing may be in flight when the tensor memory is freed
                mbar_wait(bar_drain, 0);
            }
        } else if (warp == kSoftmaxWarps + 1 || warp == kSoftmaxWarps + 2) {
            // ================= two TMA warps (K and the rotated part, V), one elected thread each =================
            if (elect_one()) {
                const uint64_t policy = l2_policy_evict_first();
                const bool is_k = warp == kSoftmaxWarps + 1;
                const int slots = is_k ? kKSlots : kVSlots;
                uint32_t mask = 0;  // parity of each slot's fills
                int32_t kv_id[kBlockPages], r_id[kBlockPages];  // the next block's pages
                Item it{};
                while (take_item(it)) {
                    const int nb = max(it.nb0, it.nb1), j0 = SPLITS ? it.j0 : 0, n_pages = (it.len + kPageSize - 1) / kPageSize;
                    const int32_t *kv_row = lp.kv_table + static_cast<size_t>(it.b) * p.MP;
                    const int32_t *r_row = p.page_table + static_cast<size_t>(it.b) * p.MP;
                    auto load_ids = [&](int j) {
#pragma unroll
                        for (int g = 0; g < kBlockPages; ++g) {
                            const int page = (j0 + j) * kBlockPages + g;
                            kv_id[g] = page < n_pages ? __ldg(kv_row + page) : 0;
                            if (is_k) r_id[g] = page < n_pages ? __ldg(r_row + page) : 0;
                        }
                    };
                    auto checked = [&](int32_t pid, int page, int limit) {  // `limit`: a page past the pool is zero fill
                        if (page >= n_pages) return limit;
                        if (pid >= 0 && pid < limit) return pid;
                        latch(p.status, kDevBadPage, it.b, pid);
                        return 0;
                    };
                    load_ids(0);
                    for (int j = 0; j < nb && ok; ++j) {
                        int32_t kv_page[kBlockPages], r_page[kBlockPages];
#pragma unroll
                        for (int g = 0; g < kBlockPages; ++g) {
                            kv_page[g] = checked(kv_id[g], (j0 + j) * kBlockPages + g, lp.kv_num_pages);
                            r_page[g] = is_k ? checked(r_id[g], (j0 + j) * kBlockPages + g, p.num_pages) : 0;
                        }
                        if (j + 1 < nb) load_ids(j + 1);
                        if (is_k && j == max(nb - 2, 0)) mbar_arrive(bar_claim);
                        const int slot = j % slots;
                        const uint32_t full = (is_k ? bar_k : bar_v) + slot * 8, dst = (is_k ? k_ring : v_ring) + slot * kKvBytes;
                        ok = mbar_wait((is_k ? bar_kfree : bar_vfree) + slot * 8, (mask >> slot & 1) ^ 1);
                        if (!ok) break;
                        mbar_arrive_expect_tx(full, is_k ? kKvBytes + kRopeBytes : kKvBytes);
                        mask ^= 1u << slot;
#pragma unroll
                        for (int g = 0; g < kBlockPages; ++g)
                            tma_load_4d(dst + g * 4096, is_k ? &tm_k : &tm_v,
                                        (kv_page[g] * p.Hq + (kv_page[g] < lp.kv_num_pages ? it.head : 0)) * 2, full, policy);
                        if (is_k) {
#pragma unroll
                            for (int g = 0; g < kBlockPages; ++g)
                                tma_load_2d(r_ring + slot * kRopeBytes + g * (kPageSize * 128), &tm_r, kLatentDim,
                                            r_page[g] * kPageSize, full, policy);
                        }
                    }
                    if (!ok) break;
                }
                if (!ok) {  // copies in flight have to land before the block's memory goes
                    latch(p.status, kDevTimeout, it.b, blockIdx.x);
                    for (int i = 0; i < slots; ++i) mbar_wait((is_k ? bar_k : bar_v) + i * 8, (mask >> i & 1) ^ 1);
                }
            }
        }
    } else {
        setmaxnreg_inc<kSoftmaxRegs>();
        // ================= softmax warpgroups: warpgroup t owns tile t, one thread per query row =================
        const int t = tid / kRows, row = tid & (kRows - 1);
        const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_buf = tm + lane_base + kColS + t * 128, p_buf = tm + lane_base + kColP + t * 128;
        const uint32_t o_buf = tm + lane_base + kColO + t * kLatentHead;
        uint32_t v_mask = 0, done = 0;  // parity of the V slots' fills by earlier items; this tile's blocks so far
        // an item's queries: neighbouring threads copy neighbouring 16 bytes, all in flight at once
        auto copy_q = [&](const Item &it) {
            constexpr int kChunks = kQDim / 8;  // 128 rows x 24 pieces over 128 threads
            const int rows = min(kRows, it.n_tok - t * kRows);
            int first = row;
            asm volatile("" : "+r"(first));  // keeps the offsets below from being held in registers across items
            if (rows <= 0) return;
            const __nv_bfloat16 *src = p.q + (static_cast<size_t>(it.row0 + t * kRows) * p.Hq + it.head) * kQDim;
#pragma unroll
            for (int i = 0; i < kChunks; ++i) {
                const int x = i * kRows + first, r = x / kChunks, c = x - r * kChunks;
                const uint32_t a = q_s + t * kQTileBytes + (c >> 3) * kQPiece + sw128_offset(r, c & 7);
                // rows past the last are zeros
                cp_async16(a, src + static_cast<size_t>(min(r, rows - 1)) * p.Hq * kQDim + c * 8, r < rows ? 16 : 0);
            }
        };
        // A wait that runs out may do so in some lanes of a warp: those go on without waiting, since the others need them in what the warp does
        // together, until the warp decides as one at the item's end.
        const Item *it = &next_item(), *after = it;
        ok = __all_sync(0xffffffffu, ok);
        if (ok && it->n_tok > 0) copy_q(*it);
        while (ok && it->n_tok > 0) {
            const int my_nb = t == 0 ? it->nb0 : it->nb1;
            const int tok = t * kRows + row;                      // token index inside the item
            const int my_pos = it->pos0 + min(tok, it->n_tok - 1);  // padding rows mirror the last token
            cp_async_wait_all();
            if (my_nb > 0) {
                fence_proxy_async();  // written through the generic proxy, read by the tensor core through the async one
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_q + t * 8);
            }
            float m_run = 0.f, l_run = 0.f;
            const float2 sc2 = make_float2(p.scale_log2, p.scale_log2);
            for (int j = 0; j < my_nb; ++j, ++done) {
                ok = ok && mbar_wait(bar_s + t * 8, done & 1);
                tc_fence_after_sync();
                const int t0 = ((SPLITS ? it->j0 : 0) + j) * kBlock;
                const bool masked = t0 + kBlock - 1 > my_pos;  // the block reaches past this row's position
                // V rows past the context inside the last page may hold NaN; 0 * NaN is NaN, so the warpgroup whose products of
                // this block come first clears them
                if (j == my_nb - 1 && t0 + kBlock > it->len && (t == 0 || j >= it->nb0)) {
                    const int valid_rows = it->len - t0;
                    const int last = min(kBlock, (valid_rows + kPageSize - 1) / kPageSize * kPageSize);
                    const int slot = j % kVSlots;
                    ok = ok && mbar_wait(bar_v + slot * 8, (v_mask >> slot ^ j / kVSlots) & 1);  // it must have landed
                    for (int x = row; x < (last - valid_rows) * (kLatentHead / 8); x += kRows) {
                        const int r = valid_rows + x / (kLatentHead / 8), c = x % (kLatentHead / 8);
                        st_shared_zero16(v_ring + slot * kKvBytes + (r >> 3) * 2048 + (c >> 3) * 1024 + (r & 7) * 128 + (c & 7) * 16);
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
                // x = (s - m) * scale against the reference as it stands, P = 2^x and its sum at once, so that the special-function unit
                // starts with the first logits; the largest logit is looked at behind them. The difference comes first: s * scale - m with a
                // rounded m is off by 2^-24 of m, more than 2^x holds where logits are beyond 1e9 (1 % more time on long turns)
                auto weigh = [&]() {
                    const float2 nm2 = make_float2(-m_run, -m_run);
                    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    float2 a[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                    for (int c = 0; c < kBlock; c += 4) {
                        const float2 x = __fmul2_rn(__fadd2_rn(make_float2(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), nm2), sc2);
                        const float2 y = __fmul2_rn(__fadd2_rn(make_float2(__uint_as_float(v[c + 2]), __uint_as_float(v[c + 3])), nm2), sc2);
                        top[(c >> 2) & 1] = max3(top[(c >> 2) & 1], __uint_as_float(v[c]), __uint_as_float(v[c + 1]));
                        top[2 + ((c >> 2) & 1)] = max3(top[2 + ((c >> 2) & 1)], __uint_as_float(v[c + 2]), __uint_as_float(v[c + 3]));
                        const float2 e = make_float2(fast_exp2(x.x), fast_exp2(x.y)), f = make_float2(fast_exp2(y.x), fast_exp2(y.y));
                        a[0] = __fadd2_rn(a[0], e);
                        a[1] = __fadd2_rn(a[1], f);
                        pk[c >> 1] = pack_bf16x2(e.x, e.y);
                        pk[(c >> 1) + 1] = pack_bf16x2(f.x, f.y);
                    }
                    sum = (a[0].x + a[0].y) + (a[1].x + a[1].y);
                    return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                };
                if (__any_sync(0xffffffffu, masked)) {  // masked logits become -inf, their exponentials exact zeros
                    const int visible = my_pos - t0 + 1;
#pragma unroll
                    for (int c = 0; c < kBlock; ++c)
                        if (c >= visible) v[c] = 0xff800000u;
                }
                if (j == 0) {  // the reference: the row's largest logit of the block; where there is no finite one, below any that comes
                    float top = -INFINITY;
#pragma unroll
                    for (int c = 0; c < kBlock; c += 2) top = max3(top, __uint_as_float(v[c]), __uint_as_float(v[c + 1]));
                    m_run = fmaxf(top, -FLT_MAX);
                }
                const float top = weigh();
                if (__any_sync(0xffffffffu, (top - m_run) * p.scale_log2 > kRaise)) {
                    // rare: the row's reference rises to its largest logit, what it has accumulated is rescaled, and the block is weighed
                    // again (its x have lost to their rounding what the last reference was lower)
                    const float raised = (top - m_run) * p.scale_log2 > kRaise ? top : m_run, alpha = fast_exp2((m_run - raised) * p.scale_log2);
                    m_run = raised;
                    if (j > 0) {
                        ok = ok && mbar_wait(bar_o + t * 8, (done - 1) & 1);
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
                ok = ok && mbar_wait(bar_o + t * 8, (done & 1) ^ 1);  // P_t has been used by the last block's product
                tc_fence_after_sync();
                tmem_st16(p_buf, *reinterpret_cast<uint32_t(*)[16]>(pk));
                tmem_st16(p_buf + 16, *reinterpret_cast<uint32_t(*)[16]>(pk + 16));
                tmem_st8(p_buf + 32, *reinterpret_cast<uint32_t(*)[8]>(pk + 32));
                tmem_wait_st();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_p + t * 8);
            }
            after = &next_item();  // this item's last logits are in registers: the next one's queries may come
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            if (after->n_tok > 0) copy_q(*after);
            v_mask ^= fills<kVSlots>(max(it->nb0, it->nb1));

            // ---- O_t / l -> bf16 rows
            auto store_cols = [&](__nv_bfloat16 *to, const uint32_t (&o)[32], float inv, bool wide) {  // 32 columns of a row
#pragma unroll
                for (int i = 0; i < 32; i += 16) {
                    uint32_t w[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) w[k] = pack_bf16x2(__uint_as_float(o[i + 2 * k]) * inv, __uint_as_float(o[i + 2 * k + 1]) * inv);
                    if (wide) {
                        store32(to + i, w);
                    } else {
                        *reinterpret_cast<uint4 *>(to + i) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4 *>(to + i + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                }
            };
            auto o_read = [&]() {
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_done + t * 8);
            };
            if (my_nb > 0) {
                ok = __all_sync(0xffffffffu, mbar_wait(bar_o + t * 8, (done - 1) & 1));
                if (!ok) break;
                tc_fence_after_sync();
            }
            const bool row_valid = tok < it->n_tok, wide = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0;
            const size_t at = static_cast<size_t>(it->row0 + min(tok, it->n_tok - 1)) * p.Hq + it->head;
            __nv_bfloat16 *orow = p.out + at * kLatentHead;
            if (!SPLITS || it->parts == 1) {
                if (my_nb > 0) {
                    const float inv = l_run == 0.f ? 0.f : 1.f / l_run;  // 0: the row sees nothing but -inf
#pragma unroll
                    for (int c = 0; c < kLatentHead; c += 32) {
                        uint32_t o[32];
                        tmem_ld32(o_buf + c, o);
                        tmem_wait_ld();
                        if (c == kLatentHead - 32) o_read();
                        if (row_valid) store_cols(orow + c, o, inv, wide);
                    }
                    if (p.lse != nullptr && row_valid) p.lse[at] = log_sum(m_run, l_run, p.scale_log2);
                }
            } else if (t * kRows < it->n_tok) {
                // A partial result; the warp that counts the last stretch of its 32 rows joins them, in their order.
                auto part_of = [&](int i) { return lp.part + static_cast<size_t>(it->first + i * p.Hq) * kPartFloats; };
                auto ml_of = [&](int i) { return reinterpret_cast<float2 *>(part_of(i) + kTiles * kPartTile) + t * kRows + row; };
                const int mine = (it->part - it->first) / p.Hq, parts = it->parts, at_row = t * kPartTile + row * 4;
                if (my_nb > 0) {
#pragma unroll
                    for (int c = 0; c < kLatentHead; c += 32) {
                        uint32_t o[32];
                        tmem_ld32(o_buf + c, o);
                        tmem_wait_ld();
                        if (c == kLatentHead - 32) o_read();
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            *reinterpret_cast<uint4 *>(part_of(mine) + at_row + (c / 4 + k) * kRows * 4) =
                                make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                    }
                }
                *ml_of(mine) = make_float2(m_run, l_run);
                int32_t *arrived = lp.arrived + arrived_set + it->first * kSoftmaxWarps + warp;
                int before = 0;
                __threadfence();
                __syncwarp();
                if (lane == 0) before = atomicAdd(arrived, 1);
                if (__shfl_sync(0xffffffffu, before, 0) == parts - 1) {
                    __threadfence();
                    float top = -INFINITY, sum = 0.f;
                    for (int i = 0; i < parts; ++i) {
                        const float2 ml = __ldcg(ml_of(i));
                        if (!(ml.y == 0.f)) top = fmaxf(top, ml.x);
                    }
                    for (int i = 0; i < parts; ++i) {
                        const float2 ml = __ldcg(ml_of(i));
                        if (!(ml.y == 0.f)) sum += ml.y * fast_exp2((ml.x - top) * p.scale_log2);
                    }
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll 1
                    for (int c = 0; c < kLatentHead; c += 32) {
                        float acc[32] = {};
#pragma unroll 4
                        for (int i = 0; i < parts; ++i) {
                            const float2 ml = __ldcg(ml_of(i));
                            const bool seen = !(ml.y == 0.f);  // a tile without blocks in a stretch has written no outputs
                            const float w = seen ? fast_exp2((ml.x - top) * p.scale_log2) : 0.f;
                            const float *from = part_of(i) + at_row + c * kRows;
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const float4 x = seen ? __ldcg(reinterpret_cast<const float4 *>(from + k * kRows * 4)) : make_float4(0.f, 0.f, 0.f, 0.f);
                                acc[4 * k] += w * x.x, acc[4 * k + 1] += w * x.y, acc[4 * k + 2] += w * x.z, acc[4 * k + 3] += w * x.w;
                            }
                        }
                        uint32_t o[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(acc[k]);
                        if (row_valid) store_cols(orow + c, o, inv, wide);
                    }
                    if (p.lse != nullptr && row_valid) p.lse[at] = log_sum(top, sum, p.scale_log2);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_taken + (taken - 2) % kItemSlots * 8);
            it = after;
        }
        cp_async_wait_all();
        if (!ok && lane == 0) latch(p.status, kDevTimeout, -1, blockIdx.x);
    }
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tm, kTmemCols);
}

}  // namespace

cudaError_t prepare_prefill_attn_latent() {
    const cudaError_t e = cudaFuncSetAttribute(prefill_attn_latent_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmemBytes));
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(prefill_attn_latent_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmemBytes));
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
    // Contexts are cut only where there may be fewer than two items per SM: beyond that the heaviest-first order evens them out.
    const long long most = static_cast<long long>((max_q_len - 1) / (kTiles * kRows) + 1) * p.a.Hq * p.a.B;
    const bool splits = p.a.B <= 32 && most <= 2 * p.num_sms;
    const dim3 grid(static_cast<unsigned>(p.num_sms));
    return launch_pdl(splits ? prefill_attn_latent_kernel<true> : prefill_attn_latent_kernel<false>, grid, dim3(kThreads), kSmemBytes, stream,
                      p.a.pdl != 0, tm_k, tm_v, tm_r, p);
}

}  // namespace pd
