// Writing and reading back the 4-bit KV cache: quantising packed new tokens into their pages and dequantising token
// ranges into bf16 pages. Format and arithmetic of a row: pd_q4.cuh.
//
// Both kernels are a pass over the tokens bound by their bytes: a token of one KV head is 4 D bytes of bf16 (K and V)
// and 9 D / 8 bytes of 4-bit page. Writing, four lanes carry a group of 64 values (16 each: what a group costs beside its
// values is paid once per 16); reading back, eight do (8 each: one 16-byte store, whole 32-byte sectors per warp). A CTA takes 16
// packed tokens, or the tokens of one page: lane groups sit on them (rounded up to a power of two, so that a single token
// spreads over the KV heads instead of idling 15 of 16 groups) and walk the KV heads.
// The work forms one list that the CTAs share out evenly. Writing, that is the packed tokens; reading back, the pages of all
// sequences, whose counts each CTA sums itself (a grid of CTAs per sequence instead left short sequences' CTAs idle, and where the host knows no lengths it had to
// launch CTAs for every page a sequence could have: 12.2 against 5.5 us to write one token of 64 sequences and read it back).
// Measured for 4 x 32768 tokens at 8 KV heads, head_dim 128: written in 119 us (670 MB), read back in
// 123 us (688 MB), each 0.87 of the copy bandwidth.
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

// How `groups` lane groups share `nt` tokens of a page: group `sub` takes token sub % 2^shift and items sub >> shift,
// + step, ... of it.
struct PageShare {
    int shift, step;
};
__device__ __forceinline__ PageShare share_page(int nt, int groups) {
    const int shift = nt <= 1 ? 0 : 32 - __clz(nt - 1);
    return {shift, groups >> shift};
}

// The sequence whose part of a list holds entry x: the last one that begins at or before it (starts[0] <= x).
__device__ __forceinline__ int owner(const int32_t *starts, int B, int x) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (starts[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Exclusive prefix sums of count(b), b < B, into cum[0 .. B] (shared memory); every thread of the CTA takes part.
template <typename Count>
__device__ void prefix_sums(int B, int32_t *cum, int32_t *warp_sums, Count count) {
    const int tid = threadIdx.x, items = (B + kThreads - 1) / kThreads, begin = min(B, tid * items), end = min(B, begin + items);
    int sum = 0;
    for (int i = begin; i < end; ++i) {
        const int c = count(i);
        cum[i] = c;
        sum += c;
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, incl, o);
        if ((tid & 31) >= o) incl += up;
    }
    if ((tid & 31) == 31) warp_sums[tid >> 5] = incl;
    __syncthreads();
    int run = incl - sum;
    for (int w = 0; w < (tid >> 5); ++w) run += warp_sums[w];
    for (int i = begin; i < end; ++i) {
        const int c = cum[i];
        cum[i] = run;
        run += c;
    }
    if (tid == kThreads - 1) cum[B] = run;
    __syncthreads();
}

// SINGLE: one token per sequence and one CTA each, which also advances the length; otherwise CTAs take 16 packed tokens at a
// time. Where a token's values lie follows from its row alone, so they are on their way while its sequence is looked for.
template <int D, bool SINGLE>
__global__ void __launch_bounds__(kThreads, 5) kv_append_q4_kernel(const AppendQ4Params p) {
    constexpr int LANES = D / 16;  // lanes per row
    static_assert(kThreads / LANES >= 2 * kPageSize, "K and V of 16 tokens side by side: the hop below is at least one");
    const int j = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    grid_dependency_wait();
    launch_dependents();
    const int begin = SINGLE ? 0 : p.q_indptr[0], end = SINGLE ? p.B : p.q_indptr[p.B];
    constexpr int TILE = SINGLE ? 1 : kPageSize;
    for (int t0 = begin + static_cast<int>(blockIdx.x) * TILE; t0 < end; t0 += static_cast<int>(gridDim.x) * TILE) {
        const int nt = min(TILE, end - t0);
        const PageShare sh = share_page(nt, kThreads / LANES);
        const int t = min(sub & ((1 << sh.shift) - 1), nt - 1);
        const size_t row = static_cast<size_t>(SINGLE && p.q_indptr != nullptr ? p.q_indptr[t0] : t0 + t) * p.Hkv;
        // Items: K and V of the KV heads in turn. The step is even, so a lane stays with K or with V. Lanes without an item of their
        // own follow along on another's: the shuffles want whole warps. The next item's values are on their way while one is
        // worked on.
        const int item = sub >> sh.shift, which = item & 1, hop = sh.step >> 1;
        const __nv_bfloat16 *first = (which ? p.v_new : p.k_new) + row * D + j * 16;
        const __nv_bfloat16 *src = first + static_cast<size_t>(item >> 1) * D;
        uint4 x0, x1;
        auto load = [&](bool live) {
            const uint4 *from = reinterpret_cast<const uint4 *>(live ? src : first);
            x0 = __ldg(from);
            x1 = __ldg(from + 1);
        };
        int h = item >> 1;
        if (!SINGLE) load(h < p.Hkv);

        int b = t0, n = 1;
        if (!SINGLE) {
            b = owner(p.q_indptr, p.B, t0 + t);
            n = p.q_indptr[b + 1] - p.q_indptr[b];
        } else if (p.q_indptr != nullptr) {
            n = p.q_indptr[b + 1] - p.q_indptr[b];
        }
        const int L = p.ctx_lens[b];
        if (SINGLE) __syncthreads();  // everyone has read the length before thread 0 advances it
        if (SINGLE && n <= 0) continue;
        const int pos = SINGLE ? L : L + (t0 + t - p.q_indptr[b]);
        const bool room = L >= 0 && L <= p.MP * kPageSize - n && pos >= 0 && pos < p.MP * kPageSize && (!SINGLE || n == 1);
        int page = -1;
        if (room) page = p.page_table[static_cast<size_t>(b) * p.MP + pos / kPageSize];
        const bool ok = page >= 0 && page < p.num_pages;
        if (!ok && j == 0) latch(p.status, room ? kDevBadPage : kDevBadLength, b, room ? page : L);
        // the length of a packed token with a bad page grows all the same, as in the bf16 append
        if (SINGLE && p.advance && threadIdx.x == 0 && room && (ok || p.q_indptr != nullptr)) p.ctx_lens[b] = L + 1;
        if (SINGLE && !ok) continue;
        if (SINGLE) load(h < p.Hkv);

        const bool mine = ok && (sub & ((1 << sh.shift) - 1)) < nt;
        const int slot = pos & (kPageSize - 1);
        uint8_t *block = p.kv4 + (static_cast<size_t>(ok ? page : 0) * p.Hkv + (item >> 1)) * q4_block_bytes<D>();
        uint2 *codes_at = reinterpret_cast<uint2 *>(q4_codes_at<D>(block, which, slot, 2 * j));
        uint32_t *rec_at = q4_record_at<D>(block, which, slot, 2 * j);
        for (int h0 = 0; h0 < p.Hkv; h0 += hop) {
            const uint4 y0 = x0, y1 = x1;
            const bool live = mine && h < p.Hkv;
            h += hop;
            src += static_cast<size_t>(hop) * D;
            if (h0 + hop < p.Hkv) load(h < p.Hkv);
            uint32_t rec;
            const uint2 codes = q4_quantize16(y0, y1, rec);
            if (live) {
                *codes_at = codes;
                if ((j & 3) == 0) *rec_at = rec;
            }
            codes_at += static_cast<size_t>(hop) * (q4_block_bytes<D>() / 8);
            rec_at += static_cast<size_t>(hop) * (q4_block_bytes<D>() / 4);
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv_dequantize_q4_kernel(const DequantizeQ4Params p) {
    constexpr int LANES = D / 8;
    __shared__ int32_t cum[kMaxBatch + 1], warp_sums[kThreads / 32];
    const int j = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    grid_dependency_wait();
    launch_dependents();
    prefix_sums(p.B, cum, warp_sums, [&](int b) {
        const int L = p.ctx_lens[b], first = p.first_token != nullptr ? p.first_token[b] : 0;
        if (L < 0 || L > p.MP * kPageSize || first < 0) {
            if (blockIdx.x == 0) latch(p.status, kDevBadLength, b, first < 0 ? first : L);
            return 0;
        }
        return first < L ? (L - 1) / kPageSize - first / kPageSize + 1 : 0;
    });
    for (int x = blockIdx.x; x < cum[p.B]; x += gridDim.x) {
        const int b = owner(cum, p.B, x);
        const int L = p.ctx_lens[b], first = p.first_token != nullptr ? p.first_token[b] : 0, pg = first / kPageSize + x - cum[b];
        const int src = p.page_table[static_cast<size_t>(b) * p.MP + pg];
        const int dst = p.dst_page_table[static_cast<size_t>(b) * p.MP + pg];
        if (src < 0 || src >= p.num_pages || dst < 0 || dst >= p.num_pages) {
            if (threadIdx.x == 0) latch(p.status, kDevBadPage, b, src < 0 || src >= p.num_pages ? src : dst);
            continue;
        }
        const int t0 = max(pg * kPageSize, first), nt = min(pg * kPageSize + kPageSize, L) - t0;
        const PageShare sh = share_page(nt, kThreads / LANES);
        const int t = sub & ((1 << sh.shift) - 1), slot = (t0 + t) % kPageSize;
        if (t >= nt) continue;
        const uint8_t *block = p.kv4 + (static_cast<size_t>(src) * p.Hkv + (sub >> sh.shift)) * q4_block_bytes<D>();
        size_t at = ((static_cast<size_t>(dst) * p.Hkv + (sub >> sh.shift)) * kPageSize + slot) * D + j * 8;
        for (int h = sub >> sh.shift; h < p.Hkv; h += sh.step) {
            const uint32_t k = *q4_codes_at<D>(block, 0, slot, j), v = *q4_codes_at<D>(block, 1, slot, j);
            const uint2 rec = *reinterpret_cast<const uint2 *>(q4_record_at<D>(block, 0, slot, j));
            *reinterpret_cast<uint4 *>(p.k_pages + at) = q4_dequantize8(k, rec.x);
            *reinterpret_cast<uint4 *>(p.v_pages + at) = q4_dequantize8(v, rec.y);
            block += static_cast<size_t>(sh.step) * q4_block_bytes<D>();
            at += static_cast<size_t>(sh.step) * kPageSize * D;
        }
    }
}

// CTAs to launch: some waves of them, because the SMs differ in speed and the hardware hands late CTAs to the fast ones
// (131072 tokens written, in an earlier form: 134 us with 20 per SM, 152 us with 5, all resident), but no more than there can be pages. How many
// pages a read-back has the host does not know, and every CTA costs about 0.1 us per SM even if it finds none: 16.
int ctas(int64_t pages_most, int most) { return static_cast<int>(pages_most < most ? (pages_most < 1 ? 1 : pages_most) : most); }

}  // namespace

cudaError_t launch_kv_append_q4(const AppendQ4Params &p, int max_q_len, int num_sms, int *launched, cudaStream_t stream) {
    if (p.B == 0 || max_q_len <= 0) return cudaSuccess;
    auto go = [&](auto *k, int grid) { return launch_pdl(k, dim3(grid), dim3(kThreads), 0, stream, p.pdl != 0, p); };
    const bool single = max_q_len == 1;
    const int grid = single ? p.B : ctas((static_cast<int64_t>(p.B) * max_q_len + kPageSize - 1) / kPageSize, num_sms * 40);
    const cudaError_t err = single ? (p.D == 128 ? go(kv_append_q4_kernel<128, true>, grid) : go(kv_append_q4_kernel<64, true>, grid))
                                   : (p.D == 128 ? go(kv_append_q4_kernel<128, false>, grid) : go(kv_append_q4_kernel<64, false>, grid));
    if (err != cudaSuccess) return err;
    *launched = 1;
    if (!p.advance || single) return err;
    AppendTokensParams a{};
    a.q_indptr = p.q_indptr;
    a.ctx_lens = p.ctx_lens;
    a.B = p.B;
    a.MP = p.MP;
    a.pdl = p.pdl;
    *launched = 2;
    return launch_advance_lens(a, stream);
}

cudaError_t launch_kv_dequantize_q4(const DequantizeQ4Params &p, int num_sms, cudaStream_t stream) {
    if (p.B == 0) return cudaSuccess;
    const dim3 grid(ctas(static_cast<int64_t>(p.B) * p.MP, num_sms * 16));
    return p.D == 128 ? launch_pdl(kv_dequantize_q4_kernel<128>, grid, dim3(kThreads), 0, stream, p.pdl != 0, p)
                      : launch_pdl(kv_dequantize_q4_kernel<64>, grid, dim3(kThreads), 0, stream, p.pdl != 0, p);
}

}  // namespace pd
