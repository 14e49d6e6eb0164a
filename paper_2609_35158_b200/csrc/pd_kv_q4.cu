// Writing and reading back the 4-bit KV cache: quantising packed new tokens into their pages and dequantising token
// ranges into bf16 pages. Format and arithmetic of a row: pd_q4.cuh.
//
// Both kernels are a pass over the tokens bound by their bytes: a token of one KV head is 4 D bytes of bf16 (K and V)
// and 9 D / 8 bytes of 4-bit page. Writing, four lanes carry a group of 64 values (16 each: what a group costs beside its
// values is paid once per 16); reading back, eight do (8 each: one 16-byte store, whole 32-byte sectors per warp). A CTA takes the
// tokens of one page: lane groups sit on its slots (rounded up to a power of two, so that a single token spreads over the
// KV heads instead of idling 15 of 16 groups) and walk the KV heads.
// The pages of all sequences form one list that the CTAs share out evenly: each CTA sums the sequences' page counts itself
// (a grid of CTAs per sequence instead left short sequences' CTAs idle, and where the host knows no lengths it had to
// launch CTAs for every page a sequence could have: 12.2 against 5.5 us to write one token of 64 sequences and read it back).
// Measured for 4 x 32768 tokens at 8 KV heads, head_dim 128: written in 134 us (670 MB, 0.78 of the copy bandwidth), read back
// in 117 us (688 MB, 0.91).
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

// The sequence whose part of the list holds entry x < cum[B].
__device__ __forceinline__ int owner(const int32_t *cum, int B, int x) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cum[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// SINGLE: one token per sequence and one CTA each, which also advances the length; otherwise packed tokens.
template <int D, bool SINGLE>
__global__ void __launch_bounds__(kThreads) kv_append_q4_kernel(const AppendQ4Params p) {
    constexpr int LANES = D / 16;  // lanes per row
    __shared__ int32_t cum[SINGLE ? 1 : kMaxBatch + 1], warp_sums[kThreads / 32];
    const int j = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    grid_dependency_wait();
    launch_dependents();
    if (!SINGLE) {
        prefix_sums(p.B, cum, warp_sums, [&](int b) {
            const int n = p.q_indptr[b + 1] - p.q_indptr[b], L = p.ctx_lens[b];
            if (n <= 0) return 0;
            if (L < 0 || L > p.MP * kPageSize - n) {
                if (blockIdx.x == 0) latch(p.status, kDevBadLength, b, L);
                return 0;
            }
            return (L + n - 1) / kPageSize - L / kPageSize + 1;
        });
    }
    const int total = SINGLE ? p.B : cum[p.B];
    for (int x = blockIdx.x; x < total; x += gridDim.x) {
        const int b = SINGLE ? x : owner(cum, p.B, x);
        const int r0 = p.q_indptr != nullptr ? p.q_indptr[b] : b, n = p.q_indptr != nullptr ? p.q_indptr[b + 1] - r0 : 1;
        const int L = p.ctx_lens[b];
        if (SINGLE) {
            __syncthreads();  // everyone has read the length before thread 0 advances it
            if (n <= 0) continue;
            if (n != 1 || L < 0 || L >= p.MP * kPageSize) {
                if (threadIdx.x == 0) latch(p.status, kDevBadLength, b, L);
                continue;
            }
        }
        const int pg = L / kPageSize + (SINGLE ? 0 : x - cum[b]);
        const int page = p.page_table[static_cast<size_t>(b) * p.MP + pg];
        const bool ok = page >= 0 && page < p.num_pages;
        if (!ok && threadIdx.x == 0) latch(p.status, kDevBadPage, b, page);
        // the length of a packed token with a bad page grows all the same, as in the bf16 append
        if (SINGLE && p.advance && threadIdx.x == 0 && (ok || p.q_indptr != nullptr)) p.ctx_lens[b] = L + 1;
        if (!ok) continue;
        const int t0 = max(pg * kPageSize, L), nt = min(pg * kPageSize + kPageSize, L + n) - t0;
        const PageShare sh = share_page(nt, kThreads / LANES);
        const int t = sub & ((1 << sh.shift) - 1), slot = (t0 + min(t, nt - 1)) % kPageSize;
        const size_t row = static_cast<size_t>(r0 + t0 - L + min(t, nt - 1)) * p.Hkv;
        // items: K and V of the KV heads in turn. Lanes without an item of their own follow along on another's: the shuffles
        // want whole warps. The next item's values are on their way while one is worked on.
        uint4 x0, x1;
        auto load = [&](int i) {
            const int item = min(i, 2 * p.Hkv - 1);
            const uint4 *src = reinterpret_cast<const uint4 *>(((item & 1) ? p.v_new : p.k_new) + (row + (item >> 1)) * D + j * 16);
            x0 = __ldg(src);
            x1 = __ldg(src + 1);
        };
        int i = sub >> sh.shift;
        load(i);
        for (int i0 = 0; i0 < 2 * p.Hkv; i0 += sh.step, i += sh.step) {
            const uint4 y0 = x0, y1 = x1;
            if (i0 + sh.step < 2 * p.Hkv) load(i + sh.step);
            uint32_t rec;
            const uint2 codes = q4_quantize16(y0, y1, rec);
            if (t < nt && i < 2 * p.Hkv) {
                uint8_t *block = p.kv4 + (static_cast<size_t>(page) * p.Hkv + (i >> 1)) * q4_block_bytes<D>();
                *reinterpret_cast<uint2 *>(q4_codes_at<D>(block, i & 1, slot, 2 * j)) = codes;
                if ((j & 3) == 0) *q4_record_at<D>(block, i & 1, slot, 2 * j) = rec;
            }
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
// (131072 tokens written: 134 us with 20 per SM, 152 us with 5, all resident), but no more than there can be pages. How many
// pages a read-back has the host does not know, and every CTA costs about 0.1 us per SM even if it finds none: 16.
int ctas(int64_t pages_most, int most) { return static_cast<int>(pages_most < most ? (pages_most < 1 ? 1 : pages_most) : most); }

}  // namespace

cudaError_t launch_kv_append_q4(const AppendQ4Params &p, int max_q_len, int num_sms, int *launched, cudaStream_t stream) {
    if (p.B == 0 || max_q_len <= 0) return cudaSuccess;
    auto go = [&](auto *k, int grid) { return launch_pdl(k, dim3(grid), dim3(kThreads), 0, stream, p.pdl != 0, p); };
    const bool single = max_q_len == 1;
    // max_q_len tokens that start inside a page touch one page more than they fill
    const int grid = single ? p.B : ctas(static_cast<int64_t>(p.B) * ((max_q_len + kPageSize - 2) / kPageSize + 1), num_sms * 40);
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
