// Writing and reading back the 4-bit KV cache: quantising packed new tokens into their pages and dequantising token
// ranges into bf16 pages. Format and arithmetic of a row: pd_q4.cuh.
//
// Both kernels are a pass over the tokens bound by their bytes: a token of one KV head is 4 D bytes of bf16 (K and V)
// and 9 D / 8 bytes of 4-bit page. Eight lanes carry a group of 64 values (8 each, one 16-byte load or store), so a
// row of head_dim 128 takes half a warp and the group's minimum and maximum three shuffle steps. A CTA takes the new
// tokens of one page at a time and walks them slot-fastest within a (KV head, K or V): its code rows are then
// contiguous in the block.
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

template <int D>
__global__ void __launch_bounds__(kThreads) kv_append_q4_kernel(const AppendQ4Params p) {
    constexpr int LANES = D / 8;  // lanes per row
    const int b = blockIdx.y, j = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    grid_dependency_wait();
    launch_dependents();
    const int r0 = p.q_indptr != nullptr ? p.q_indptr[b] : b;
    const int n = p.q_indptr != nullptr ? p.q_indptr[b + 1] - r0 : 1;
    const int L = p.ctx_lens[b];
    if (n <= 0) return;
    if (L < 0 || L > p.MP * kPageSize - n) {
        if (threadIdx.x == 0 && blockIdx.x == 0) latch(p.status, kDevBadLength, b, L);
        return;
    }
    bool ok = true;
    for (int pg = L / kPageSize + blockIdx.x; pg * kPageSize < L + n; pg += gridDim.x) {
        const int page = p.page_table[static_cast<size_t>(b) * p.MP + pg];
        if (page < 0 || page >= p.num_pages) {
            if (threadIdx.x == 0) latch(p.status, kDevBadPage, b, page);
            ok = false;
            continue;
        }
        const int t0 = max(pg * kPageSize, L), nt = min(pg * kPageSize + kPageSize, L + n) - t0;
        const int items = nt * 2 * p.Hkv;  // rows; a warp's rows run or skip together, the shuffles need every lane
        for (int i0 = 0; i0 < items; i0 += kThreads / LANES) {
            const int i = min(i0 + sub, items - 1);
            const int hw = i / nt, pos = t0 + (i - hw * nt), kvh = hw >> 1, which = hw & 1, slot = pos % kPageSize;
            const __nv_bfloat16 *src = (which ? p.v_new : p.k_new) + (static_cast<size_t>(r0 + pos - L) * p.Hkv + kvh) * D + j * 8;
            uint32_t rec;
            const uint32_t codes = q4_quantize8(__ldg(reinterpret_cast<const uint4 *>(src)), rec);
            if (i0 + sub < items) {
                uint8_t *block = p.kv4 + (static_cast<size_t>(page) * p.Hkv + kvh) * q4_block_bytes<D>();
                *q4_codes_at<D>(block, which, slot, j) = codes;
                if ((j & 7) == 0) *q4_record_at<D>(block, which, slot, j) = rec;
            }
        }
    }
    // one CTA per sequence (single tokens): nobody else reads this length any more
    if (p.advance && gridDim.x == 1) {
        __syncthreads();
        if (threadIdx.x == 0 && (ok || p.q_indptr != nullptr)) p.ctx_lens[b] = L + n;
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv_dequantize_q4_kernel(const DequantizeQ4Params p) {
    constexpr int LANES = D / 8;
    const int b = blockIdx.y, j = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    grid_dependency_wait();
    launch_dependents();
    const int L = p.ctx_lens[b], first = p.first_token != nullptr ? p.first_token[b] : 0;
    if (L < 0 || L > p.MP * kPageSize || first < 0) {
        if (threadIdx.x == 0 && blockIdx.x == 0) latch(p.status, kDevBadLength, b, first < 0 ? first : L);
        return;
    }
    for (int pg = first / kPageSize + blockIdx.x; pg * kPageSize < L; pg += gridDim.x) {
        const int src = p.page_table[static_cast<size_t>(b) * p.MP + pg];
        const int dst = p.dst_page_table[static_cast<size_t>(b) * p.MP + pg];
        if (src < 0 || src >= p.num_pages || dst < 0 || dst >= p.num_pages) {
            if (threadIdx.x == 0) latch(p.status, kDevBadPage, b, src < 0 || src >= p.num_pages ? src : dst);
            continue;
        }
        const int t0 = max(pg * kPageSize, first), nt = min(pg * kPageSize + kPageSize, L) - t0;
        const int items = nt * 2 * p.Hkv;
        for (int i = sub; i < items; i += kThreads / LANES) {
            const int hw = i / nt, slot = (t0 + (i - hw * nt)) % kPageSize, kvh = hw >> 1, which = hw & 1;
            uint8_t *block = const_cast<uint8_t *>(p.kv4) + (static_cast<size_t>(src) * p.Hkv + kvh) * q4_block_bytes<D>();
            const uint4 v = q4_dequantize8(*q4_codes_at<D>(block, which, slot, j), *q4_record_at<D>(block, which, slot, j));
            __nv_bfloat16 *out = (which ? p.v_pages : p.k_pages) + ((static_cast<size_t>(dst) * p.Hkv + kvh) * kPageSize + slot) * D + j * 8;
            *reinterpret_cast<uint4 *>(out) = v;
        }
    }
}

// CTAs per sequence: enough to fill the device a few times over, no more than a sequence has pages.
int ctas_per_sequence(int pages_most, int batch, int num_sms) {
    const int want = (num_sms * 8 + batch - 1) / batch;
    return pages_most < want ? (pages_most < 1 ? 1 : pages_most) : want;
}

}  // namespace

cudaError_t launch_kv_append_q4(const AppendQ4Params &p, int max_q_len, int num_sms, int *launched, cudaStream_t stream) {
    if (p.B == 0 || max_q_len <= 0) return cudaSuccess;
    // max_q_len tokens that start inside a page touch one page more than they fill
    const int x = max_q_len == 1 ? 1 : ctas_per_sequence((max_q_len + kPageSize - 2) / kPageSize + 1, p.B, num_sms);
    const dim3 grid(x, p.B);
    const cudaError_t err = p.D == 128 ? launch_pdl(kv_append_q4_kernel<128>, grid, dim3(kThreads), 0, stream, p.pdl != 0, p)
                                       : launch_pdl(kv_append_q4_kernel<64>, grid, dim3(kThreads), 0, stream, p.pdl != 0, p);
    if (err != cudaSuccess) return err;
    *launched = 1;
    if (!p.advance || x == 1) return err;
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
    const dim3 grid(ctas_per_sequence(p.MP, p.B, num_sms), p.B);
    return p.D == 128 ? launch_pdl(kv_dequantize_q4_kernel<128>, grid, dim3(kThreads), 0, stream, p.pdl != 0, p)
                      : launch_pdl(kv_dequantize_q4_kernel<64>, grid, dim3(kThreads), 0, stream, p.pdl != 0, p);
}

}  // namespace pd
