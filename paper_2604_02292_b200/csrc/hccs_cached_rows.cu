// HCCS attention over the int8 cache, the simple form: one CTA per (query token, head).
//
// With r_j = max(x_j + D - m, 0) in 0..127 a score is s_j = F + S*r_j, F = B - S*D, so that
//     Z = F*count + S*sum r,   sum s V = F*sum V + S*sum r V
// hold exactly in integers (|sum r V| <= 127*128*131072 < 2^31).  The logits of a row need one byte each and
// stay in shared memory between the pass over K and the pass over V.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "hccs_device.cuh"
#include "hccs_internal.h"

namespace hccs {

namespace {

constexpr int kThreads = 128;

__global__ void __launch_bounds__(kThreads) cached_rows_kernel(const __grid_constant__ CachedAttnArgs a) {
    extern __shared__ __align__(16) uint8_t xs[];             // per key: its logit, and whether it is seen
    __shared__ uint4 q_s[8];
    __shared__ int red[3][4];
    const int t = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
    // the sequence of token t
    int lo = 0, hi = a.B;                                     // last b with q_start[b] <= t
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.q_start[mid] <= t) lo = mid; else hi = mid;
    }
    const int b = lo, s0 = max(a.q_start[b], 0), s1 = min(a.q_start[b + 1], a.T);
    if (t < s0 || t >= s1) return;
    const int i = t - s0, nq = s1 - s0;
    const int64_t cap = (int64_t)a.max_pages << a.page_shift;
    const int n_pos = (int)max(min((int64_t)a.kv_len[b], cap), (int64_t)0);
    const int n = min(n_pos, a.max_kv);
    if (tid == 0 && (n != a.kv_len[b] || nq > a.max_q)) atomicOr(a.status, STATUS_BAD_LENGTH);
    if (i >= a.max_q) return;
    const int prefix = n_pos - nq;
    const int kvh = h / a.group;
    const int32_t *table = a.page_table + (int64_t)b * a.max_pages;
    const int words = a.d / 16;
    uint32_t *seen_bits = reinterpret_cast<uint32_t *>(xs + ((a.max_kv + 15) & ~15));
    for (int w = tid; w < (n + 31) / 32; w += kThreads) seen_bits[w] = 0;
    if (tid < words) q_s[tid] = reinterpret_cast<const uint4 *>(a.Q + ((int64_t)t * a.Hq + h) * a.d)[tid];
    __syncthreads();
    const int64_t M = a.mult[h], R = 1ll << (a.requant_shift - 1);
    // pass over K
    int m = -1000;
    for (int j = tid; j < n; j += kThreads) {
        bool seen = true;
        if (j >= prefix) {
            const int jj = j - prefix;
            seen = a.tree_mask ? (jj < nq && jj < a.max_q && jj < 32 * a.tree_words && ((a.tree_mask[(int64_t)t * a.tree_words + (jj >> 5)] >> (jj & 31)) & 1))
                               : jj <= i;
        }
        const int page = table[j >> a.page_shift];
        if ((uint32_t)page >= (uint32_t)a.num_pages) { atomicOr(a.status, STATUS_BAD_PAGE); seen = false; }
        int x = -128;
        if (seen) {
            const uint4 *kr = reinterpret_cast<const uint4 *>(
                a.k_pages + ((((int64_t)page * a.Hkv + kvh) << a.page_shift) + (j & ((1 << a.page_shift) - 1))) * a.d);
            int acc = 0;
            for (int w = 0; w < words; ++w) {
                const uint4 kv = kr[w], qv = q_s[w];
                acc = __dp4a((int)kv.x, (int)qv.x, acc);
                acc = __dp4a((int)kv.y, (int)qv.y, acc);
                acc = __dp4a((int)kv.z, (int)qv.z, acc);
                acc = __dp4a((int)kv.w, (int)qv.w, acc);
            }
            x = (int)min(max((acc * M + R) >> a.requant_shift, (int64_t)-128), (int64_t)127);
            m = max(m, x);
        }
        xs[j] = (uint8_t)(int8_t)x;
        if (seen) atomicOr(&seen_bits[j >> 5], 1u << (j & 31));
    }
    for (int o = 16; o; o >>= 1) m = max(m, __shfl_xor_sync(~0u, m, o));
    if ((tid & 31) == 0) red[0][tid >> 5] = m;
    __syncthreads();
    m = max(max(red[0][0], red[0][1]), max(red[0][2], red[0][3]));
    const HeadEntry th = a.table[h];
    const int64_t F = th.B - th.S * th.D;
    // count and sum of r
    int count = 0, rsum = 0;
    for (int j = tid; j < n; j += kThreads) {
        if (!((seen_bits[j >> 5] >> (j & 31)) & 1)) continue;
        ++count;
        rsum += max((int)(int8_t)xs[j] + th.D - m, 0);
    }
    for (int o = 16; o; o >>= 1) {
        count += __shfl_xor_sync(~0u, count, o);
        rsum += __shfl_xor_sync(~0u, rsum, o);
    }
    if ((tid & 31) == 0) { red[1][tid >> 5] = count; red[2][tid >> 5] = rsum; }
    __syncthreads();
    count = red[1][0] + red[1][1] + red[1][2] + red[1][3];
    rsum = red[2][0] + red[2][1] + red[2][2] + red[2][3];
    const int64_t Z = F * count + (int64_t)th.S * rsum;
    if (tid >= a.d) return;
    int rv = 0, vsum = 0;
    for (int j = 0; j < n; ++j) {
        if (!((seen_bits[j >> 5] >> (j & 31)) & 1)) continue;
        const int page = table[j >> a.page_shift];
        const int v = a.v_pages[((((int64_t)page * a.Hkv + kvh) << a.page_shift) + (j & ((1 << a.page_shift) - 1))) * a.d + tid];
        vsum += v;
        rv += v * max((int)(int8_t)xs[j] + th.D - m, 0);
    }
    const int64_t num = F * vsum + (int64_t)th.S * rv;
    const int64_t at = ((int64_t)t * a.Hq + h) * a.d + tid;
    float y = 0.0f;
    int o = 0;
    if (count > 0) {
        if (a.recip == HCCS_RECIP_REAL) {
            y = (float)num * (a.scale[h] / (float)Z);
        } else {
            const uint32_t z = (uint32_t)Z;
            o = (int)num * (int)(a.recip == HCCS_RECIP_CLB ? reciprocal<true, true>(z) : reciprocal<true, false>(z));
            y = (float)o * a.scale[h];
        }
    }
    if (a.out_type == HCCS_I32) static_cast<int32_t *>(a.O)[at] = o;
    else if (a.out_type == HCCS_F32) static_cast<float *>(a.O)[at] = y;
    else if (a.out_type == HCCS_BF16) static_cast<__nv_bfloat16 *>(a.O)[at] = __float2bfloat16_rn(y);
    else static_cast<__half *>(a.O)[at] = __float2half_rn(y);
}

}  // namespace

cudaError_t launch_cached_attention(const CachedAttnArgs &a, cudaStream_t stream, uint64_t *launches) {
    if (a.max_q == 1) {
        const cudaError_t e = launch_cached_decode(a, stream);
        if (e == cudaSuccess && launches) ++*launches;
        return e;
    }
    const size_t smem = (size_t)a.max_kv + 16 + a.max_kv / 8 + 4;
    if (smem > 200 * 1024) return cudaErrorInvalidValue;
    cudaError_t e = cudaFuncSetAttribute(cached_rows_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
    if (e != cudaSuccess) return e;
    cached_rows_kernel<<<dim3((unsigned)a.T, (unsigned)a.Hq), kThreads, smem, stream>>>(a);
    e = cudaGetLastError();
    if (e == cudaSuccess && launches) ++*launches;
    return e;
}

}  // namespace hccs
