// What the kernels of HCCS attention over the int8 cache share (they serve attention to an encoder's states as well: CROSS).
//
// With r_j = max(x_j + D - m, 0) in 0..127 a score is s_j = F + S*r_j, F = B - S*D >= 0, so that
//     Z = F*count + S*sum r,   sum s V = F*sum V + S*sum r V
// hold exactly in integers: sum r V is an int8 x int8 contraction that never leaves int32
// (127 * 128 * 131072 < 2^31), whatever the table, and sums of parts join without rounding.
#pragma once
#include <atomic>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "hccs_device.cuh"
#include "hccs_internal.h"
#include "hccs_tcgen05.cuh"

namespace hccs {

constexpr int kNone = -(1 << 30);          // below every accumulator

// of a whole warp: one try by all lanes is nearly always enough
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *abortp, uint32_t *status, long long limit) {
    if (__all_sync(~0u, mbar_try_wait(bar, parity))) return true;
    return __all_sync(~0u, mbar_wait(bar, parity, abortp, status, limit));
}

__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

// Where the new tokens and the keys of a sequence are.
struct SequenceAt {
    int s0, nq;        // first token, number of queries (those beyond max_q are not computed)
    int n;             // keys that may be seen
    int prefix;        // keys before the new ones (negative where there are fewer keys than queries); cross: all of them
    int k0;            // cross: the first key's place among the states
    bool cut;          // a length was beyond its bound
};
__device__ __forceinline__ SequenceAt cross_sequence(const CachedAttnArgs &a, int q0, int q1, int k0, int kv) {
    SequenceAt q;
    q.s0 = min(max(q0, 0), a.T);
    q.nq = min(max(q1, q.s0), a.T) - q.s0;
    q.k0 = k0;
    q.n = k0 < 0 || k0 > a.states ? 0 : max(min(min(kv, a.states - k0), a.max_kv), 0);
    q.prefix = q.n;
    q.cut = q.n != kv || q.nq > a.max_q;       // (without keys no start is a wrong one)
    return q;
}
// Keys [x, y) that query q of a sequence sees of an encoder's states: x = y = 0 where none.  Bounds are any int32, so they are cut
// and compared before one is taken from the other.
__device__ __forceinline__ int2 range_of(const CachedAttnArgs &a, const SequenceAt &seq, int q) {
    if (!a.key_range) return make_int2(0, seq.n);
    const int2 r = reinterpret_cast<const int2 *>(a.key_range)[(int64_t)seq.s0 + q];
    const int x = max(r.x, 0), y = min(r.y, seq.n);
    return x < y ? make_int2(x, y) : make_int2(0, 0);
}
template <bool CROSS = false>
__device__ __forceinline__ SequenceAt sequence_at(const CachedAttnArgs &a, int b) {
    if constexpr (CROSS) return cross_sequence(a, a.q_start[b], a.q_start[b + 1], a.k_start[b], a.kv_len[b]);
    SequenceAt q;
    const int s0 = min(max(a.q_start[b], 0), a.T), s1 = min(max(a.q_start[b + 1], s0), a.T);
    const int kv = a.kv_len[b];
    q.k0 = 0;
    const int pos = (int)max(min((int64_t)kv, (int64_t)a.max_pages << a.page_shift), (int64_t)0);
    q.s0 = s0;
    q.nq = s1 - s0;
    q.n = min(pos, a.max_kv);
    q.prefix = pos - q.nq;
    q.cut = q.n != kv || q.nq > a.max_q;
    return q;
}

// Requantisation of one head, x = clamp((acc*M + R) >> sh, -128, 127) with R = 2^(sh-1), as one clamp and one
// multiply-add: with lo and hi the accumulators between which x moves from -128 to 127 (steps below one, so
// both ends are reached) and k = 24 - sh, clamp(acc - lo, 0, hi - lo) * (M << k) + ((lo*M + R) << k) has x as
// its (signed) top byte; every value fits 32 bits.  M = 0 gives x = 0.  (The kernel for few keys has the same rule without fp64, head_requant.)
struct Requant {
    uint32_t mk, ck;
    int neg_lo, span;
};
constexpr int kAccLimit = 1 << 21;         // |acc| <= 128 * 128 * 128
__device__ __forceinline__ Requant make_requant(int M, int sh) {
    Requant q;
    const int64_t R = 1ll << (sh - 1);
    int lo = -kAccLimit, hi = kAccLimit;
    if (M > 0) {
        // floors of quotients below 2^32 by divisors below 2^13: exact through one fp64 division, whose
        // error (2^-21) is below the distance of a fraction from the next integer (2^-13)
        const double m = (double)M;
        const double a = floor((double)((128ll << sh) + R) / m), b = floor((double)((128ll << sh) - 1 - R) / m);
        if (a < (double)kAccLimit) lo = -(int)a;
        if (b < (double)kAccLimit) hi = (int)b;
    }
    q.mk = (uint32_t)M << (24 - sh);
    q.ck = (uint32_t)(uint64_t)(((int64_t)lo * M + R) << (24 - sh));
    q.neg_lo = -lo;
    q.span = hi - lo;
    return q;
}
__device__ __forceinline__ uint32_t requant_top(const Requant &q, int acc) {
    return (uint32_t)__viaddmin_s32_relu(acc, q.neg_lo, q.span) * q.mk + q.ck;
}

// One output value from num = sum s V and the row's Z (0: the row sees nothing): the integer of the int16
// path, or its product with the scale, or num * (scale / Z); each step rounded once to fp32.  Scales below 2^-60 are divided
// 2^64 times as large, since with Z up to 2^32 the quotient would lose bits below the normal range.
struct RowFactor {
    float scale;       // real: scale / Z; integer modes: the scale
    float unit;        // real: 1, or 2^-64 for a scale that was taken 2^64 times as large
    int rho;           // integer modes
};
__device__ __forceinline__ RowFactor row_factor(const CachedAttnArgs &a, int64_t Z, float scale) {
    RowFactor f;
    f.rho = 0;
    f.scale = 0.0f;
    f.unit = 1.0f;
    if (Z > 0) {
        if (a.recip == HCCS_RECIP_REAL) {
            const bool tiny = fabsf(scale) < 0x1p-60f;
            f.scale = (tiny ? scale * 0x1p64f : scale) / (float)Z;
            f.unit = tiny ? 0x1p-64f : 1.0f;
        } else {
            f.rho = (int)(a.recip == HCCS_RECIP_CLB ? reciprocal<true, true>((uint32_t)Z) : reciprocal<true, false>((uint32_t)Z));
            f.scale = scale;
        }
    }
    return f;
}
// Four neighbouring values as they are stored, in the low `size` words (two or four).
template <typename Int>
__device__ __forceinline__ uint4 output4(const CachedAttnArgs &a, const Int (&num)[4], const RowFactor &f) {
    int o[4];
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (a.recip == HCCS_RECIP_REAL) {
            o[e] = 0;
            y[e] = (float)num[e] * f.scale * f.unit;
        } else {
            o[e] = (int)num[e] * f.rho;
            y[e] = (float)o[e] * f.scale;
        }
    }
    if (a.out_type == HCCS_I32) return make_uint4((uint32_t)o[0], (uint32_t)o[1], (uint32_t)o[2], (uint32_t)o[3]);
    if (a.out_type == HCCS_F32) return make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
    if (a.out_type == HCCS_BF16) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(y[0], y[1]), hi = __floats2bfloat162_rn(y[2], y[3]);
        return make_uint4(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi), 0u, 0u);
    }
    const __half2 lo = __floats2half2_rn(y[0], y[1]), hi = __floats2half2_rn(y[2], y[3]);
    return make_uint4(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi), 0u, 0u);
}
__device__ __forceinline__ bool output_is_wide(const CachedAttnArgs &a) { return a.out_type == HCCS_I32 || a.out_type == HCCS_F32; }
// `at` is the index of the first of the four.
__device__ __forceinline__ void store_output4(const CachedAttnArgs &a, int64_t at, const int64_t (&num)[4], const RowFactor &f) {
    const uint4 v = output4(a, num, f);
    if (output_is_wide(a)) *reinterpret_cast<uint4 *>(static_cast<uint32_t *>(a.O) + at) = v;
    else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.O) + at) = make_uint2(v.x, v.y);
}

// A pool as [num_pages * Hkv][page_size][D] bytes, boxes of a page's rows (`most` at most), swizzled over the whole row.
inline bool make_page_map(CUtensorMap *map, const void *pool, const CachedAttnArgs &a, int most) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t page = (cuuint64_t)1 << a.page_shift;
    const int d = a.d;
    const cuuint64_t dims[3] = {(cuuint64_t)d, page, (cuuint64_t)a.num_pages * a.Hkv};
    const cuuint64_t strides[2] = {(cuuint64_t)d, page * d};
    const cuuint32_t box[3] = {(cuuint32_t)d, page < (cuuint64_t)most ? (cuuint32_t)page : (cuuint32_t)most, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void *>(pool), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Keys or values of an encoder's states, [states][Hkv][D] bytes, boxes of `most` keys of one head, swizzled over the whole row.
inline bool make_states_map(CUtensorMap *map, const void *states, int64_t stride, const CachedAttnArgs &a, int most) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const int d = a.d;
    const bool none = a.states == 0;           // (no load is ever issued then, but a map has an address and an extent)
    const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)a.Hkv, (cuuint64_t)(none ? 1 : a.states)};
    const cuuint64_t strides[2] = {(cuuint64_t)d, (cuuint64_t)(none ? (int64_t)a.Hkv * d : stride)};
    const cuuint32_t box[3] = {(cuuint32_t)d, 1, (cuuint32_t)most};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void *>(none ? (const void *)a.Q : states), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Raises a kernel's limits (dynamic shared memory, clusters of sixteen) once per kernel and device: `done` is the
// kernel's own array of flags.
inline cudaError_t raise_limits(const void *kernel, int smem, std::atomic<bool> (&done)[64]) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < 64 && done[dev].load(std::memory_order_acquire))) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess && dev < 64) done[dev].store(true, std::memory_order_release);
    return e;
}

constexpr int kMaxSplit = 16;              // CTAs per cluster

// Clusters of 1 .. 16 CTAs of one kernel that the current device holds at a time, with all of an SM's shared memory per CTA
// (how many depends on how the device's SMs are grouped; asked once per kernel and device).
struct Active { int n[kMaxSplit + 1]; std::atomic<bool> known; };
template <typename K>
cudaError_t active_clusters(K kernel, int threads, size_t smem, Active (&all)[64], const Active **out) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    Active &a = all[dev < 64 ? dev : 63];
    if (!a.known.load(std::memory_order_acquire) || dev >= 63) {
        for (int s = 1; s <= kMaxSplit; ++s) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)s, 64, 1);
            cfg.blockDim = dim3((unsigned)threads);
            cfg.dynamicSmemBytes = smem;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = (unsigned)s;
            attr[0].val.clusterDim.y = 1;
            attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            e = cudaOccupancyMaxActiveClusters(&a.n[s], kernel, &cfg);
            if (e != cudaSuccess) return e;
        }
        a.known.store(true, std::memory_order_release);
    }
    *out = &a;
    return cudaSuccess;
}

}  // namespace hccs
