// The int8 key/value cache: tokens rotated, quantised and written to their slots, and sequences read back.
//
// Both are bound by HBM: every element is read once and written once (2 or 4 bytes in and one out, or the
// reverse), a thread moving 16 codes of one head with 16-byte loads and stores.
//
// Exactness of the codes.  A code is the exact quotient y / step rounded to nearest; a border decides a whole
// step, so the value next to it needs more than fp32.  Computed in fp32,
//     z = (x*c -+ p*s) * (1/step)
// is off by at most (|x*c| + |p*s|)/step * 5.1 * 2^-24: half a step of 2^-24 each for c and s (rounded from
// fp64), the two products, the sum, 1/step and the last product, all relative to |x*c| + |p*s|.  With
// margin = (|x| + |p|) * scale/step * 2^-21 (8 * 2^-24, and |c|, |s| <= |scale|), a z that is further than margin
// from every border k + 1/2 has the right code; the others (about one in ten thousand) are computed again in
// fp64 by the definition.  NaN and infinities fail the comparison and go there too.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "hccs_device.cuh"
#include "hccs_internal.h"

namespace hccs {

namespace {

constexpr int kThreads = 256;
constexpr int kItem = 16;                  // codes per thread and step

template <typename T> struct Raw { uint4 w[sizeof(T) * kItem / 16]; };

template <typename T>
__device__ __forceinline__ Raw<T> load_raw(const T *p) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * kItem / 16); ++i) r.w[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
    return r;
}
__device__ __forceinline__ void unpack(const Raw<float> &r, float (&x)[kItem]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[4 * i] = __uint_as_float(r.w[i].x); x[4 * i + 1] = __uint_as_float(r.w[i].y);
        x[4 * i + 2] = __uint_as_float(r.w[i].z); x[4 * i + 3] = __uint_as_float(r.w[i].w);
    }
}
__device__ __forceinline__ void unpack(const Raw<__nv_bfloat16> &r, float (&x)[kItem]) {
    const uint32_t *w = reinterpret_cast<const uint32_t *>(r.w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const Raw<__half> &r, float (&x)[kItem]) {
    const __half2 *w = reinterpret_cast<const __half2 *>(r.w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 f = __half22float2(w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

// The definition, in fp64: (x*c + p*s) / step rounded to nearest even (s carries the sign), NaN -> 0.
__device__ __noinline__ int code_exact(float x, float p, double c, double s, float step) {
    const double y = __dadd_rn(__dmul_rn((double)x, c), __dmul_rn((double)p, s));
    const double z = rint(y / (double)step);
    return z != z ? 0 : (int)fmin(fmax(z, -128.0), 127.0);
}

// cos and sin of the pairs of one token.  A thread reads the 16 (halves) or 8 (neighbours) pairs of its item as
// vectors; the skew of four words per sixteen puts the four different items of a 128-dim head on different banks.
constexpr int kPairs = HCCS_MAX_ROT_DIM / 2;
__device__ __forceinline__ constexpr int skew(int pair) { return pair + (pair >> 4) * 4; }
struct __align__(16) Turn {
    float c[kPairs + 16], s[kPairs + 16];
    double cd[kPairs], sd[kPairs];
};

// One CTA: kTok tokens and, of each, the items blockIdx.y, blockIdx.y + gridDim.y, ... (kThreads at a time).
template <typename T, int kTok>
__global__ void __launch_bounds__(kThreads)
cache_write_kernel(const __grid_constant__ CacheWriteArgs a, FastDiv div_items, int per_head_shift) {
    __shared__ Turn turn[kTok];
    const int items = (int)div_items.d;                       // of one token
    const int t0 = blockIdx.x * kTok;
    const int tokens = min(kTok, a.T - t0);
    const int total = tokens * items;
    const int rot = a.rope.rot_dim, half = rot >> 1;
    const bool inter = a.rope.interleaved != 0;

    struct Place { int token, head, c0, kind; const T *src; };         // kind: 0 query, 1 key, 2 value
    auto place = [&](int idx) -> Place {
        Place p;
        const int tok = kTok == 1 ? 0 : (int)fast_div((uint32_t)idx, div_items);
        const int item = idx - tok * items;
        int head = item >> per_head_shift;
        p.token = t0 + tok;
        p.c0 = (item & ((1 << per_head_shift) - 1)) * kItem;
        const T *base;
        int64_t stride;
        if (head < a.Hq) { p.kind = 0; base = static_cast<const T *>(a.q); stride = a.q_stride; }
        else if (head < a.Hq + a.Hkv) { p.kind = 1; head -= a.Hq; base = static_cast<const T *>(a.k); stride = a.k_stride; }
        else { p.kind = 2; head -= a.Hq + a.Hkv; base = static_cast<const T *>(a.v); stride = a.v_stride; }
        p.head = head;
        p.src = base + p.token * stride + head * a.d;
        return p;
    };
    // the first item's loads are in flight while the angles are computed
    int idx = blockIdx.y * kThreads + threadIdx.x;
    Place pl;
    Raw<T> raw;
    if (idx < total) { pl = place(idx); raw = load_raw(pl.src + pl.c0); }
    if (rot > 0) {
        for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
            const int tok = i / half, pair = i - tok * half;
            double s, c;
            sincos(__dmul_rn((double)a.positions[t0 + tok], a.rope.freq[pair]), &s, &c);
            c = __dmul_rn(c, a.rope.scale);
            s = __dmul_rn(s, a.rope.scale);
            Turn &tn = turn[tok];
            tn.cd[pair] = c; tn.sd[pair] = s;
            tn.c[skew(pair)] = (float)c; tn.s[skew(pair)] = (float)s;
        }
        __syncthreads();
    }
    const int step_idx = gridDim.y * kThreads;
    while (idx < total) {
        const int next = idx + step_idx;
        Place npl = pl;
        Raw<T> nraw;
        if (next < total) { npl = place(next); nraw = load_raw(npl.src + npl.c0); }

        int8_t *dst = nullptr;
        if (pl.kind == 0) {
            dst = a.q8 + ((int64_t)pl.token * a.Hq + pl.head) * a.d + pl.c0;
        } else {
            const int64_t slot = a.slots[pl.token];
            if (slot >= a.num_slots) {
                atomicOr(a.status, STATUS_BAD_SLOT);
            } else if (slot >= 0) {
                const int64_t page = slot >> a.page_shift, off = slot & ((1 << a.page_shift) - 1);
                dst = (pl.kind == 1 ? a.k_pages : a.v_pages) + ((((page * a.Hkv + pl.head) << a.page_shift) + off) * a.d + pl.c0);
            }
        }
        if (dst) {
            const float step = a.step[pl.kind * HCCS_MAX_CACHE_HEADS + pl.head];
            const float inv = 1.0f / step;
            float x[kItem];
            unpack(raw, x);
            int code[kItem];
            if (pl.kind == 2 || pl.c0 >= rot) {
#pragma unroll
                for (int e = 0; e < kItem; ++e) {
                    const float z = x[e] * inv, r = rintf(z);
                    if (fabsf(z - r) < 0.5f - fabsf(z) * 0x1p-21f) code[e] = (int)fminf(fmaxf(r, -128.0f), 127.0f);
                    else code[e] = code_exact(x[e], 0.0f, 1.0, 0.0, step);
                }
            } else {
                const Turn &tn = turn[kTok == 1 ? 0 : pl.token - t0];
                const float bound = fabsf((float)a.rope.scale) * inv * 0x1p-21f;
                float p[kItem], c[kItem], s[kItem];           // partner, cosine, sine with the partner's sign
                bool whole = false;                           // every dim of the item is rotated, pairs in a vector
                if (inter) {
                    whole = pl.c0 + kItem <= rot;
                    if (whole) {
                        const int at = skew(pl.c0 >> 1);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float4 cv = *reinterpret_cast<const float4 *>(&tn.c[at + 4 * i]);
                            const float4 sv = *reinterpret_cast<const float4 *>(&tn.s[at + 4 * i]);
                            const float cc[4] = {cv.x, cv.y, cv.z, cv.w}, ss[4] = {sv.x, sv.y, sv.z, sv.w};
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int e = 8 * i + 2 * j;
                                c[e] = c[e + 1] = cc[j];
                                s[e] = -ss[j]; s[e + 1] = ss[j];
                                p[e] = x[e + 1]; p[e + 1] = x[e];
                            }
                        }
                    }
                } else {
                    whole = (half & (kItem - 1)) == 0;        // items lie in one half, and so do their partners
                    if (whole) {
                        const bool low = pl.c0 < half;
                        const int at = skew(low ? pl.c0 : pl.c0 - half);
                        unpack(load_raw(pl.src + (low ? pl.c0 + half : pl.c0 - half)), p);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 cv = *reinterpret_cast<const float4 *>(&tn.c[at + 4 * i]);
                            const float4 sv = *reinterpret_cast<const float4 *>(&tn.s[at + 4 * i]);
                            c[4 * i] = cv.x; c[4 * i + 1] = cv.y; c[4 * i + 2] = cv.z; c[4 * i + 3] = cv.w;
                            s[4 * i] = sv.x; s[4 * i + 1] = sv.y; s[4 * i + 2] = sv.z; s[4 * i + 3] = sv.w;
                        }
#pragma unroll
                        for (int e = 0; e < kItem; ++e) s[e] = low ? -s[e] : s[e];
                    }
                }
                if (!whole) {                                 // a pair at a time
#pragma unroll
                    for (int e = 0; e < kItem; ++e) {
                        const int dim = pl.c0 + e;
                        const bool turned = dim < rot;
                        const bool first = inter ? (dim & 1) == 0 : dim < half;
                        const int pair = !turned ? 0 : inter ? dim >> 1 : (first ? dim : dim - half);
                        const int other = !turned ? dim : inter ? dim ^ 1 : (first ? dim + half : dim - half);
                        p[e] = to_float(pl.src[other]);
                        c[e] = turned ? tn.c[skew(pair)] : 1.0f;
                        s[e] = !turned ? 0.0f : first ? -tn.s[skew(pair)] : tn.s[skew(pair)];
                        if (!turned) p[e] = 0.0f;
                    }
                }
#pragma unroll
                for (int e = 0; e < kItem; ++e) {
                    const float z = fmaf(x[e], c[e], p[e] * s[e]) * inv, r = rintf(z);
                    // (an unturned dim has c = 1, which the scale need not bound)
                    const float margin = (fabsf(x[e]) + fabsf(p[e])) * fmaxf(bound, whole ? 0.0f : inv * 0x1p-21f);
                    if (fabsf(z - r) < 0.5f - margin) {
                        code[e] = (int)fminf(fmaxf(r, -128.0f), 127.0f);
                    } else {
                        const int dim = pl.c0 + e;
                        if (dim >= rot) {
                            code[e] = code_exact(x[e], 0.0f, 1.0, 0.0, step);
                        } else {
                            const bool first = inter ? (dim & 1) == 0 : dim < half;
                            const int pair = inter ? dim >> 1 : (first ? dim : dim - half);
                            code[e] = code_exact(x[e], p[e], tn.cd[pair], first ? -tn.sd[pair] : tn.sd[pair], step);
                        }
                    }
                }
            }
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = __byte_perm(__byte_perm(code[4 * i], code[4 * i + 1], 0x0040), __byte_perm(code[4 * i + 2], code[4 * i + 3], 0x0040), 0x5410);
            *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        idx = next;
        pl = npl;
        raw = nraw;
    }
}

template <typename T> __device__ __forceinline__ void store16(T *p, const float (&x)[kItem]);
template <> __device__ __forceinline__ void store16<float>(float *p, const float (&x)[kItem]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<float4 *>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
}
template <> __device__ __forceinline__ void store16<__nv_bfloat16>(__nv_bfloat16 *p, const float (&x)[kItem]) {
    __nv_bfloat162 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    reinterpret_cast<uint4 *>(p)[0] = reinterpret_cast<const uint4 *>(v)[0];
    reinterpret_cast<uint4 *>(p)[1] = reinterpret_cast<const uint4 *>(v)[1];
}
template <> __device__ __forceinline__ void store16<__half>(__half *p, const float (&x)[kItem]) {
    __half2 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
    reinterpret_cast<uint4 *>(p)[0] = reinterpret_cast<const uint4 *>(v)[0];
    reinterpret_cast<uint4 *>(p)[1] = reinterpret_cast<const uint4 *>(v)[1];
}

constexpr int kReadTokens = 16;            // tokens per CTA of the read; each thread takes several items in turn

// One CTA: tokens kReadTokens * blockIdx.x ... of sequence blockIdx.y, all heads; blockIdx.z 0 keys, 1 values.
template <typename T>
__global__ void __launch_bounds__(kThreads)
cache_read_kernel(const __grid_constant__ CacheReadArgs a, int per_head_shift) {
    const int which = a.k_out ? (int)blockIdx.z : 1;
    const int8_t *pool = which == 0 ? a.k_pages : a.v_pages;
    T *out = static_cast<T *>(which == 0 ? a.k_out : a.v_out);
    const int b = blockIdx.y;
    const int start = a.out_start[b];
    const int64_t want = (int64_t)a.out_start[b + 1] - start;
    int len = (int)max(min(want, min((int64_t)a.max_len, (int64_t)a.max_pages << a.page_shift)), (int64_t)0);
    if (start < 0 || start > a.rows) len = 0;
    else len = min(len, a.rows - start);
    if (blockIdx.x == 0 && threadIdx.x == 0 && len != want) atomicOr(a.status, STATUS_BAD_LENGTH);
    const int j0 = blockIdx.x * kReadTokens;
    const int tokens = min(kReadTokens, len - j0);
    if (tokens <= 0) return;
    const int32_t *table = a.page_table + (int64_t)b * a.max_pages;
    // items ordered token, chunk inside a head: the codes of one head lie back to back in its page, and a head's
    // row of the output is a full run of sectors
    const int per_head = 1 << per_head_shift;
    const int total = tokens * a.Hkv * per_head;
#pragma unroll 4
    for (int idx = threadIdx.x; idx < total; idx += kThreads) {
        const int c0 = (idx & (per_head - 1)) * kItem;
        const int th = idx >> per_head_shift;
        const int tok = th / a.Hkv, head = th - tok * a.Hkv;
        const int j = j0 + tok;
        const int page = table[j >> a.page_shift];
        uint4 v = make_uint4(0, 0, 0, 0);
        if ((uint32_t)page < (uint32_t)a.num_pages)
            v = __ldg(reinterpret_cast<const uint4 *>(
                pool + (((((int64_t)page * a.Hkv + head) << a.page_shift) + (j & ((1 << a.page_shift) - 1))) * a.d + c0)));
        else
            atomicOr(a.status, STATUS_BAD_PAGE);
        const float step = a.step[which * HCCS_MAX_CACHE_HEADS + head];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        float x[kItem];
#pragma unroll
        for (int i = 0; i < kItem; ++i) x[i] = (float)(int8_t)(w[i >> 2] >> (8 * (i & 3))) * step;
        store16<T>(out + ((int64_t)(start + j) * a.Hkv + head) * a.d + c0, x);
    }
}

template <typename T>
cudaError_t write_typed(const CacheWriteArgs &a, cudaStream_t stream) {
    const int shift = a.d == 128 ? 3 : 2;
    const int items = (a.Hq + 2 * a.Hkv) << shift;
    const FastDiv div = make_fastdiv((uint32_t)items);
    if ((int64_t)a.T * items >= 8ll * 148 * kThreads) {
        const dim3 grid((unsigned)((a.T + 3) / 4), 1);
        cache_write_kernel<T, 4><<<grid, kThreads, 0, stream>>>(a, div, shift);
    } else {
        const dim3 grid((unsigned)a.T, (unsigned)((items + kThreads - 1) / kThreads));
        cache_write_kernel<T, 1><<<grid, kThreads, 0, stream>>>(a, div, shift);
    }
    return cudaGetLastError();
}

template <typename T>
cudaError_t read_typed(const CacheReadArgs &a, cudaStream_t stream) {
    const dim3 grid((unsigned)((a.max_len + kReadTokens - 1) / kReadTokens), (unsigned)a.B, a.k_out && a.v_out ? 2 : 1);
    cache_read_kernel<T><<<grid, kThreads, 0, stream>>>(a, a.d == 128 ? 3 : 2);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_cache_write(const CacheWriteArgs &a, int type, cudaStream_t stream, uint64_t *launches) {
    const cudaError_t e = type == HCCS_F32 ? write_typed<float>(a, stream)
                          : type == HCCS_BF16 ? write_typed<__nv_bfloat16>(a, stream) : write_typed<__half>(a, stream);
    if (e == cudaSuccess && launches) ++*launches;
    return e;
}

cudaError_t launch_cache_read(const CacheReadArgs &a, int type, cudaStream_t stream, uint64_t *launches) {
    const cudaError_t e = type == HCCS_F32 ? read_typed<float>(a, stream)
                          : type == HCCS_BF16 ? read_typed<__nv_bfloat16>(a, stream) : read_typed<__half>(a, stream);
    if (e == cudaSuccess && launches) ++*launches;
    return e;
}

}  // namespace hccs
