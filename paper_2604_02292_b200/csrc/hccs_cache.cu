// The int8 key/value cache: tokens rotated, quantised and written to their slots, and sequences read back.
//
// Every element is read once and written once (2 or 4 bytes in and one out, or the reverse).  Reading back is bound by
// HBM: 8 sequences of 8192 tokens (8 heads of 128, to bf16) in 65 us, 6.2 TB/s.  Writing is bound by instructions, about
// twenty per element with the margins below (issue slots 70 % busy, DRAM 45 %): 16384 tokens (32 + 8 + 8 heads of 128,
// bf16, all of a head rotated) in 74 us, 4.1 TB/s; without rotation 60 us, 5.0 TB/s.
//
// Exactness of the codes.  A code is the exact quotient y / step rounded to nearest; a border decides a whole
// step, so the value next to it needs more than fp32.  Computed in fp32,
//     z = (a*c - b*s) * (1/step)
// is off by at most X * 7 * 2^-24, X = (|a| + |b|) * |scale|/step: 1.5 for c and s (the angle is reduced to a part of a
// turn in fp64 and held in two floats, sincospi is good to one ulp, the join rounds once), 1 each for the scale's own
// rounding and its product, for the product and the sum, for 1/step, and half for the distance from the border, where X
// is at least a half.  With margin = X * 8 * 2^-24, a z that is further than margin from every border k + 1/2 has the
// right code; the few pairs with any other (one in five thousand on usual data) are computed in fp64 by the
// definition.  NaN and infinities fail the comparison too, and the turn of an angle beyond 2^24 is made NaN: its
// reduction would be off by more than that share.  Dims that are not rotated need no fp64: see
// code_of_quotient.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "hccs_device.cuh"
#include "hccs_internal.h"

namespace hccs {

namespace {

constexpr int kThreads = 256;

// Eight neighbouring elements as they are loaded.
template <typename T> struct Raw { uint4 w[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Raw<T> load_raw(const T *p) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.w[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
    return r;
}
// elements 4g .. 4g + 3
__device__ __forceinline__ void unpack4(const Raw<float> &r, int g, float (&x)[4]) {
    x[0] = __uint_as_float(r.w[g].x); x[1] = __uint_as_float(r.w[g].y); x[2] = __uint_as_float(r.w[g].z); x[3] = __uint_as_float(r.w[g].w);
}
__device__ __forceinline__ void unpack4(const Raw<__nv_bfloat16> &r, int g, float (&x)[4]) {
    const uint32_t w[2] = {g ? r.w[0].z : r.w[0].x, g ? r.w[0].w : r.w[0].y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack4(const Raw<__half> &r, int g, float (&x)[4]) {
    const uint32_t w[2] = {g ? r.w[0].z : r.w[0].x, g ? r.w[0].w : r.w[0].y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

// cos and sin of the pairs of one token.  A thread reads the eight pairs of its item as vectors; the skew of four
// words per 32 puts the items of a head on different banks.
constexpr int kPairs = HCCS_MAX_ROT_DIM / 2;
__device__ __forceinline__ constexpr int skew(int pair) { return pair + (pair >> 5) * 4; }
struct __align__(16) Turn { float c[kPairs + 4], s[kPairs + 4], ns[kPairs + 4]; };      // ns = -s

// Two fp32 operations per instruction.
struct F2 { uint64_t v; };
__device__ __forceinline__ F2 f2(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split(F2 a, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a.v)); }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
// Nearest integer of z (|z| < 2^22, as the margin sees to) in `n`; returns the distance of z from it.
__device__ __forceinline__ float nearest(float z, int &n) {
    const float t = __fadd_rn(z, 12582912.0f);                 // 1.5 * 2^23
    n = __float_as_int(t) - 0x4b400000;
    return fabsf(__fsub_rn(z, __fsub_rn(t, 12582912.0f)));
}
// The code of x / step, exactly and in fp32.  k is the nearest integer of x * (1/step), or its neighbour; what is left,
// x - k*step, is a multiple of the last place of step (or of x, where x is smaller) and no larger than about half a
// step, so one fused multiply-add gives it without rounding, and half a step is exact: beyond half, or at half of an odd
// k, the neighbour is right.  (Steps like 0.03 or 1/32 put many 16-bit inputs exactly on a border.)
__device__ __forceinline__ int code_of_quotient(float x, float step, float inv) {
    const float z = fminf(fmaxf(x * inv, -200.0f), 200.0f);
    int k;
    nearest(z, k);
    const float left = fmaf(-(float)k, step, x), half = 0.5f * step;
    if (fabsf(left) > half || (fabsf(left) == half && (k & 1))) k += left > 0.0f ? 1 : -1;
    return x != x ? 0 : k;
}
__device__ __forceinline__ uint32_t pack4(int n0, int n1, int n2, int n3) {      // four integers clamped to int8
    uint32_t hi, d;
    asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(hi) : "r"(n3), "r"(n2), "r"(0));
    asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(n1), "r"(n0), "r"(hi));
    return d;
}

// A pair by the definition, in fp64: the codes of a' and b', packed into the low two bytes.
__device__ __noinline__ uint32_t code_pair(float a, float b, double position, double freq, double scale, float step) {
    double s, c;
    sincos(__dmul_rn(position, freq), &s, &c);
    c = __dmul_rn(c, scale);
    s = __dmul_rn(s, scale);
    const double u = rint(__dsub_rn(__dmul_rn((double)a, c), __dmul_rn((double)b, s)) / (double)step);
    const double v = rint(__dadd_rn(__dmul_rn((double)b, c), __dmul_rn((double)a, s)) / (double)step);
    const int m = u != u ? 0 : (int)fmin(fmax(u, -128.0), 127.0), n = v != v ? 0 : (int)fmin(fmax(v, -128.0), 127.0);
    return (uint32_t)(m & 255) | (uint32_t)(n & 255) << 8;
}

// Items of heads whose rotated part is no multiple of 16 dims: a dim at a time, in fp32 where that is sure.
template <typename T>
__device__ __noinline__ int8_t code_of(const T *head, int dim, int rot, bool inter, const Turn *turn, double position, const double *freq,
                                       double scale, float step) {
    const float x = to_float(head[dim]), inv = 1.0f / step;
    if (dim >= rot) return (int8_t)max(min(code_of_quotient(x, step, inv), 127), -128);
    const int half = rot >> 1;
    const bool first = inter ? (dim & 1) == 0 : dim < half;
    const int pair = inter ? dim >> 1 : (first ? dim : dim - half);
    const float p = to_float(head[inter ? dim ^ 1 : (first ? dim + half : dim - half)]);
    const float s = turn->s[skew(pair)];
    const float z = __fmul_rn(fmaf(x, turn->c[skew(pair)], __fmul_rn(p, first ? -s : s)), inv);
    int n;
    if (fmaf(fabsf(x) + fabsf(p), fmaxf(fabsf((float)scale) * inv * 0x1p-21f, 0x1p-125f), nearest(z, n)) < 0.5f) return (int8_t)max(min(n, 127), -128);
    const uint32_t two = first ? code_pair(x, p, position, freq[pair], scale, step) : code_pair(p, x, position, freq[pair], scale, step) >> 8;
    return (int8_t)(two & 255);
}

// A thread owns one item, two chunks of eight dims of one head, and walks over the CTA's tokens with the loads of the
// next on their way: head, kind, step and place in the tables of cosines are worked out once (with the items of a
// token in turn to each thread, a prompt of 16384 tokens took 130 us).  The chunks are half a part (rotated or not)
// apart, so that neighbouring lanes read and write neighbouring chunks, and in the half layout a's partner is b.
constexpr int kWriteThreads = 384;         // most threads per CTA: all items of a token where they fit, so that its angles are computed once
constexpr int kTokens = 16;                // most tokens per CTA

template <typename T>
__global__ void __launch_bounds__(kWriteThreads, 2)
cache_write_kernel(const __grid_constant__ CacheWriteArgs a, int items, int per_head_shift, int per_cta) {
    __shared__ Turn turn[kTokens];
    const int t0 = blockIdx.x * per_cta;
    const int tokens = min(per_cta, a.T - t0);
    const int rot = a.rope.rot_dim, half = rot >> 1;
    const bool inter = a.rope.interleaved != 0;
    const bool aligned = (rot & 15) == 0;                     // rotated items hold eight whole pairs

    const int item = blockIdx.y * blockDim.x + threadIdx.x;
    int head = item >> per_head_shift, chunk = item & ((1 << per_head_shift) - 1);
    const int all = 1 << per_head_shift, some = (rot + 15) >> 4;              // items of a head, and those with rotated dims
    if (some != 0 && some != all) {
        // the rotated items of all heads first, then the others: a warp with both kinds would take both branches below
        const int rotated = (a.Hq + a.Hkv) * some, i = item - rotated;
        if (i < 0) { head = item / some; chunk = item - head * some; }
        else if (i < (a.Hq + a.Hkv) * (all - some)) { head = i / (all - some); chunk = some + i - head * (all - some); }
    }
    const int kind = head < a.Hq ? 0 : head < a.Hq + a.Hkv ? 1 : 2;            // query, key, value
    head -= kind == 0 ? 0 : kind == 1 ? a.Hq : a.Hq + a.Hkv;
    const bool mine = item < items;
    const bool turned = kind != 2 && (aligned ? chunk * 16 < rot : chunk * 16 < ((rot + 15) & ~15));
    int dim_a, dim_b;
    if (!aligned || kind == 2) { dim_a = aligned ? chunk * 8 : chunk * 16; dim_b = aligned ? dim_a + (a.d >> 1) : dim_a + 8; }
    else if (turned) { dim_a = chunk * 8; dim_b = dim_a + half; }
    else { dim_a = rot + (chunk - (rot >> 4)) * 8; dim_b = dim_a + ((a.d - rot) >> 1); }
    const int64_t stride = kind == 0 ? a.q_stride : kind == 1 ? a.k_stride : a.v_stride;
    const T *src = static_cast<const T *>(kind == 0 ? a.q : kind == 1 ? a.k : a.v) + t0 * stride + head * a.d;
    Raw<T> raw_a, raw_b;
    if (mine && tokens > 0) { raw_a = load_raw(src + dim_a); raw_b = load_raw(src + dim_b); }

    if (rot > 0) {
        // a thread stays with one pair (two in a CTA of 32 threads): the next power of two of pairs side by side, several
        // tokens abreast (with pairs and tokens in turn, and a division for each, a prompt took 2.5 us more)
        const int wide = min(1 << (32 - __clz(half - 1)), (int)blockDim.x), abreast = (int)blockDim.x / wide;
        const int tok0 = (int)threadIdx.x / wide;
        for (int pair = (int)threadIdx.x & (wide - 1); pair < half && tok0 < abreast; pair += wide) {
            const double freq = a.rope.freq[pair];
            const float scale = (float)a.rope.scale;
            for (int tok = tok0; tok < tokens; tok += abreast) {
                // the angle as the definition rounds it, in turns, less the whole ones: exact but for 2^-53 of the turns
                const double angle = __dmul_rn((double)a.positions[t0 + tok], freq), turns = __dmul_rn(angle, 0.15915494309189533577);
                const double part = turns - rint(turns);
                const float hi = (float)part, lo = (float)(part - (double)hi) * 6.2831853f;
                float s, c;
                sincospif(2.0f * hi, &s, &c);
                // beyond 2^24 radians the turns are no longer good to the margin's share (2^-27): NaN sends all codes to fp64
                if (!(fabs(angle) < 0x1p24)) c = s = __int_as_float(0x7fffffff);
                const float ss = (s + lo * c) * scale;
                turn[tok].c[skew(pair)] = (c - lo * s) * scale;
                turn[tok].s[skew(pair)] = ss;
                turn[tok].ns[skew(pair)] = -ss;
            }
        }
        __syncthreads();
    }
    if (!mine) return;
    const float step = a.step[kind * HCCS_MAX_CACHE_HEADS + head], inv = 1.0f / step;
    const F2 inv2 = f2(inv, inv), neg_inv2 = f2(-inv, -inv);
    // (never so small that it loses digits below the normal range: values near 2^128 with steps near 2^100)
    const float bound = -fmaxf((turned ? fabsf((float)a.rope.scale) : 1.0f) * inv * 0x1p-21f, 0x1p-125f);
    const F2 bound2 = f2(bound, bound), half2 = f2(0.5f, 0.5f), magic2 = f2(12582912.0f, 12582912.0f), unmagic2 = f2(-12582912.0f, -12582912.0f);
    // nearest integers of w * (1/step) for two values; `sure` stays if both are further than their margins from a border
    auto nearest2 = [&](F2 w, F2 limit, int &n0, int &n1, bool &sure) {
        const F2 t = fma2(w, inv2, magic2);
        const F2 d = fma2(w, neg_inv2, add2(t, unmagic2));
        float t0_, t1_, d0, d1, l0, l1;
        split(t, t0_, t1_);
        split(d, d0, d1);
        split(limit, l0, l1);
        n0 = __float_as_int(t0_) - 0x4b400000;
        n1 = __float_as_int(t1_) - 0x4b400000;
        sure = sure & (fabsf(d0) < l0) & (fabsf(d1) < l1);
    };
    const int at_a = skew(inter ? dim_a >> 1 : dim_a), at_b = skew(inter ? dim_b >> 1 : dim_a + 4);
    int8_t *q_dst = a.q8 + ((int64_t)t0 * a.Hq + head) * a.d;
    int8_t *const pool = kind == 1 ? a.k_pages : a.v_pages;
    int64_t slot = kind != 0 ? a.slots[t0] : 0;
    auto place = [&](int64_t at) -> int8_t * {
        if (at >= a.num_slots) atomicOr(a.status, STATUS_BAD_SLOT);
        if (at < 0 || at >= a.num_slots) return nullptr;
        const int64_t page = at >> a.page_shift, off = at & ((1 << a.page_shift) - 1);
        return pool + (((page * a.Hkv + head) << a.page_shift) + off) * a.d;
    };
    uint32_t redo = 0;                                        // bit 2j + g: chunk g of token j again, see below
    for (int j = 0; j < tokens; ++j) {
        Raw<T> next_a, next_b;
        if (j + 1 < tokens) { next_a = load_raw(src + stride + dim_a); next_b = load_raw(src + stride + dim_b); }
        const int64_t next_slot = kind != 0 && j + 1 < tokens ? a.slots[t0 + j + 1] : 0;
        int8_t *const dst = kind == 0 ? q_dst : place(slot);  // the head
        if (dst) {
            const Turn &tn = turn[j];
            uint32_t wa[2], wb[2];                            // the codes of the two chunks
            if (!turned) {
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    float x[4], y[4];
                    unpack4(raw_a, g, x);
                    unpack4(raw_b, g, y);
                    int nx[4], ny[4];
                    bool sure = true;
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        nearest2(f2(x[e], x[e + 1]), fma2(f2(fabsf(x[e]), fabsf(x[e + 1])), bound2, half2), nx[e], nx[e + 1], sure);
                        nearest2(f2(y[e], y[e + 1]), fma2(f2(fabsf(y[e]), fabsf(y[e + 1])), bound2, half2), ny[e], ny[e + 1], sure);
                    }
                    if (!sure) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            nx[e] = code_of_quotient(x[e], step, inv);
                            ny[e] = code_of_quotient(y[e], step, inv);
                        }
                    }
                    wa[g] = pack4(nx[0], nx[1], nx[2], nx[3]);
                    wb[g] = pack4(ny[0], ny[1], ny[2], ny[3]);
                }
            } else if (aligned) {
                // four pairs (u, v) at a time: in halves elements 4g ... of either chunk, else the neighbours of chunk g
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    float u[4], v[4];
                    if (inter) {
                        float lo[4], hi[4];
                        unpack4(g ? raw_b : raw_a, 0, lo);
                        unpack4(g ? raw_b : raw_a, 1, hi);
                        u[0] = lo[0]; v[0] = lo[1]; u[1] = lo[2]; v[1] = lo[3];
                        u[2] = hi[0]; v[2] = hi[1]; u[3] = hi[2]; v[3] = hi[3];
                    } else {
                        unpack4(raw_a, g, u);
                        unpack4(raw_b, g, v);
                    }
                    int nu[4], nv[4];
                    bool sure = true;
                    const int at = g ? at_b : at_a;
                    const float4 c = *reinterpret_cast<const float4 *>(&tn.c[at]), s = *reinterpret_cast<const float4 *>(&tn.s[at]),
                                 ns = *reinterpret_cast<const float4 *>(&tn.ns[at]);
                    const F2 c2[2] = {f2(c.x, c.y), f2(c.z, c.w)}, s2[2] = {f2(s.x, s.y), f2(s.z, s.w)}, ns2[2] = {f2(ns.x, ns.y), f2(ns.z, ns.w)};
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const F2 u2 = f2(u[2 * i], u[2 * i + 1]), v2 = f2(v[2 * i], v[2 * i + 1]);
                        const F2 limit = fma2(f2(fabsf(u[2 * i]) + fabsf(v[2 * i]), fabsf(u[2 * i + 1]) + fabsf(v[2 * i + 1])), bound2, half2);
                        nearest2(fma2(u2, c2[i], mul2(v2, ns2[i])), limit, nu[2 * i], nu[2 * i + 1], sure);
                        nearest2(fma2(v2, c2[i], mul2(u2, s2[i])), limit, nv[2 * i], nv[2 * i + 1], sure);
                    }
                    if (!sure) redo |= 1u << (2 * j + g);
                    if (inter) {
                        const uint32_t lo = pack4(nu[0], nv[0], nu[1], nv[1]), hi = pack4(nu[2], nv[2], nu[3], nv[3]);
                        if (g) { wb[0] = lo; wb[1] = hi; } else { wa[0] = lo; wa[1] = hi; }
                    } else {
                        wa[g] = pack4(nu[0], nu[1], nu[2], nu[3]);
                        wb[g] = pack4(nv[0], nv[1], nv[2], nv[3]);
                    }
                }
            }
            if (aligned || !turned) {
                *reinterpret_cast<uint2 *>(dst + dim_a) = make_uint2(wa[0], wa[1]);
                *reinterpret_cast<uint2 *>(dst + dim_b) = make_uint2(wb[0], wb[1]);
            } else {
                redo |= 3u << (2 * j);                        // a dim at a time
            }
        }
        src += stride;
        q_dst += (int64_t)a.Hq * a.d;
        slot = next_slot;
        raw_a = next_a; raw_b = next_b;
    }
    // What was next to a border, four pairs at a time (a dim at a time where items do not hold whole pairs).  Behind the loop: a
    // call in it, however rare, costs its registers.
    src -= (int64_t)tokens * stride;
    q_dst -= (int64_t)tokens * a.Hq * a.d;
    while (redo) {
        const int bit = __ffs(redo) - 1, j = bit >> 1, g = bit & 1;
        redo &= redo - 1;
        int8_t *const dst = kind == 0 ? q_dst + (int64_t)j * a.Hq * a.d : place(a.slots[t0 + j]);
        const T *const row = src + j * stride;
        const Turn &tn = turn[j];
        const double position = (double)a.positions[t0 + j];
        if (!aligned) {
#pragma unroll 1
            for (int e = 0; e < 8; ++e) {
                const int dim = (g ? dim_b : dim_a) + e;
                dst[dim] = code_of(row, dim, rot, inter, &tn, position, a.rope.freq, a.rope.scale, step);
            }
            continue;
        }
        const int chunk_g = g ? dim_b : dim_a, at = g ? at_b : at_a, first = inter ? chunk_g >> 1 : dim_a + 4 * g;
        float u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u[i] = to_float(row[inter ? chunk_g + 2 * i : dim_a + 4 * g + i]);
            v[i] = to_float(row[inter ? chunk_g + 2 * i + 1 : dim_b + 4 * g + i]);
        }
        int nu[4], nv[4];
        uint32_t unsure = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float c = tn.c[at + i], s = tn.s[at + i], limit = fmaf(fabsf(u[i]) + fabsf(v[i]), bound, 0.5f);
            const float du = nearest(__fmul_rn(fmaf(u[i], c, -__fmul_rn(v[i], s)), inv), nu[i]);
            const float dv = nearest(__fmul_rn(fmaf(v[i], c, __fmul_rn(u[i], s)), inv), nv[i]);
            unsure |= du < limit && dv < limit ? 0u : 1u << i;
        }
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
            if (!((unsure >> i) & 1)) continue;
            const float x = i == 0 ? u[0] : i == 1 ? u[1] : i == 2 ? u[2] : u[3], y = i == 0 ? v[0] : i == 1 ? v[1] : i == 2 ? v[2] : v[3];
            const uint32_t n2 = code_pair(x, y, position, a.rope.freq[first + i], a.rope.scale, step);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                nu[k] = k == i ? (int8_t)(n2 & 255) : nu[k];
                nv[k] = k == i ? (int8_t)(n2 >> 8) : nv[k];
            }
        }
        if (inter) {
            *reinterpret_cast<uint2 *>(dst + chunk_g) = make_uint2(pack4(nu[0], nv[0], nu[1], nv[1]), pack4(nu[2], nv[2], nu[3], nv[3]));
        } else {
            *reinterpret_cast<uint32_t *>(dst + dim_a + 4 * g) = pack4(nu[0], nu[1], nu[2], nu[3]);
            *reinterpret_cast<uint32_t *>(dst + dim_b + 4 * g) = pack4(nv[0], nv[1], nv[2], nv[3]);
        }
    }
}

// 16 bytes of the output: 8 or 4 codes of one head in their values, rounded to fp32 and then to T.  A byte becomes a float by
// its place in the mantissa of 2^23 (the converter would be four times slower than the stores).
template <typename T> __device__ __forceinline__ uint4 values16(const uint32_t *w, float step) {
    constexpr int kN = 16 / sizeof(T);
    float x[kN];
    const F2 bias = f2(-8388736.0f, -8388736.0f), step2 = f2(step, step);           // 2^23 + 128
#pragma unroll
    for (int i = 0; i < kN; i += 2) {
        const uint32_t u = w[i >> 2] ^ 0x80808080u;
        const F2 v = f2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7540 + (i & 3))), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7541 + (i & 3))));
        split(mul2(add2(v, bias), step2), x[i], x[i + 1]);
    }
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            o[i] = __float_as_uint(x[i]);
        } else if constexpr (std::is_same<T, __half>::value) {
            const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
            o[i] = *reinterpret_cast<const uint32_t *>(&h);
        } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            o[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// A thread owns 16 bytes of a token's row (head, dims and step worked out once) and walks over the CTA's tokens, four at a
// time with their loads together.  blockIdx.x: tokens; blockIdx.y: sequence; blockIdx.z: column group, of the keys first, then
// of the values.
constexpr int kReadBatch = 4;
template <typename T>
__global__ void __launch_bounds__(kThreads)
cache_read_kernel(const __grid_constant__ CacheReadArgs a, int columns, int group_columns, int groups, int per_cta) {
    constexpr int kN = 16 / sizeof(T);
    const int which = a.k_out ? (int)blockIdx.z / groups : 1;
    const int8_t *pool = which == 0 ? a.k_pages : a.v_pages;
    T *out = static_cast<T *>(which == 0 ? a.k_out : a.v_out);
    const int b = blockIdx.y;
    const int start = a.out_start[b];
    const int64_t want = (int64_t)a.out_start[b + 1] - start;
    int len = (int)max(min(want, min((int64_t)a.max_len, (int64_t)a.max_pages << a.page_shift)), (int64_t)0);
    if (start < 0 || start > a.rows) len = 0;
    else len = min(len, a.rows - start);
    if (blockIdx.x == 0 && threadIdx.x == 0 && len != want) atomicOr(a.status, STATUS_BAD_LENGTH);
    const int j0 = blockIdx.x * per_cta, j1 = min(j0 + per_cta, len);
    const int abreast = (int)blockDim.x / group_columns;                          // tokens side by side
    const int lane_token = (int)threadIdx.x / group_columns;
    const int column = (int)(blockIdx.z % groups) * group_columns + (int)threadIdx.x - lane_token * group_columns;
    if (lane_token >= abreast || column >= columns) return;
    const int per_head = a.d / kN, head = column / per_head, dim = (column - head * per_head) * kN;
    const float step = a.step[which * HCCS_MAX_CACHE_HEADS + head];
    const int32_t *table = a.page_table + (int64_t)b * a.max_pages;
    const int8_t *const mine = pool + ((int64_t)head << a.page_shift) * a.d + dim;
    const int64_t page_bytes = ((int64_t)a.Hkv << a.page_shift) * a.d;
    const int in_page = (1 << a.page_shift) - 1;
    T *dst = out + ((int64_t)start * a.Hkv) * a.d + column * kN;
    for (int j = j0 + lane_token; j < j1; j += abreast * kReadBatch) {
        int page[kReadBatch];
        uint32_t w[kReadBatch][kN / 4];
#pragma unroll
        for (int i = 0; i < kReadBatch; ++i) page[i] = __ldg(table + (min(j + i * abreast, j1 - 1) >> a.page_shift));
#pragma unroll
        for (int i = 0; i < kReadBatch; ++i) {
            const int jj = min(j + i * abreast, j1 - 1);
            const bool there = (uint32_t)page[i] < (uint32_t)a.num_pages;
            const int8_t *src = mine + (there ? page[i] : 0) * page_bytes + (jj & in_page) * a.d;
            if constexpr (kN == 8) {
                const uint2 v = __ldg(reinterpret_cast<const uint2 *>(src));
                w[i][0] = v.x;
                w[i][1] = v.y;
            } else {
                w[i][0] = __ldg(reinterpret_cast<const uint32_t *>(src));
            }
        }
#pragma unroll
        for (int i = 0; i < kReadBatch; ++i) {
            const int jj = j + i * abreast;
            if (jj >= j1) break;
            uint4 v = values16<T>(w[i], step);
            if ((uint32_t)page[i] >= (uint32_t)a.num_pages) {
                atomicOr(a.status, STATUS_BAD_PAGE);
                v = make_uint4(0, 0, 0, 0);
            }
            *reinterpret_cast<uint4 *>(dst + (int64_t)jj * a.Hkv * a.d) = v;
        }
    }
}

template <typename T>
cudaError_t write_typed(const CacheWriteArgs &a, cudaStream_t stream) {
    const int shift = a.d == 128 ? 3 : 2;
    const int items = (a.Hq + 2 * a.Hkv) << shift;
    // Whole warps: all items of a token in one CTA where they fit, else in equal parts; a step of a few tokens, which has
    // no other way to fill the SMs, in CTAs of 128.
    const bool few = (int64_t)a.T * items < 148 * kWriteThreads;
    const int groups = (items + (few ? 128 : kWriteThreads) - 1) / (few ? 128 : kWriteThreads);
    const int threads = ((items + groups - 1) / groups + 31) / 32 * 32;
    // Tokens per CTA: sixteen at most, and as many as make the waves of CTAs (24 warps per SM) come out even
    const int64_t slots = 148 * (2 * kWriteThreads / threads), all = (int64_t)a.T * groups;
    const int64_t waves = (all + slots * kTokens - 1) / (slots * kTokens);
    int per_cta = (int)((all + slots * waves - 1) / (slots * waves));
    per_cta = per_cta < 1 ? 1 : per_cta > kTokens ? kTokens : per_cta;
    cache_write_kernel<T><<<dim3((unsigned)((a.T + per_cta - 1) / per_cta), (unsigned)groups), threads, 0, stream>>>(a, items, shift, per_cta);
    return cudaGetLastError();
}

template <typename T>
cudaError_t read_typed(const CacheReadArgs &a, cudaStream_t stream) {
    const int columns = a.Hkv * a.d / (16 / (int)sizeof(T));                      // 16-byte pieces of a token's row
    const int groups = (columns + kThreads - 1) / kThreads;
    const int group_columns = (columns + groups - 1) / groups;
    const int abreast = kThreads / group_columns;
    const int threads = (abreast * group_columns + 31) / 32 * 32;
    // tokens per CTA: two batches, fewer where that leaves SMs without work
    const int z = groups * (a.k_out && a.v_out ? 2 : 1);
    int64_t per_cta = (int64_t)abreast * kReadBatch * 2;
    const int64_t spread = (int64_t)a.max_len * a.B * z / (8 * 148);
    if (per_cta > spread) per_cta = spread < abreast ? abreast : spread;
    const dim3 grid((unsigned)((a.max_len + per_cta - 1) / per_cta), (unsigned)a.B, (unsigned)z);
    cache_read_kernel<T><<<grid, threads, 0, stream>>>(a, columns, group_columns, groups, (int)per_cta);
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
