// HCCS attention over the int8 cache for single new tokens: the query heads of one kv head (up to 16) against its
// keys, split over the CTAs of a cluster.
//
// Bound: HBM.  Every key and value code is read once, 2*D bytes per key and kv head; a code takes part in at most
// 16 multiply-adds, which mma.sync (m16n8k32, int8) does while the loads of other warps are in flight.
//
// Two passes, because the clamp of the distance needs the row maximum first: over K (the logits stay in shared
// memory, one byte each), then over V.  A warp takes tiles of 32 keys; the order of the keys inside a tile is
// chosen so that the accumulators of Q.K^T a lane holds are exactly the bytes it owes to the A fragment of r.V, so
// logits never change lanes; K rows are B fragments as they are stored (16 bytes per lane, the order of the dims
// being the same for Q); V is transposed 4x4 bytes at a time by PRMTs.
// The CTAs of a cluster exchange their row maxima and at the end their sums through distributed shared memory:
// one launch, no workspace, and exact integers, so the split changes no bit.
#include <cooperative_groups.h>

#include "hccs_cached.cuh"

namespace hccs {

namespace {

namespace cg = cooperative_groups;

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kTileKeys = 32;

__device__ __forceinline__ void mma_s8(int (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }

// bytes 0..3 of a word that belong to keys below nb
__device__ __forceinline__ uint32_t byte_mask(int nb) { return nb >= 4 ? 0xffffffffu : nb <= 0 ? 0u : (1u << (8 * nb)) - 1u; }

// r of four logits (x + 128 per byte) in 16-bit pairs: max(xu - c, 0), c2 = -c in both lanes
__device__ __forceinline__ uint32_t closeness4(uint32_t w, uint32_t c2) {
    const uint32_t ev = __viaddmax_s16x2(w & 0x00ff00ffu, c2, 0u);
    const uint32_t od = __viaddmax_s16x2(prmt(w, 0, 0x4341), c2, 0u);
    return prmt(ev, od, 0x6240);
}

// D: head dim.  HI: more than 8 rows (the fragments' rows 8..15 are rows too; otherwise row 8 is all ones and
// collects sum V for nothing).
template <int D, bool HI>
__global__ void __launch_bounds__(kThreads, 2)
cached_decode_kernel(const __grid_constant__ CachedAttnArgs a, int row_tiles, int tiles_per_cta) {
    constexpr int kChunks = D / 64;            // 16-byte chunks of a K row per lane
    constexpr int kVWords = D / 32;            // words of a V row per lane: dims 4*kVWords*nn ...
    constexpr int kDims = 4 * kVWords;         // dims per lane and key, n tiles of r.V
    constexpr int kRows = HI ? 16 : 8;
    constexpr int kWords = HI ? 4 : 2;         // logit words per lane and tile
    constexpr int kStride = D + 8;             // row stride of the sums: rows on different banks
    extern __shared__ __align__(16) uint32_t xs[];                 // [tile][word][lane]
    __shared__ int sums[kRows + 1][kStride];                       // sum r V at [row][w*8 + nn]; last row: sum V
    __shared__ int row_max[kRows], row_sum[kRows + 1];             // last: keys seen
    __shared__ Requant rq_s[kRows];

    const int split = gridDim.x, rank = blockIdx.x;
    const int kvh = blockIdx.y / row_tiles, row0 = (blockIdx.y - kvh * row_tiles) * kRows;
    const int b = blockIdx.z;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c = lane & 3, nn = lane >> 2;
    const SequenceAt seq = sequence_at(a, b);
    if (seq.cut && tid == 0 && blockIdx.x + blockIdx.y == 0) atomicOr(a.status, STATUS_BAD_LENGTH);
    if (seq.nq == 0) return;                                       // the whole cluster
    // the new token sees the keys before it and, unless a tree mask hides it, itself
    int self = 1;
    if (a.tree_mask) self = a.tree_mask[(int64_t)seq.s0 * a.tree_words] & 1;
    const int n = min(max(seq.prefix + self, 0), seq.n);
    const int rows = min(kRows, a.group - row0);
    const int head0 = kvh * a.group + row0;
    const int32_t *table = a.page_table + (int64_t)b * a.max_pages;
    const int tiles = (n + kTileKeys - 1) / kTileKeys;
    // the sequence's own tiles, shared out evenly (tiles_per_cta bounds what shared memory holds)
    const int per = min((tiles + split - 1) / split, tiles_per_cta);
    const int tile0 = min(rank * per, tiles), tile1 = min(tile0 + per, tiles);

    for (int i = tid; i < (kRows + 1) * kStride; i += kThreads) (&sums[0][0])[i] = 0;
    if (tid == kRows) row_sum[kRows] = 0;
    if (tid < kRows) {
        row_max[tid] = -(1 << 30);
        row_sum[tid] = 0;
        rq_s[tid] = make_requant(tid < rows ? a.mult[head0 + tid] : 0, a.requant_shift);
    }
    // Q as A fragments: lane (nn, c) holds chunk c (and c + 4) of rows nn and nn + 8
    uint32_t qf[2 * kChunks][4];
    {
        const int8_t *q = a.Q + ((int64_t)seq.s0 * a.Hq + head0) * D;
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
            uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
            if (nn < rows) lo = *reinterpret_cast<const uint4 *>(q + nn * D + ch * 64 + c * 16);
            if (HI && nn + 8 < rows) hi = *reinterpret_cast<const uint4 *>(q + (nn + 8) * D + ch * 64 + c * 16);
            qf[2 * ch][0] = lo.x; qf[2 * ch][1] = hi.x; qf[2 * ch][2] = lo.y; qf[2 * ch][3] = hi.y;
            qf[2 * ch + 1][0] = lo.z; qf[2 * ch + 1][1] = hi.z; qf[2 * ch + 1][2] = lo.w; qf[2 * ch + 1][3] = hi.w;
        }
    }
    // Offset in a pool of the 16 keys half `hf` of a tile, and how many of them are seen.
    auto half_at = [&](int tile, int hf, int &seen) -> int64_t {
        const int key = tile * kTileKeys + 16 * hf;
        seen = min(max(n - key, 0), 16);
        if (seen == 0) return 0;
        const int page = __ldg(table + (key >> a.page_shift));
        if ((uint32_t)page >= (uint32_t)a.num_pages) {
            if (lane == 0) atomicOr(a.status, STATUS_BAD_PAGE);
            seen = 0;
            return 0;
        }
        return ((((int64_t)page * a.Hkv + kvh) << a.page_shift) + (key & ((1 << a.page_shift) - 1))) * D;
    };
    __syncthreads();
    const Requant rq0 = rq_s[nn], rq1 = HI ? rq_s[nn + 8] : rq_s[nn];

    // ---- pass over K
    int max0 = -(1 << 30), max1 = -(1 << 30);
    const int k_lane = (4 * (nn >> 1) + (nn & 1)) * D + c * 16;    // n tile t: + 2*D for odd t, half t / 2
    for (int tile = tile0 + warp; tile < tile1; tile += kWarps) {
        int seen[2];
        uint4 kr[4][kChunks];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int8_t *p = a.k_pages + half_at(tile, hf, seen[hf]) + k_lane;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int ch = 0; ch < kChunks; ++ch) kr[2 * hf + t][ch] = __ldg(reinterpret_cast<const uint4 *>(p + t * 2 * D + ch * 64));
        }
        int acc[4][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0;
#pragma unroll
            for (int ch = 0; ch < kChunks; ++ch) {
                mma_s8(acc[t], qf[2 * ch], kr[t][ch].x, kr[t][ch].y);
                mma_s8(acc[t], qf[2 * ch + 1], kr[t][ch].z, kr[t][ch].w);
            }
        }
        if (seen[0] + seen[1] < 32) {          // the last tile, or a bad page
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (4 * c + 2 * (t & 1) + e >= seen[t >> 1]) acc[t][e] = acc[t][2 + e] = -(1 << 30);
        }
        uint32_t *x = xs + (size_t)(tile - tile0) * (kWords * 32) + lane;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int(&p)[4] = acc[2 * hf], (&q)[4] = acc[2 * hf + 1];
            max0 = __vimax3_s32(__vimax3_s32(max0, p[0], p[1]), q[0], q[1]);
            x[hf * 32] = prmt(prmt(requant_top(rq0, p[0]), requant_top(rq0, p[1]), 0x0073),
                              prmt(requant_top(rq0, q[0]), requant_top(rq0, q[1]), 0x0073), 0x5410) ^ 0x80808080u;
            if (HI) {
                max1 = __vimax3_s32(__vimax3_s32(max1, p[2], p[3]), q[2], q[3]);
                x[(2 + hf) * 32] = prmt(prmt(requant_top(rq1, p[2]), requant_top(rq1, p[3]), 0x0073),
                                        prmt(requant_top(rq1, q[2]), requant_top(rq1, q[3]), 0x0073), 0x5410) ^ 0x80808080u;
            }
        }
    }
    max0 = max(max0, __shfl_xor_sync(~0u, max0, 1));
    max0 = max(max0, __shfl_xor_sync(~0u, max0, 2));
    if (c == 0) atomicMax(&row_max[nn], max0);
    if (HI) {
        max1 = max(max1, __shfl_xor_sync(~0u, max1, 1));
        max1 = max(max1, __shfl_xor_sync(~0u, max1, 2));
        if (c == 0) atomicMax(&row_max[nn + 8], max1);
    }

    // ---- the row maxima of the cluster; the first V tile is on its way meanwhile
    const int v_lane = 4 * c * D + nn * kDims;
    uint32_t vr[8][kVWords];
    int seen[2] = {0, 0};
    auto load_v = [&](int tile) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int8_t *p = a.v_pages + half_at(tile, hf, seen[hf]) + v_lane;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (kVWords == 4) {
                    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p + i * D));
                    vr[4 * hf + i][0] = v.x; vr[4 * hf + i][1] = v.y; vr[4 * hf + i][2] = v.z; vr[4 * hf + i][3] = v.w;
                } else {
                    const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p + i * D));
                    vr[4 * hf + i][0] = v.x; vr[4 * hf + i][1] = v.y;
                }
            }
        }
    };
    if (tile0 + warp < tile1) load_v(tile0 + warp);
    cg::cluster_group cluster = cg::this_cluster();
    int m0, m1 = 0;
    if (split > 1) {
        cluster.sync();
        m0 = -(1 << 30);
        m1 = -(1 << 30);
        for (int r = 0; r < split; ++r) {
            const int *other = cluster.map_shared_rank(row_max, r);
            m0 = max(m0, other[nn]);
            if (HI) m1 = max(m1, other[nn + 8]);
        }
    } else {
        __syncthreads();
        m0 = row_max[nn];
        if (HI) m1 = row_max[nn + 8];
    }
    // c = m + 128 - D per row, negated, in both 16-bit lanes
    auto neg_c = [&](const Requant &rq, int m, int row) -> uint32_t {
        const int top = ((int)requant_top(rq, m) >> 24) + 128;
        const int v = (row < rows ? a.table[head0 + row].D : 0) - top;
        return prmt((uint32_t)v, 0, 0x1010);
    };
    const uint32_t c0 = neg_c(rq0, m0, nn), c1 = HI ? neg_c(rq1, m1, nn + 8) : 0u;

    // ---- pass over V
    int acc[kDims][4];
#pragma unroll
    for (int w = 0; w < kDims; ++w) acc[w][0] = acc[w][1] = acc[w][2] = acc[w][3] = 0;
    int vsum[HI ? kDims : 1];
#pragma unroll
    for (int w = 0; w < (HI ? kDims : 1); ++w) vsum[w] = 0;
    int rs0 = 0, rs1 = 0, count = 0;
    for (int tile = tile0 + warp; tile < tile1; tile += kWarps) {
        const uint32_t *x = xs + (size_t)(tile - tile0) * (kWords * 32) + lane;
        const uint32_t k0 = byte_mask(seen[0] - 4 * c), k1 = byte_mask(seen[1] - 4 * c);
        count += seen[0] + seen[1];
        uint32_t rf[4];
        rf[0] = closeness4(x[0], c0) & k0;
        rf[2] = closeness4(x[32], c0) & k1;
        rs0 = __dp4a(rf[0], 0x01010101u, __dp4a(rf[2], 0x01010101u, (uint32_t)rs0));
        const uint32_t one0 = k0 & 0x01010101u, one1 = k1 & 0x01010101u;
        if (HI) {
            rf[1] = closeness4(x[64], c1) & k0;
            rf[3] = closeness4(x[96], c1) & k1;
            rs1 = __dp4a(rf[1], 0x01010101u, __dp4a(rf[3], 0x01010101u, (uint32_t)rs1));
        } else {
            rf[1] = nn == 0 ? one0 : 0u;
            rf[3] = nn == 0 ? one1 : 0u;
        }
#pragma unroll
        for (int q = 0; q < kVWords; ++q) {
            uint32_t o[2][4];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const uint32_t w0 = vr[4 * hf][q], w1 = vr[4 * hf + 1][q], w2 = vr[4 * hf + 2][q], w3 = vr[4 * hf + 3][q];
                const uint32_t t0 = prmt(w0, w1, 0x5140), t1 = prmt(w2, w3, 0x5140);
                const uint32_t t2 = prmt(w0, w1, 0x7362), t3 = prmt(w2, w3, 0x7362);
                o[hf][0] = prmt(t0, t1, 0x5410); o[hf][1] = prmt(t0, t1, 0x7632);
                o[hf][2] = prmt(t2, t3, 0x5410); o[hf][3] = prmt(t2, t3, 0x7632);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mma_s8(acc[4 * q + j], rf, o[0][j], o[1][j]);
                if constexpr (HI) vsum[4 * q + j] = __dp4a((int)o[0][j], (int)one0, __dp4a((int)o[1][j], (int)one1, vsum[4 * q + j]));
            }
        }
        if (tile + kWarps < tile1) load_v(tile + kWarps);
    }

    // ---- the CTA's sums in shared memory: column of n tile w is nn' = 2c + e, dim kDims*nn' + w
#pragma unroll
    for (int w = 0; w < kDims; ++w)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int at = w * 8 + 2 * c + e;
            atomicAdd(&sums[nn][at], acc[w][e]);
            if (HI) atomicAdd(&sums[nn + 8][at], acc[w][2 + e]);
            else if (nn == 0) atomicAdd(&sums[kRows][at], acc[w][2 + e]);
        }
    if constexpr (HI) {
#pragma unroll
        for (int w = 0; w < kDims; ++w) {
            int v = vsum[w];
            v += __shfl_xor_sync(~0u, v, 1);
            v += __shfl_xor_sync(~0u, v, 2);
            if (c == 0) atomicAdd(&sums[kRows][w * 8 + nn], v);
        }
        rs1 += __shfl_xor_sync(~0u, rs1, 1);
        rs1 += __shfl_xor_sync(~0u, rs1, 2);
        if (c == 0) atomicAdd(&row_sum[nn + 8], rs1);
    }
    rs0 += __shfl_xor_sync(~0u, rs0, 1);
    rs0 += __shfl_xor_sync(~0u, rs0, 2);
    if (c == 0) atomicAdd(&row_sum[nn], rs0);
    if (lane == 0) atomicAdd(&row_sum[kRows], count);
    if (split > 1) cluster.sync(); else __syncthreads();

    // ---- join: a thread finishes four dims of a row, the rows and dims shared out over the cluster
    for (int i = rank * kThreads + tid; i < rows * (D / 4); i += split * kThreads) {
        const int row = i / (D / 4), dim = (i % (D / 4)) * 4;
        int rv[4] = {0, 0, 0, 0}, vs[4] = {0, 0, 0, 0}, rs = 0, keys = 0;
        for (int r = 0; r < split; ++r) {
            const int *so = split > 1 ? cluster.map_shared_rank(&sums[0][0], r) : &sums[0][0];
            const int *ro = split > 1 ? cluster.map_shared_rank(row_sum, r) : row_sum;
            rs += ro[row];
            keys += ro[kRows];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = ((dim + e) % kDims) * 8 + (dim + e) / kDims;
                rv[e] += so[row * kStride + at];
                vs[e] += so[kRows * kStride + at];
            }
        }
        const int h = head0 + row;
        const HeadEntry th = a.table[h];
        const int64_t F = th.B - th.S * th.D;
        const int64_t Z = F * keys + (int64_t)th.S * rs;
        int64_t num[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] = F * vs[e] + (int64_t)th.S * rv[e];
        store_output4(a, ((int64_t)seq.s0 * a.Hq + h) * D + dim, num, row_factor(a, Z, a.scale[h]));
    }
    if (split > 1) cluster.sync();             // nobody leaves while its sums are read
}

template <int D, bool HI>
cudaError_t launch_typed(const CachedAttnArgs &a, cudaStream_t stream) {
    constexpr int kRows = HI ? 16 : 8;
    const int row_tiles = (a.group + kRows - 1) / kRows;
    const int tiles = (a.max_kv + kTileKeys - 1) / kTileKeys;
    const int64_t groups = (int64_t)a.B * a.Hkv * row_tiles;
    // Clusters large enough that about two CTAs per SM have work, as long as every warp keeps a tile; and so large
    // that the logits of a CTA's keys fit its shared memory (16 bytes a key at most: 8192 keys of 131072).
    const size_t tile_bytes = (HI ? 4 : 2) * 128;
    int split = 1;
    while (split < 16 && (((groups * split < 2 * 148) && tiles > split * kWarps) || (size_t)((tiles + split - 1) / split) * tile_bytes > 96 * 1024)) split *= 2;
    const int per = (tiles + split - 1) / split;
    const size_t smem = (size_t)per * tile_bytes;
    auto kernel = cached_decode_kernel<D, HI>;
    static bool raised[64] = {};
    const cudaError_t e = raise_limits((const void *)kernel, 160 * 1024, raised);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)split, (unsigned)(a.Hkv * row_tiles), (unsigned)a.B);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)split;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, row_tiles, per);
}

}  // namespace

cudaError_t launch_cached_decode(const CachedAttnArgs &a, cudaStream_t stream) {
    if (a.d == 128) return a.group > 8 ? launch_typed<128, true>(a, stream) : launch_typed<128, false>(a, stream);
    return a.group > 8 ? launch_typed<64, true>(a, stream) : launch_typed<64, false>(a, stream);
}

}  // namespace hccs
