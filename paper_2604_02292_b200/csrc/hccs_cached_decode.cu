// HCCS attention over the int8 cache for single new tokens: the query heads of one kv head (up to 16) against its
// keys, split over the CTAs of a cluster.
//
// Bound: HBM.  Every key and value code is read once, 2*D bytes per key and kv head; a code takes part in at most
// 16 multiply-adds, which mma.sync (m16n8k32, int8) does while the loads are in flight.  64 sequences of 8192 keys (32
// query heads on 8 of 128): 162 us, 6.6 TB/s; 32 of 4096: 45 us, 6.0 TB/s.  One sequence of 131072 keys (8 kv heads):
// 60 us, 4.5 TB/s, on 80 CTAs of sixteen warps: the two passes need all of a row's maxima, so a kv head has one cluster,
// and of clusters of more than ten CTAs the device does not hold eight at a time.  Groups of more than 16 query heads read
// the codes once per 16: 64 sequences of 8192 keys, one kv head, 16, 32, 64, 128 query heads: 36, 63, 120, 211 us.
//
// Two passes, because the clamp of the distance needs the row maximum first: over K (the logits stay in shared
// memory, one byte each), then over V.  A warp takes tiles of 32 keys; the order of the keys inside a tile is
// chosen so that the accumulators of Q.K^T a lane holds are exactly the bytes it owes to the A fragment of r.V, so
// logits never change lanes; K rows are B fragments as they are stored (16 bytes per lane, the order of the dims
// being the same for Q); V is transposed 4x4 bytes at a time by PRMTs.  Every warp has a ring of its own that its lane 0
// fills by TMA (a box per page or per tile), K tiles first and then V tiles in one sequence, so V is on its way while the
// maxima are exchanged.  (On 268 MB the same ring filled by 16-byte cp.async took 69 us, stalled in the load/store unit; loads
// straight to registers, a tile in flight per warp, 50 us; this 45.)
// The CTAs of a cluster take tiles in turn, push their row maxima to each other between the passes and their sums to
// the CTA that finishes a dim at the end, through distributed shared memory: one launch, no workspace, and exact
// integers, so the split changes no bit.
#include <math.h>

#include "hccs_cached.cuh"

namespace hccs {

namespace {

constexpr int kTileKeys = 32;
constexpr int kDepth = 2;                  // tiles on their way per warp

__device__ __forceinline__ void mma_s8(int (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// the address of `p` in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t remote(const void *p, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void push(uint32_t dst, int v) { asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(dst), "r"(v) : "memory"); }
__device__ __forceinline__ void push4(uint32_t dst, const int4 &v) {
    asm volatile("st.shared::cluster.v4.s32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// bytes 0..3 of a word that belong to keys below nb
__device__ __forceinline__ uint32_t byte_mask(int nb) { return nb >= 4 ? 0xffffffffu : nb <= 0 ? 0u : (1u << (8 * nb)) - 1u; }

// r of four logits (x + 128 per byte) in 16-bit pairs: max(xu - c, 0), c2 = -c in both lanes
__device__ __forceinline__ uint32_t closeness4(uint32_t w, uint32_t c2) {
    const uint32_t ev = __viaddmax_s16x2(w & 0x00ff00ffu, c2, 0u);
    const uint32_t od = __viaddmax_s16x2(prmt(w, 0, 0x4341), c2, 0u);
    return prmt(ev, od, 0x6240);
}

// W: warps per CTA, 8 or 16
template <int D, bool HI, int W>
struct Sizes {
    static constexpr int kWarps = W;
    static constexpr int kRows = HI ? 16 : 8;
    static constexpr int kTileBytes = kTileKeys * D;
    static constexpr int kRing = kWarps * kDepth * kTileBytes;     // bytes of copies on their way
    static constexpr int kPitch = D + 16;                          // words between the rows of a warp's sums
    static constexpr int kSums = kWarps * (kRows + 1) * kPitch * 4;
    // the sums take the place of ring and logits once both passes are through
    // per tile of keys a byte per logit and row, and the keys seen
    static constexpr size_t smem(int tiles, int rows) {
        const size_t passes = (size_t)kRing + (size_t)tiles * (kTileKeys * (rows < kRows ? rows : kRows) + 4);
        return 1024 + (passes > (size_t)kSums ? passes : (size_t)kSums);
    }
};


// D: head dim.  HI: more than 8 rows (the fragments' rows 8..15 are rows too; otherwise row 8 is all ones and
// collects sum V for nothing).  tiles_per_warp bounds what shared memory holds.
// CROSS: queries on an encoder's states.  The rows of a kv head are its (query, head) pairs, all of which see the same keys:
// those of the sequence, or where max_q is 1 those of the query's key range.  Up to `merge` neighbouring sequences of one query that read the
// same states (hypotheses about one input) are rows of one CTA too, that of the first of them, where launch_typed leaves room for them: 32
// queries, two by two on the same states of up to 1499 keys (16 heads of 64), in 14.4 us instead of 20.5 (12.0 to 12.4 since kernels overlap).
// 8 queries on 32768 keys (32 heads on 8 of 128): 84 to 90 us, 6.0 to 6.4 TB/s.
template <int D, bool HI, int W, bool CROSS>
__global__ void __launch_bounds__(32 * W, 16 / W)
cached_decode_kernel(const __grid_constant__ CachedAttnArgs a, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, int row_tiles, int tiles_per_warp, int merge) {
    using S = Sizes<D, HI, W>;
    constexpr int kWarps = W, kThreads = 32 * W;
    constexpr int kChunks = D / 64;            // 16-byte chunks of a K row per lane
    constexpr int kVWords = D / 32;            // words of a V row per lane: dims 4*kVWords*nn ...
    constexpr int kDims = 4 * kVWords;         // dims per lane and key, n tiles of r.V
    constexpr int kRows = S::kRows, kPitch = S::kPitch;
    constexpr int kQuads = D / 4;
    extern __shared__ uint8_t smem_raw[];
    __shared__ int row_max[kRows], row_sum[kRows + 1];             // row_sum, last: keys seen
    __shared__ int all_max[kMaxSplit][kRows], all_sum[kMaxSplit][kRows + 1];       // of every CTA of the cluster
    __shared__ int4 all_quads[(kQuads + kMaxSplit - 1) * (kRows + 1)];             // [CTA][this CTA's quad of dims][row; last: sum V]
    __shared__ Requant rq_s[kRows];
    __shared__ __align__(8) uint64_t full[kWarps][kDepth];
    __shared__ int abort_flag;

    const int split = gridDim.x, rank = blockIdx.x;
    const int kvh = blockIdx.y / row_tiles, row0 = (blockIdx.y - kvh * row_tiles) * kRows;
    const int b = blockIdx.z;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c = lane & 3, nn = lane >> 2;
    uint8_t *const smem = smem_raw + (((smem_u32(smem_raw) + 1023u) & ~1023u) - smem_u32(smem_raw));      // (the swizzles count from there)
    if (tid == 0) abort_flag = 0;
    if (!CROSS && split > 1) cluster_arrive(); // the other CTAs run: waited for before the first push
    if constexpr (CROSS) previous_kernel_done();
    const int32_t *table = CROSS ? nullptr : a.page_table + (int64_t)b * a.max_pages;
    // tiles in turn to the warps of the cluster: the first does not depend on the length
    const int first = rank * kWarps + warp, stride = kWarps * split;
    auto page_at = [&](int key) -> int {
        if constexpr (CROSS) return 0;
        return (key >> a.page_shift) < a.max_pages ? __ldg(table + (key >> a.page_shift)) : -1;
    };
    int page[2] = {page_at(first * kTileKeys), page_at(first * kTileKeys + 16)};
    const SequenceAt seq = sequence_at<CROSS>(a, b);
    int together = 1;                          // sequences
    if (CROSS && merge > 1) {
        // blocks of `merge` sequences: in a block, those with the states of the one before them leave
        const int from = b - b % merge, other = min(from + min(lane, merge - 1), a.B - 1);
        const int ks = a.k_start[other], kl = a.kv_len[other];
        const int mine = __shfl_sync(~0u, ks, b - from), keys = __shfl_sync(~0u, kl, b - from);
        const uint32_t same = __ballot_sync(~0u, lane < merge && from + lane < a.B && ks == mine && kl == keys) >> (b - from);
        const bool follows = __shfl_sync(~0u, (int)(ks == mine && kl == keys), max(b - from - 1, 0)) && b > from;
        if (follows) {
            if (seq.cut && tid == 0 && blockIdx.x + blockIdx.y == 0) atomicOr(a.status, STATUS_BAD_LENGTH);
            return;                            // (the whole cluster)
        }
        together = same == ~0u ? 32 : __ffs(~same) - 1;
    }
    if (CROSS && split > 1) cluster_arrive();
    const int rows = !CROSS ? min(kRows, a.group - row0) : merge > 1 ? together * a.group : min(kRows, min(seq.nq, a.max_q) * a.group - row0);
    const int head0 = kvh * a.group + row0;
    // the row's token, or -1: its sequence has none
    auto token_of = [&](int row) -> int {
        if (!CROSS || merge <= 1) return seq.nq <= 0 ? -1 : seq.s0 + (CROSS ? (row0 + row) / a.group : 0);
        const int at = b + row / a.group, s0 = min(max(a.q_start[at], 0), a.T);
        return min(a.q_start[at + 1], a.T) > s0 ? s0 : -1;
    };
    auto head_of = [&](int row) -> int { return CROSS ? kvh * a.group + (row0 + row) % a.group : head0 + row; };
    if (seq.cut && tid == 0 && blockIdx.x + blockIdx.y == 0) atomicOr(a.status, STATUS_BAD_LENGTH);
    // the new token sees the keys before it and, unless a tree mask hides it, itself
    int self = 1;
    if (a.tree_mask && seq.nq > 0) self = a.tree_mask[(int64_t)seq.s0 * a.tree_words] & 1;
    int n = CROSS ? seq.n : min(max(seq.prefix + self, 0), seq.n), k0 = seq.k0;
    if (CROSS && a.key_range && seq.nq > 0) {
        const int2 r = range_of(a, seq, 0);
        n = r.y - r.x;
        k0 += r.x;
    }
    const int tiles = (seq.nq > 0 || (CROSS && merge > 1)) && rows > 0 ? (n + kTileKeys - 1) / kTileKeys : 0;
    const int mine = min(first < tiles ? (tiles - first + stride - 1) / stride : 0, tiles_per_warp);

    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * kDepth * S::kTileBytes);
    // logits of a tile: [half of its keys][row, four words of four keys each]; a lane whose row is none has no place
    const int max_rows = min(kRows, CROSS ? a.max_q * a.group * merge : a.group), x_half = 4 * max_rows, x_tile = 2 * x_half;
    uint32_t *const xs = reinterpret_cast<uint32_t *>(smem + S::kRing) + warp * x_tile + lane;               // + tile * kWarps * x_tile
    uint32_t *const seen_s = reinterpret_cast<uint32_t *>(smem + S::kRing) + (size_t)tiles_per_warp * kWarps * x_tile + warp;   // + tile * kWarps
    const bool has0 = nn < max_rows, has1 = HI && nn + 8 < max_rows;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < kDepth; ++i) mbar_init(smem_u32(&full[warp][i]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncwarp();
    // Copy number x of this warp: K tiles 0 .. mine-1, then V tiles; a box per 16 or 32 keys, those that are not there or whose
    // page is not left out (what the place held is finite, and their logits are masked).
    const int boxes = !CROSS && a.page_shift < 5 ? 2 : 1;
    auto copy = [&](int x) {
        if (lane != 0) return;
        const bool values = x >= mine;
        const int key = (first + (values ? x - mine : x) * stride) * kTileKeys;
        const uint32_t dst = ring + (x % kDepth) * S::kTileBytes, bar = smem_u32(&full[warp][x % kDepth]);
        const CUtensorMap *map = values ? &map_v : &map_k;
        if constexpr (CROSS) {                 // (keys behind the last one seen are some other's, or zeros behind all of them)
            mbar_expect_tx(bar, (uint32_t)S::kTileBytes);
            tma_load_3d(dst, map, 0, kvh, k0 + key, bar);
            return;
        }
        const bool r0 = (uint32_t)page[0] < (uint32_t)a.num_pages, r1 = boxes == 2 && key + 16 < n && (uint32_t)page[1] < (uint32_t)a.num_pages;
        mbar_expect_tx(bar, (uint32_t)((r0 ? 1 : 0) + (r1 ? 1 : 0)) * (S::kTileBytes / boxes));
        if (r0) tma_load_3d(dst, map, 0, key & ((1 << a.page_shift) - 1), page[0] * a.Hkv + kvh, bar);
        if (r1) tma_load_3d(dst + S::kTileBytes / 2, map, 0, 0, page[1] * a.Hkv + kvh, bar);
    };
    bool ok = true;
    auto landed = [&](int x) {
        ok = __all_sync(~0u, mbar_wait(smem_u32(&full[warp][x % kDepth]), (x / kDepth) & 1, &abort_flag, a.status, a.wait_cycles));
        if (!ok)       // given up: the copies on their way (this one and the next) land before the CTA may leave, again with a limit
            for (int y = x; y < min(x + kDepth, 2 * mine); ++y) mbar_wait_bounded(smem_u32(&full[warp][y % kDepth]), (y / kDepth) & 1, a.wait_cycles);
    };
    // Row r of a tile is swizzled over its D bytes: 16-byte chunk ch sits at ch ^ (r & 7), or ch ^ (r / 2 & 3) for D = 64.  Of K a
    // lane reads chunk c (and c + 4) of keys 16*half + 4*(nn/2) + 2*(t & 1) + (nn & 1), n tile t; of V, dims kDims*nn ... of
    // keys 16*half + 4c + i.
    auto chunk_at = [&](int r, int ch) -> uint32_t { return (uint32_t)(r * D + ((ch ^ (D == 128 ? r & 7 : (r >> 1) & 3)) << 4)); };
    const int k_row = 4 * (nn >> 1) + (nn & 1);
    auto look_up = [&](int x) {                // the pages of copy x
        if (x >= 2 * mine) return;
        const int key = (first + (x >= mine ? x - mine : x) * stride) * kTileKeys;
        page[0] = page_at(key);
        page[1] = page_at(key + 16);
    };
    // keys of the halves of tile number i that are seen, as they were when its K was copied
    uint32_t seen_next[kDepth];
    auto seen_of = [&](int i) -> uint32_t {
        const int key = (first + i * stride) * kTileKeys;
        uint32_t s = 0;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            int v = min(max(n - key - 16 * hf, 0), 16);
            if (!CROSS && v > 0 && (uint32_t)page[hf] >= (uint32_t)a.num_pages) {
                if (lane == 0) atomicOr(a.status, STATUS_BAD_PAGE);
                v = 0;
            }
            s |= (uint32_t)v << (8 * hf);
        }
        return s;
    };
#pragma unroll
    for (int x = 0; x < kDepth; ++x) {
        seen_next[x] = 0;
        if (x < 2 * mine) {
            if (x < mine) seen_next[x] = seen_of(x);
            copy(x);
            look_up(x + 1);
        }
    }

    if (tid == kRows) row_sum[kRows] = 0;
    if (tid < kRows) {
        row_max[tid] = kNone;
        row_sum[tid] = 0;
        rq_s[tid] = make_requant(tid < rows ? a.mult[head_of(tid)] : 0, a.requant_shift);
    }
    // Q as A fragments: lane (nn, c) holds chunk c (and c + 4) of rows nn and nn + 8
    uint32_t qf[2 * kChunks][4];
    {
        auto q = [&](int row) -> const int8_t * {          // NULL: no such row, or nothing to see
            const int token = row < rows && mine > 0 ? token_of(row) : -1;
            return token < 0 ? nullptr : a.Q + ((int64_t)token * a.Hq + head_of(row)) * D;
        };
        const int8_t *const q0 = q(nn), *const q1 = HI ? q(nn + 8) : nullptr;
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
            uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
            if (q0) lo = *reinterpret_cast<const uint4 *>(q0 + ch * 64 + c * 16);
            if (q1) hi = *reinterpret_cast<const uint4 *>(q1 + ch * 64 + c * 16);
            qf[2 * ch][0] = lo.x; qf[2 * ch][1] = hi.x; qf[2 * ch][2] = lo.y; qf[2 * ch][3] = hi.y;
            qf[2 * ch + 1][0] = lo.z; qf[2 * ch + 1][1] = hi.z; qf[2 * ch + 1][2] = lo.w; qf[2 * ch + 1][3] = hi.w;
        }
    }
    __syncthreads();
    const Requant rq0 = rq_s[nn], rq1 = HI ? rq_s[nn + 8] : rq_s[nn];

    // ---- pass over K
    int max0 = kNone, max1 = kNone;
    for (int i = 0; i < mine; ++i) {
        landed(i);
        if (!ok) break;
        const uint32_t src = ring + (i % kDepth) * S::kTileBytes;
        const uint32_t seen = seen_next[0];
        int acc[4][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0;
#pragma unroll
            for (int ch = 0; ch < kChunks; ++ch) {
                uint32_t k0, k1, k2, k3;
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(k0), "=r"(k1), "=r"(k2), "=r"(k3) : "r"(src + chunk_at(k_row + 2 * (t & 1) + 16 * (t >> 1), c + 4 * ch)) : "memory");
                mma_s8(acc[t], qf[2 * ch], k0, k1);
                mma_s8(acc[t], qf[2 * ch + 1], k2, k3);
            }
        }
        const int s0 = (int)(seen & 255u), s1 = (int)(seen >> 8);
        if (s0 + s1 < 32) {                    // the last tile, or a bad page
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (4 * c + 2 * (t & 1) + e >= (t < 2 ? s0 : s1)) acc[t][e] = acc[t][2 + e] = kNone;
        }
        uint32_t *x = xs + i * (kWarps * x_tile);
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int(&p)[4] = acc[2 * hf], (&q)[4] = acc[2 * hf + 1];
            max0 = __vimax3_s32(__vimax3_s32(max0, p[0], p[1]), q[0], q[1]);
            const uint32_t w0 = prmt(prmt(requant_top(rq0, p[0]), requant_top(rq0, p[1]), 0x0073),
                                     prmt(requant_top(rq0, q[0]), requant_top(rq0, q[1]), 0x0073), 0x5410) ^ 0x80808080u;
            if (has0) x[hf * x_half] = w0;
            if (HI) {
                max1 = __vimax3_s32(__vimax3_s32(max1, p[2], p[3]), q[2], q[3]);
                const uint32_t w1 = prmt(prmt(requant_top(rq1, p[2]), requant_top(rq1, p[3]), 0x0073),
                                         prmt(requant_top(rq1, q[2]), requant_top(rq1, q[3]), 0x0073), 0x5410) ^ 0x80808080u;
                if (has1) x[hf * x_half + 32] = w1;
            }
        }
        if (lane == 0) seen_s[i * kWarps] = seen;
        // the words of this tile are in registers: its place takes the next copy
#pragma unroll
        for (int d = 0; d + 1 < kDepth; ++d) seen_next[d] = seen_next[d + 1];
        if (i + kDepth < mine) seen_next[kDepth - 1] = seen_of(i + kDepth);
        __syncwarp();
        if (i + kDepth < 2 * mine) copy(i + kDepth);
        look_up(i + kDepth + 1);
    }
    max0 = max(max0, __shfl_xor_sync(~0u, max0, 1));
    max0 = max(max0, __shfl_xor_sync(~0u, max0, 2));
    if (c == 0) atomicMax(&row_max[nn], max0);
    if (HI) {
        max1 = max(max1, __shfl_xor_sync(~0u, max1, 1));
        max1 = max(max1, __shfl_xor_sync(~0u, max1, 2));
        if (c == 0) atomicMax(&row_max[nn + 8], max1);
    }

    // ---- the row maxima of the cluster
    __syncthreads();
    int m0, m1 = 0;
    if (split > 1) {
        cluster_wait();                        // every CTA has started
        if (tid < split * kRows) push(remote(&all_max[rank][tid % kRows], tid / kRows), row_max[tid % kRows]);
        cluster_arrive();
        cluster_wait();
        m0 = m1 = kNone;
        for (int r = 0; r < split; ++r) {
            m0 = max(m0, all_max[r][nn]);
            if (HI) m1 = max(m1, all_max[r][nn + 8]);
        }
    } else {
        m0 = row_max[nn];
        if (HI) m1 = row_max[nn + 8];
    }
    // c = m + 128 - D per row, negated, in both 16-bit lanes
    auto neg_c = [&](const Requant &rq, int m, int row) -> uint32_t {
        const int top = ((int)requant_top(rq, m) >> 24) + 128;
        const int v = (row < rows ? a.table[head_of(row)].D : 0) - top;
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
    for (int i = 0; ok && i < mine; ++i) {
        landed(mine + i);
        if (!ok) break;
        const uint32_t src = ring + ((mine + i) % kDepth) * S::kTileBytes;
        const uint32_t *x = xs + i * (kWarps * x_tile);
        const uint32_t seen = seen_s[i * kWarps];
        const int s0 = (int)(seen & 255u), s1 = (int)(seen >> 8);
        const uint32_t k0 = byte_mask(s0 - 4 * c), k1 = byte_mask(s1 - 4 * c);
        count += s0 + s1;
        uint32_t rf[4];
        rf[0] = has0 ? closeness4(x[0], c0) & k0 : 0u;
        rf[2] = has0 ? closeness4(x[x_half], c0) & k1 : 0u;
        rs0 = __dp4a(rf[0], 0x01010101u, __dp4a(rf[2], 0x01010101u, (uint32_t)rs0));
        const uint32_t one0 = k0 & 0x01010101u, one1 = k1 & 0x01010101u;
        if (HI) {
            rf[1] = has1 ? closeness4(x[32], c1) & k0 : 0u;
            rf[3] = has1 ? closeness4(x[x_half + 32], c1) & k1 : 0u;
            rs1 = __dp4a(rf[1], 0x01010101u, __dp4a(rf[3], 0x01010101u, (uint32_t)rs1));
        } else {
            rf[1] = nn == 0 ? one0 : 0u;
            rf[3] = nn == 0 ? one1 : 0u;
        }
        uint32_t vr[8][kVWords];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int r = 16 * (k >> 2) + 4 * c + (k & 3);
            if constexpr (kVWords == 4)
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(vr[k][0]), "=r"(vr[k][1]), "=r"(vr[k][2]), "=r"(vr[k][3]) : "r"(src + chunk_at(r, nn)) : "memory");
            else
                asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(vr[k][0]), "=r"(vr[k][1]) : "r"(src + chunk_at(r, nn >> 1) + (nn & 1) * 8) : "memory");
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
        __syncwarp();
        if (i + kDepth < mine) copy(mine + i + kDepth);
        look_up(mine + i + kDepth + 1);
    }
    __syncthreads();                           // ring and logits are done with: the sums take their place

    // ---- the warps' sums, as quads of dims: the accumulators of n tile w and column nn' = 2c + e are dim kDims*nn' + w.
    // Quad q sits at q ^ ((q >> 3) & 3): the four lanes of a row write to different banks
    {
        int *const slab = reinterpret_cast<int *>(smem) + warp * (kRows + 1) * kPitch;
        auto put = [&](int row, int quad, int x0, int x1, int x2, int x3) {
            *reinterpret_cast<int4 *>(slab + row * kPitch + 4 * (quad ^ ((quad >> 3) & 3))) = make_int4(x0, x1, x2, x3);
        };
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int k = 0; k < kVWords; ++k) {
                const int quad = kVWords * (2 * c + e) + k;
                put(nn, quad, acc[4 * k][e], acc[4 * k + 1][e], acc[4 * k + 2][e], acc[4 * k + 3][e]);
                if (HI) put(nn + 8, quad, acc[4 * k][2 + e], acc[4 * k + 1][2 + e], acc[4 * k + 2][2 + e], acc[4 * k + 3][2 + e]);
                else if (nn == 0) put(kRows, quad, acc[4 * k][2 + e], acc[4 * k + 1][2 + e], acc[4 * k + 2][2 + e], acc[4 * k + 3][2 + e]);
            }
        if constexpr (HI) {
#pragma unroll
            for (int w = 0; w < kDims; ++w) {
                vsum[w] += __shfl_xor_sync(~0u, vsum[w], 1);
                vsum[w] += __shfl_xor_sync(~0u, vsum[w], 2);
            }
            if (c == 0) {
#pragma unroll
                for (int k = 0; k < kVWords; ++k) put(kRows, kVWords * nn + k, vsum[4 * k], vsum[4 * k + 1], vsum[4 * k + 2], vsum[4 * k + 3]);
            }
            rs1 += __shfl_xor_sync(~0u, rs1, 1);
            rs1 += __shfl_xor_sync(~0u, rs1, 2);
            if (c == 0) atomicAdd(&row_sum[nn + 8], rs1);
        }
        rs0 += __shfl_xor_sync(~0u, rs0, 1);
        rs0 += __shfl_xor_sync(~0u, rs0, 2);
        if (c == 0) atomicAdd(&row_sum[nn], rs0);
        if (lane == 0) atomicAdd(&row_sum[kRows], count);
    }
    __syncthreads();
    // the CTA's sums to the CTA that finishes their dims: quad q is CTA q % split's number q / split
    const int own = (kQuads + split - 1) / split;
    for (int i = tid; i < kQuads * (kRows + 1); i += kThreads) {
        const int row = i / kQuads, quad = i % kQuads;
        int4 v = make_int4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const int4 p = *reinterpret_cast<const int4 *>(reinterpret_cast<const int *>(smem) + (w * (kRows + 1) + row) * kPitch + 4 * (quad ^ ((quad >> 3) & 3)));
            v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
        }
        int4 *dst = &all_quads[(rank * own + quad / split) * (kRows + 1) + row];
        if (split > 1) push4(remote(dst, quad % split), v); else *dst = v;
    }
    if (split > 1) {
        for (int i = tid; i < split * (kRows + 1); i += kThreads) push(remote(&all_sum[rank][i % (kRows + 1)], i / (kRows + 1)), row_sum[i % (kRows + 1)]);
        cluster_arrive();
        cluster_wait();                        // nobody writes here any more, and nobody else is written to
    } else {
        if (tid <= kRows) all_sum[0][tid] = row_sum[tid];
        __syncthreads();
    }

    // ---- join: a thread finishes four dims of a row
    if (seq.nq > 0 || (CROSS && merge > 1))
        for (int i = tid; i < rows * own; i += kThreads) {
            const int row = i / own, q = i % own;
            if (q * split + rank >= kQuads) continue;
            const int token = token_of(row);
            if (token < 0) continue;
            int rv[4] = {0, 0, 0, 0}, vs[4] = {0, 0, 0, 0}, rs = 0, keys = 0;
            for (int r = 0; r < split; ++r) {
                const int4 p = all_quads[(r * own + q) * (kRows + 1) + row], s = all_quads[(r * own + q) * (kRows + 1) + kRows];
                rv[0] += p.x; rv[1] += p.y; rv[2] += p.z; rv[3] += p.w;
                vs[0] += s.x; vs[1] += s.y; vs[2] += s.z; vs[3] += s.w;
                rs += all_sum[r][row];
                keys += all_sum[r][kRows];
            }
            const int h = head_of(row);
            const HeadEntry th = a.table[h];
            const int64_t F = th.B - th.S * th.D;
            int64_t num[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) num[e] = F * vs[e] + (int64_t)th.S * rv[e];
            store_output4(a, ((int64_t)token * a.Hq + h) * D + 4 * (q * split + rank), num, row_factor(a, F * keys + (int64_t)th.S * rs, a.scale[h]));
        }
}

constexpr size_t kMaxSmem = 210 * 1024;    // dynamic; the kernel's own arrays take up to 16 KB more
constexpr size_t kHalfSmem = 98 * 1024;    // two CTAs per SM

struct Plan { int split, per_warp; double cost; };      // cost: infinite where no cluster size has the shared memory

// What a launch with W warps per CTA and clusters of `s` costs, in microseconds: waves of clusters, each the time of a CTA's
// share of a kv head's codes at a CTA's rate (measured 42 GB/s with eight warps, 53 with sixteen or for two CTAs of eight on one
// SM, as long as the wave's CTAs do not ask for more than the 6.4 TB/s of the memory) plus about 4.5 us for the chain of loads at the start, the exchanges and the join.  Measured, 256 kv
// heads x 4096 keys: s = 1, 2, 4: 44, 53, 66 us (the formula: 46, 59, 71); 8 kv heads x 131072 keys: eight warps, s = 8, 10, 16: 100,
// 81, 72 (106, 86, 86), sixteen warps, s = 8, 9, 10, 11: 71, 65, 60, 108 (85, 76, 69, 127; from eleven on the device holds seven
// clusters at a time); 512 x 8192: sixteen warps, s = 1: 174; eight warps, s = 1, 2, 4: 198, 181, 205 (210; 203, 213, 223).
template <int D, bool HI, int W, bool CROSS>
cudaError_t plan_for(const CachedAttnArgs &a, int64_t groups, int rows, Plan &best) {
    using S = Sizes<D, HI, W>;
    static Active known[64];
    static std::atomic<bool> raised[64];
    auto kernel = cached_decode_kernel<D, HI, W, CROSS>;
    cudaError_t e = raise_limits((const void *)kernel, (int)kMaxSmem, raised);
    const Active *active = nullptr;
    if (e == cudaSuccess) e = active_clusters(kernel, 32 * W, kMaxSmem, known, &active);
    if (e != cudaSuccess) return e;
    best.cost = HUGE_VAL;
    const int tiles = (a.max_kv + kTileKeys - 1) / kTileKeys;
    const double bytes = 2.0 * a.max_kv * D;
    for (int s = 1; s <= kMaxSplit; ++s) {
        const int per = (tiles + s * W - 1) / (s * W);
        const size_t smem = S::smem(per * W, rows);
        if (smem > kMaxSmem || active->n[s] < 1) continue;
        if (s > 1 && per < 2 && (tiles + (s - 1) * W - 1) / ((s - 1) * W) == per) break;      // no warp has less to do
        const int64_t at_a_time = (int64_t)active->n[s] * (W == 8 && smem <= kHalfSmem ? 2 : 1);
        const double ctas = (double)(groups < at_a_time ? groups : at_a_time) * s;
        double rate = W == 16 ? 53e3 : groups > active->n[s] ? 26.5e3 : 42e3;      // bytes per microsecond
        if (ctas * rate > 6.4e6) rate = 6.4e6 / ctas;
        double waves = (double)((groups + at_a_time - 1) / at_a_time);
        if (waves > 2) waves = (double)groups / at_a_time + 0.5;
        const double cost = waves * (4.5 + (s > 1 ? 0.5 + 0.1 * s : 0.0) + bytes / s / rate);
        if (cost < best.cost) { best.cost = cost; best.split = s; best.per_warp = per; }
    }
    return cudaSuccess;
}

template <int D, bool HI, int W, bool CROSS>
cudaError_t launch_plan(const CachedAttnArgs &a, const Plan &p, int rows, int row_tiles, int merge, cudaStream_t stream) {
    CUtensorMap mk, mv;
    if (CROSS ? !make_states_map(&mk, a.k_pages, a.k_stride, a, kTileKeys) || !make_states_map(&mv, a.v_pages, a.v_stride, a, kTileKeys)
              : !make_page_map(&mk, a.k_pages, a, kTileKeys) || !make_page_map(&mv, a.v_pages, a, kTileKeys))
        return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.split, (unsigned)(a.Hkv * row_tiles), (unsigned)a.B);
    cfg.blockDim = dim3(32 * W);
    cfg.dynamicSmemBytes = Sizes<D, HI, W>::smem(p.per_warp * W, rows);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.split;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CROSS ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, cached_decode_kernel<D, HI, W, CROSS>, a, mk, mv, row_tiles, p.per_warp, merge);
}

template <int D, bool HI, bool CROSS>
cudaError_t launch_typed(const CachedAttnArgs &a, cudaStream_t stream) {
    constexpr int kRows = Sizes<D, HI, 8>::kRows;
    int rows = CROSS ? a.max_q * a.group : a.group;                 // of a kv head
    // Room for the rows of sequences that share their states, eight rows in all (so none with more than four heads per kv head), where
    // there may be any and the logits of eight rows leave room for two CTAs on an SM: up to 3872 keys of 128 dims, 7936 of 64.
    // Whether any share is known on the device alone.  32 queries, four by four on the same states (16 heads of 128): on 577, 1499, 3872
    // keys 10.7, 16.4, 32.9 us, apart 18.4, 29.6, 60.6; with two by two of four heads per kv head no change (16.2, apart 15.9).  Beyond
    // that they stay apart: on 3904, 8192, 16384 keys 61, 115, 220 us, together 33, 46, 90; but room that nobody takes costs 4 to 9 % there
    // (32 queries that share nothing, 16384 keys: 325 us, with room 339; 8 on 32768 keys, 32 heads on 8: 84, 91).
    int merge = 1;
    if (CROSS && a.max_q == 1 && !a.key_range && a.B > 1 && Sizes<D, HI, 8>::smem((a.max_kv + kTileKeys - 1) / kTileKeys + 8, kRows) <= kHalfSmem)
        merge = kRows / a.group > 1 ? kRows / a.group : 1;
    rows *= merge;
    const int row_tiles = (rows + kRows - 1) / kRows;
    const int64_t groups = (int64_t)a.B * a.Hkv * row_tiles;
    Plan p8, p16;
    cudaError_t e = plan_for<D, HI, 8, CROSS>(a, groups, rows, p8);
    if (e == cudaSuccess) e = plan_for<D, HI, 16, CROSS>(a, groups, rows, p16);
    if (e != cudaSuccess) return e;
    // (sixteen warps' rings leave no room for the logits of many rows of long caches: d = 128, 16 rows, more than 81920 keys;
    // eight warps in clusters of sixteen hold all that is allowed)
    if (p8.cost == HUGE_VAL && p16.cost == HUGE_VAL) return cudaErrorInvalidConfiguration;
    return p16.cost < p8.cost ? launch_plan<D, HI, 16, CROSS>(a, p16, rows, row_tiles, merge, stream)
                              : launch_plan<D, HI, 8, CROSS>(a, p8, rows, row_tiles, merge, stream);
}

template <bool CROSS>
cudaError_t launch_rows_of_kv_heads(const CachedAttnArgs &a, int rows, cudaStream_t stream) {
    if (a.d == 128) return rows > 8 ? launch_typed<128, true, CROSS>(a, stream) : launch_typed<128, false, CROSS>(a, stream);
    return rows > 8 ? launch_typed<64, true, CROSS>(a, stream) : launch_typed<64, false, CROSS>(a, stream);
}

}  // namespace

cudaError_t launch_cached_decode(const CachedAttnArgs &a, cudaStream_t stream) { return launch_rows_of_kv_heads<false>(a, a.group, stream); }
cudaError_t launch_cross_decode(const CachedAttnArgs &a, cudaStream_t stream) {
    return launch_rows_of_kv_heads<true>(a, a.max_q * a.group, stream);
}

}  // namespace hccs
