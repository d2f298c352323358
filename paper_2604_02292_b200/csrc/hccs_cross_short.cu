// HCCS attention of many queries to few states (256 keys at most): the words of a prompt, the patches of an image.
//
// As in the kernel for longer states (hccs_cached_tile.cu) a CTA takes tiles of 128 rows, (query, head) pairs of one kv head, the two
// contractions run on the tensor cores, and with r = max(x + D - m, 0) <= 127
//     sum s V = F*sum V + S*sum r V,  Z = F*n + S*sum r,  F = B - S*D.
// All logits of a tile fit tensor memory here (128 rows x 256 columns of int32, twice), so Q.K^T is computed once and read twice, and
// K and V stay in shared memory for all tiles of a chunk.  sum V is the same for every row: a warp of its own adds V up once per
// chunk.  All sums fit int32: |sum r V| < 2^22, S < 2^7, F < 2^15, |sum V| <= 2^15.
//
// CTAs are persistent and take chunks (up to `per_chunk` tiles of one sequence and kv head) in turn.  Two stages, each with half
// of tensor memory, a Q tile, a panel of r and eight row warps, take the tiles alternately: while one waits for a product or
// stores its rows, the other has the integer pipe.  O takes columns of its own in the stage's half where the keys leave room,
// else those of S (all of whose logits have been read twice by then).
//
// Roles: sixteen row warps (two threads per row, half of the keys and of the dims each), a warp each for the copies of Q, the
// copies of K and V, Q.K^T, r.V, and the sums of V.
#include "hccs_cached.cuh"
#include "hccs_tcgen05.cuh"

namespace hccs {

namespace {

constexpr int kRowWarps = 16, kQWarp = 16, kKvWarp = 17, kQkWarp = 18, kPvWarp = 19, kSumWarp = 20;
constexpr int kThreads = 672;                    // 21 warps: 96 registers a thread
constexpr int kTile = 128;
constexpr int kStage = 256;                      // threads and tensor-memory columns of a stage
constexpr int kMaxKeys = 256;
constexpr uint32_t kTmemCols = 512;
constexpr int kStageRow = 64;                    // bytes of a row that a warp stages at a time for its stores

constexpr uint32_t kIdescQK = instr_desc(1, 1, 0, 128, 0);                      // (the keys join at run time)
template <int D> constexpr uint32_t kIdescPVOf = instr_desc(0, 1, 1, 128, D);   // r.V: uint8 x int8, V MN-major

struct ShortBarriers {
    uint64_t q_full[2], q_free[2];               // a stage's Q tile
    uint64_t s_full[2], s_free[2];               // its logits
    uint64_t r_ready[2], o_full[2];
    uint64_t k_full[2], k_free[2], v_full[2], v_free[2];      // by chunk
    uint64_t sum_full[2], sum_free[2];           // sum V, by chunk
    uint64_t drained[2];                         // a given-up CTA: the products of either issuer are through
};

// A chunk, the same for every role: up to per_chunk tiles of one sequence and kv head.  What has to be read for it is fetched a
// chunk ahead.
struct ChunkRaw { int q0, q1, k0, kv; };
struct Chunk {
    int kvh, tile0, tiles;                       // tiles: with rows
    SequenceAt seq;
};

struct ShortPlan {
    int per_chunk, chunks_per, chunks;           // tiles of a chunk, chunks of a (sequence, kv head), all of them
    int keys;                                    // of the K and V tiles: a multiple of 32
    int v_slots;
    int queries;                                 // per tile
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
cross_short_kernel(const __grid_constant__ CachedAttnArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const ShortPlan plan) {
    constexpr int kTileBytes = kTile * D;
    constexpr uint64_t kSwizzle = D == 128 ? kSwizzle128 : kSwizzle64;
    constexpr uint32_t kIdescPV = kIdescPVOf<D>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) ShortBarriers bars;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ int part_max[2][2][kTile], part_sum[2][2][kTile];   // [stage][half][row]
    __shared__ __align__(16) int vsum[2][D];
    __shared__ int row_at[kTile];                                  // where a row of a tile lies in Q and O

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(~0u, tid >> 5, 0);                // (uniform in the compiler's eyes too)
    volatile int *abortp = &abort_flag;
    const int nk = plan.keys, kv_bytes = nk * D;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *gen = smem_raw + (base - smem_u32(smem_raw));
    const int panel_bytes = ((nk + 127) >> 7) * kTile * 128;       // r of a stage: 128 rows x 128 keys, 128-byte swizzle, once or twice
    const uint32_t s_q = base, s_k = s_q + 2 * kTileBytes, s_v = s_k + 2 * kv_bytes, s_r = s_v + plan.v_slots * kv_bytes;
    const uint32_t o_col = nk + D <= kStage ? kStage - D : 0;      // O's columns in its stage's half
    const bool apart = o_col != 0;

    if (tid == 0) {
        abort_flag = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bars.q_full[i]), 1);
            mbar_init(smem_u32(&bars.q_free[i]), 1);
            mbar_init(smem_u32(&bars.s_full[i]), 1);
            mbar_init(smem_u32(&bars.s_free[i]), kStage);
            mbar_init(smem_u32(&bars.r_ready[i]), kStage);
            mbar_init(smem_u32(&bars.o_full[i]), 1);
            mbar_init(smem_u32(&bars.k_full[i]), 1);
            mbar_init(smem_u32(&bars.k_free[i]), 1);
            mbar_init(smem_u32(&bars.v_full[i]), 1);
            mbar_init(smem_u32(&bars.v_free[i]), 2);               // the products and the sums
            mbar_init(smem_u32(&bars.sum_full[i]), 1);
            mbar_init(smem_u32(&bars.sum_free[i]), kRowWarps);
            mbar_init(smem_u32(&bars.drained[i]), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (tid < kTile) row_at[tid] = (tid / a.group * a.Hq + tid % a.group) * D;
    if (warp == kPvWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_slot;
    auto wait = [&](uint64_t *bar, uint32_t parity) -> bool { return warp_wait(smem_u32(bar), parity, abortp, a.status, a.wait_cycles); };

    auto fetch = [&](int c) -> ChunkRaw {
        ChunkRaw r = {0, 0, 0, 0};
        if (c < plan.chunks) {
            const int b = c / (plan.chunks_per * a.Hkv);
            r.q0 = __ldg(a.q_start + b);
            r.q1 = __ldg(a.q_start + b + 1);
            r.k0 = __ldg(a.k_start + b);
            r.kv = __ldg(a.kv_len + b);
        }
        return r;
    };
    auto chunk_of = [&](int c, const ChunkRaw &r) -> Chunk {
        Chunk k;
        const int pair = c / plan.chunks_per;
        k.kvh = pair % a.Hkv;
        k.seq = cross_sequence(a, r.q0, r.q1, r.k0, r.kv);
        k.tile0 = (c - pair * plan.chunks_per) * plan.per_chunk;
        const int all = (min(k.seq.nq, a.max_q) + plan.queries - 1) / plan.queries;
        k.tiles = max(min(all - k.tile0, plan.per_chunk), 0);
        return k;
    };
    const int step = gridDim.x;

    if (warp == kQWarp) {
        // ===================================================== copies of Q: tile number `it` of the CTA into stage it & 1
        int it = 0;
        bool ok = true;
        const uint32_t bytes = (uint32_t)(plan.queries * a.group * D);
        ChunkRaw raw = fetch(blockIdx.x);
        for (int c = blockIdx.x; ok && c < plan.chunks; c += step) {
            const Chunk k = chunk_of(c, raw);
            raw = fetch(c + step);
            if (k.seq.cut && k.tile0 == 0 && k.kvh == 0 && lane == 0) atomicOr(a.status, STATUS_BAD_LENGTH);
            if (k.seq.n == 0) continue;
            for (int t = 0; t < k.tiles; ++t, ++it) {
                const int st = it & 1;
                if (it >= 2) ok = wait(&bars.q_free[st], ((it >> 1) - 1) & 1);
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(smem_u32(&bars.q_full[st]), bytes);
                    tma_load_3d(s_q + st * kTileBytes, &map_q, 0, k.kvh * a.group, k.seq.s0 + (k.tile0 + t) * plan.queries, smem_u32(&bars.q_full[st]));
                }
                __syncwarp();
            }
        }
        // (the last copy of each stage has landed before the CTA may leave, whatever became of its readers; again with a limit)
        for (int x = max(it - 2, 0); x < it; ++x) mbar_wait_bounded(smem_u32(&bars.q_full[x & 1]), (x >> 1) & 1, a.wait_cycles);
    } else if (warp == kKvWarp) {
        // ===================================================== copies of K and V, a chunk ahead where there is a slot
        int kc = 0;
        bool ok = true;
        int sent_v = 0;
        ChunkRaw raw = fetch(blockIdx.x);
        for (int c = blockIdx.x; ok && c < plan.chunks; c += step) {
            const Chunk k = chunk_of(c, raw);
            raw = fetch(c + step);
            if (k.seq.n == 0 || k.tiles == 0) continue;
            const int ks = kc & 1, vs = plan.v_slots == 2 ? kc & 1 : 0, vround = plan.v_slots == 2 ? kc >> 1 : kc;
            if (kc >= 2) ok = wait(&bars.k_free[ks], ((kc >> 1) - 1) & 1);
            if (!ok) break;
            if (lane == 0) {
                mbar_expect_tx(smem_u32(&bars.k_full[ks]), (uint32_t)kv_bytes);
                tma_load_3d(s_k + ks * kv_bytes, &map_k, 0, k.kvh, k.seq.k0, smem_u32(&bars.k_full[ks]));
            }
            __syncwarp();
            ++kc;
            if (vround >= 1) ok = wait(&bars.v_free[vs], (vround - 1) & 1);
            if (!ok) break;
            if (lane == 0) {
                mbar_expect_tx(smem_u32(&bars.v_full[vs]), (uint32_t)kv_bytes);
                tma_load_3d(s_v + vs * kv_bytes, &map_v, 0, k.kvh, k.seq.k0, smem_u32(&bars.v_full[vs]));
            }
            __syncwarp();
            ++sent_v;
        }
        for (int x = max(kc - 2, 0); x < kc; ++x) mbar_wait_bounded(smem_u32(&bars.k_full[x & 1]), (x >> 1) & 1, a.wait_cycles);
        for (int x = max(sent_v - plan.v_slots, 0); x < sent_v; ++x)
            mbar_wait_bounded(smem_u32(&bars.v_full[x % plan.v_slots]), (x / plan.v_slots) & 1, a.wait_cycles);
    } else if (warp == kQkWarp) {
        // ===================================================== S = Q.K^T (the whole warp walks, an elected thread issues)
        const uint64_t dq = smem_desc(s_q, 16, 8 * D, kSwizzle), dk = smem_desc(s_k, 16, 8 * D, kSwizzle);
        const uint32_t idesc = kIdescQK | (uint32_t)(nk >> 3) << 17;
        int it = 0, kc = 0;
        bool ok = true;
        ChunkRaw raw = fetch(blockIdx.x);
        for (int c = blockIdx.x; ok && c < plan.chunks; c += step) {
            const Chunk k = chunk_of(c, raw);
            raw = fetch(c + step);
            if (k.seq.n == 0 || k.tiles == 0) continue;
            const int ks = kc & 1;
            ok = wait(&bars.k_full[ks], (kc >> 1) & 1);
            const uint32_t k_lo = (uint32_t)dk + ((uint32_t)(ks * kv_bytes) >> 4);
            for (int t = 0; ok && t < k.tiles; ++t, ++it) {
                const int st = it & 1;
                if (it >= 2) ok = wait(&bars.s_free[st], ((it >> 1) - 1) & 1);
                if (ok) ok = wait(&bars.q_full[st], (it >> 1) & 1);
                if (!ok) break;
                tcgen05_fence_after();
                const uint32_t q_lo = (uint32_t)dq + ((uint32_t)(st * kTileBytes) >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int x = 0; x < D / 32; ++x)
                        tcgen05_mma_i8(tmem + st * kStage, make_u64(q_lo + 2 * x, (uint32_t)(dq >> 32)), make_u64(k_lo + 2 * x, (uint32_t)(dk >> 32)), idesc, x != 0);
                    tcgen05_commit(smem_u32(&bars.s_full[st]));
                    tcgen05_commit(smem_u32(&bars.q_free[st]));
                    if (t == k.tiles - 1) tcgen05_commit(smem_u32(&bars.k_free[ks]));
                }
                __syncwarp();
            }
            ++kc;
        }
    } else if (warp == kPvWarp) {
        // ===================================================== O = r.V
        const uint64_t dr = smem_desc(s_r, 16, 1024, kSwizzle128), dv = smem_desc(s_v, 8 * D, 8 * D, kSwizzle);
        int it = 0, kc = 0;
        bool ok = true;
        ChunkRaw raw = fetch(blockIdx.x);
        for (int c = blockIdx.x; ok && c < plan.chunks; c += step) {
            const Chunk k = chunk_of(c, raw);
            raw = fetch(c + step);
            if (k.seq.n == 0 || k.tiles == 0) continue;
            const int vs = plan.v_slots == 2 ? kc & 1 : 0, vround = plan.v_slots == 2 ? kc >> 1 : kc;
            ok = wait(&bars.v_full[vs], vround & 1);
            const uint32_t v_lo = (uint32_t)dv + ((uint32_t)(vs * kv_bytes) >> 4);
            for (int t = 0; ok && t < k.tiles; ++t, ++it) {
                const int st = it & 1;
                ok = wait(&bars.r_ready[st], (it >> 1) & 1);
                if (!ok) break;
                tcgen05_fence_after();
                const uint32_t r_lo = (uint32_t)dr + ((uint32_t)(st * panel_bytes) >> 4);
                if (elect_one()) {
                    for (int x = 0; x < nk / 32; ++x)
                        tcgen05_mma_i8(tmem + st * kStage + o_col, make_u64(r_lo + (x >> 2) * (kTile * 128 >> 4) + 2 * (x & 3), (uint32_t)(dr >> 32)),
                                       make_u64(v_lo + (x * 32 * D >> 4), (uint32_t)(dv >> 32)), kIdescPV, x != 0);
                    tcgen05_commit(smem_u32(&bars.o_full[st]));
                    if (t == k.tiles - 1) tcgen05_commit(smem_u32(&bars.v_free[vs]));
                }
                __syncwarp();
            }
            ++kc;
        }
    } else if (warp == kSumWarp) {
        // ===================================================== sum V: a lane adds 16 dims of every kLanes-th key
        constexpr int kPieces = D / 16, kLanes = 32 / kPieces;
        const int piece = lane % kPieces, first = lane / kPieces;
        int kc = 0;
        bool ok = true;
        ChunkRaw raw = fetch(blockIdx.x);
        for (int c = blockIdx.x; ok && c < plan.chunks; c += step) {
            const Chunk k = chunk_of(c, raw);
            raw = fetch(c + step);
            if (k.seq.n == 0 || k.tiles == 0) continue;
            const int vs = plan.v_slots == 2 ? kc & 1 : 0, vround = plan.v_slots == 2 ? kc >> 1 : kc;
            if (kc >= 2) ok = wait(&bars.sum_free[kc & 1], ((kc >> 1) - 1) & 1);
            if (ok) ok = wait(&bars.v_full[vs], vround & 1);
            if (!ok) break;
            const uint8_t *v = gen + (s_v - base) + vs * kv_bytes;
            int sum[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[i] = 0;
#pragma unroll 2
            for (int r = first; r < k.seq.n; r += kLanes) {
                const uint4 w = *reinterpret_cast<const uint4 *>(v + r * D + ((piece ^ (D == 128 ? r & 7 : (r >> 1) & 3)) << 4));
                const int x[4] = {(int)w.x, (int)w.y, (int)w.z, (int)w.w};
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[i] = __dp4a(x[i >> 2], 1 << (8 * (i & 3)), sum[i]);
            }
#pragma unroll
            for (int o = kPieces; o < 32; o <<= 1)
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[i] += __shfl_xor_sync(~0u, sum[i], o);
            if (first == 0) {
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<int4 *>(&vsum[kc & 1][piece * 16 + i]) = make_int4(sum[i], sum[i + 1], sum[i + 2], sum[i + 3]);
            }
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_u32(&bars.sum_full[kc & 1]));
                mbar_arrive(smem_u32(&bars.v_free[vs]));
            }
            __syncwarp();
            ++kc;
        }
    } else {
        // ===================================================== row warps: threads t and t + 128 of a stage own row t, half of the
        // keys and of the dims each
        const int stage = warp >> 3, half = (warp >> 2) & 1, quarter = warp & 3, t = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16, s_at = tmem + lanes + stage * kStage, o_at = s_at + o_col + half * (D / 2);
        const int width = nk >> 1, key0 = half * width;            // a multiple of 16
        uint8_t *const panel = gen + (s_r - base) + stage * panel_bytes;
        uint8_t *const staged = panel + (warp & 7) * (32 * kStageRow);      // (taken when the tile's products are through)
        const bool wide = output_is_wide(a);
        const int elem = wide ? 4 : 2;
        auto stage_barrier = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(stage + 1), "n"(kStage) : "memory"); };
        int it = 0, kc = 0;
        bool ok = true;          // a wait given up: the rest is walked through for the stage's barriers alone
        ChunkRaw raw = fetch(blockIdx.x);
        for (int c = blockIdx.x; c < plan.chunks; c += step) {
            const Chunk k = chunk_of(c, raw);
            raw = fetch(c + step);
            if (k.tiles == 0) continue;
            const int rows_left = min(k.seq.nq, a.max_q) * a.group;
            const int64_t o0 = ((int64_t)k.seq.s0 * a.Hq + (int64_t)k.kvh * a.group) * D + half * (D / 2);
            // a lane of the stores takes piece lane % 4 of rows lane / 4, + 8, ... of the warp's 32
            auto store_rows = [&](int tile, int at_dim, bool zeros) {
                const int left = rows_left - tile * plan.queries * a.group;
                uint8_t *const out = static_cast<uint8_t *>(a.O) + (o0 + (int64_t)tile * plan.queries * a.Hq * D + at_dim) * elem + (lane & 3) * 16;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = i * 8 + (lane >> 2), row = quarter * 32 + r;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (!zeros) v = *reinterpret_cast<const uint4 *>(staged + r * kStageRow + (((lane & 3) ^ ((r >> 1) & 3)) << 4));
                    if (row < min(left, plan.queries * a.group)) *reinterpret_cast<uint4 *>(out + (int64_t)row_at[row] * elem) = v;
                }
            };
            const int dims_at_a_time = kStageRow / elem;
            if (k.seq.n == 0) {                                    // nothing to see: zeros
                for (int x = stage; x < k.tiles; x += 2)
                    for (int dim = 0; dim < D / 2; dim += dims_at_a_time) store_rows(k.tile0 + x, dim, true);
                continue;
            }
            const int h = k.kvh * a.group + t % a.group;
            const int4 e = *reinterpret_cast<const int4 *>(a.table + h);
            const int M = a.mult[h], sh = a.requant_shift, shl = 24 - sh;
            const Requant rq = make_requant(M, sh);
            const double inv = M > 0 ? 1.0 / (double)M : 0.0;
            const int F = e.x - e.y * e.z, n = k.seq.n;
            const int lo = -rq.neg_lo, hi = lo + rq.span;
            const float scale = a.scale[h];
            bool sums = false;                                     // sum V of the chunk has been waited for
            for (int x = 0; x < k.tiles; ++x, ++it) {
                if ((it & 1) != stage) continue;
                const uint32_t phase = (it >> 1) & 1;
                // ---- the largest accumulator
                if (ok) ok = wait(&bars.s_full[stage], phase);
                tcgen05_fence_after();
                int amax = kNone;
                for (int i = 0; ok && i + 32 <= width; i += 32) {
                    if (key0 + i >= n) break;
                    uint32_t acc[32];
                    tmem_ld32(s_at + key0 + i, acc);
                    if (key0 + i + 32 > n) {
                        const uint32_t mask = low_bits(n - key0 - i);
#pragma unroll
                        for (int j = 0; j < 32; ++j) acc[j] = (mask >> j) & 1 ? acc[j] : (uint32_t)kNone;
                    }
#pragma unroll
                    for (int j = 0; j < 32; j += 2) amax = __vimax3_s32(amax, (int)acc[j], (int)acc[j + 1]);
                }
                const int tail = key0 + (width & ~31);             // 16 more keys where the width is odd that way
                if (ok && (width & 16) && tail < n) {
                    uint32_t acc[16];
                    tmem_ld16(s_at + tail, acc);
                    const uint32_t mask = low_bits(n - tail);
#pragma unroll
                    for (int j = 0; j < 16; j += 2)
                        amax = __vimax3_s32(amax, (mask >> j) & 1 ? (int)acc[j] : kNone, (mask >> (j + 1)) & 1 ? (int)acc[j + 1] : kNone);
                }
                part_max[stage][half][t] = amax;
                stage_barrier();
                amax = max(amax, part_max[stage][half ^ 1][t]);
                // ---- r: with u = m - D, accumulators are clamped to [lo_u, hi], lo_u the smallest whose logit reaches max(u, -128); then
                // clamp(acc - lo_u, 0, hi - lo_u)*(M << shl) + (((lo_u*M + R) << shl) - (u << 24)) has r as its top byte
                const int u = ((int)requant_top(rq, amax) >> 24) - e.z;
                int lo_u = lo;
                if (M > 0) {
                    // ceil of num / M, |num| < 2^33 and M < 2^13: num * inv is off by less than 2^-19, a fraction is 2^-13 or more
                    const double q = ceil(((double)u * (double)(1 << sh) - (double)(1 << (sh - 1))) * inv - 0x1p-15);
                    lo_u = (int)fmin(fmax(q, (double)lo), (double)hi);
                }
                const int neg_lo = -lo_u, span = hi - lo_u;
                const uint32_t mk = rq.mk, ck = (((uint32_t)lo_u * (uint32_t)M + (1u << (sh - 1))) << shl) - ((uint32_t)u << 24);
                int rsum = 0;
                auto bytes4 = [&](const uint32_t *acc) -> uint32_t {
                    uint32_t y[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) y[j] = (uint32_t)__viaddmin_s32_relu((int)acc[j], neg_lo, span) * mk + ck;
                    return __byte_perm(__byte_perm(y[0], y[1], 0x0073), __byte_perm(y[2], y[3], 0x0073), 0x5410);
                };
                auto put16 = [&](int key, const uint32_t *w) {     // 16 keys of the row into the panel
                    *reinterpret_cast<uint4 *>(panel + (key >> 7) * (kTile * 128) + t * 128 + ((((key & 127) >> 4) ^ (t & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                };
                auto masked = [&](uint32_t w, uint32_t mask) -> uint32_t { return w & ((((mask & 15u) * 0x00204081u) & 0x01010101u) * 255u); };
                for (int i = 0; ok && i + 32 <= width; i += 32) {
                    uint32_t w[8];
                    if (key0 + i < n) {
                        uint32_t acc[32];
                        tmem_ld32(s_at + key0 + i, acc);
                        const uint32_t mask = low_bits(n - key0 - i);
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[j] = bytes4(acc + 4 * j);
                        if (mask != ~0u) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) w[j] = masked(w[j], mask >> (4 * j));
                        }
#pragma unroll
                        for (int j = 0; j < 8; ++j) rsum = (int)__dp4a(w[j], 0x01010101u, (uint32_t)rsum);
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[j] = 0u;
                    }
                    put16(key0 + i, w);
                    put16(key0 + i + 16, w + 4);
                }
                if (ok && (width & 16)) {
                    uint32_t w[4] = {0u, 0u, 0u, 0u};
                    if (tail < n) {
                        uint32_t acc[16];
                        tmem_ld16(s_at + tail, acc);
                        const uint32_t mask = low_bits(n - tail);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            w[j] = masked(bytes4(acc + 4 * j), mask >> (4 * j));
                            rsum = (int)__dp4a(w[j], 0x01010101u, (uint32_t)rsum);
                        }
                    }
                    put16(tail, w);
                }
                tcgen05_fence_before();
                if (apart) mbar_arrive(smem_u32(&bars.s_free[stage]));
                part_sum[stage][half][t] = rsum;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(smem_u32(&bars.r_ready[stage]));
                stage_barrier();
                rsum += part_sum[stage][half ^ 1][t];
                const RowFactor f = row_factor(a, (int64_t)F * n + (int64_t)e.y * rsum, scale);
                if (ok && !sums) {
                    ok = wait(&bars.sum_full[kc & 1], (kc >> 1) & 1);
                    sums = true;
                }
                if (ok) ok = wait(&bars.o_full[stage], phase);
                if (!ok) continue;
                tcgen05_fence_after();
                // ---- the rows' outputs, 64 bytes of each at a time, through the warp's part of the panel: four lanes store a row's piece
                const int steps = D / 2 * elem / kStageRow;
                for (int y = 0; y < steps; ++y) {
                    auto quad = [&](int dim, const uint32_t *o) -> uint4 {
                        const int4 vs = *reinterpret_cast<const int4 *>(&vsum[kc & 1][half * (D / 2) + dim]);
                        const int num[4] = {e.y * (int)o[0] + F * vs.x, e.y * (int)o[1] + F * vs.y, e.y * (int)o[2] + F * vs.z, e.y * (int)o[3] + F * vs.w};
                        return output4(a, num, f);
                    };
                    auto put = [&](int p, const uint4 &v) { *reinterpret_cast<uint4 *>(staged + lane * kStageRow + ((p ^ ((lane >> 1) & 3)) << 4)) = v; };
                    if (wide) {
                        uint32_t o[16];
                        tmem_ld16(o_at + y * 16, o);
#pragma unroll
                        for (int p = 0; p < 4; ++p) put(p, quad(y * 16 + 4 * p, o + 4 * p));
                    } else {
                        uint32_t o[32];
                        tmem_ld32(o_at + y * 32, o);
#pragma unroll
                        for (int p = 0; p < 4; ++p) {
                            const uint4 v0 = quad(y * 32 + 8 * p, o + 8 * p), v1 = quad(y * 32 + 8 * p + 4, o + 8 * p + 4);
                            put(p, make_uint4(v0.x, v0.y, v1.x, v1.y));
                        }
                    }
                    if (y == steps - 1) {
                        tcgen05_fence_before();
                        if (!apart) mbar_arrive(smem_u32(&bars.s_free[stage]));
                    }
                    __syncwarp();
                    store_rows(k.tile0 + x, y * dims_at_a_time, false);
                    __syncwarp();
                }
            }
            // (a warp without a tile in this chunk waits as well: nobody is a chunk ahead of the sums)
            if (ok && !sums) ok = wait(&bars.sum_full[kc & 1], (kc >> 1) & 1);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars.sum_free[kc & 1]));
            ++kc;
        }
    }
    __syncwarp();
    tcgen05_fence_before();
    __syncthreads();
    if (*abortp) {
        // Some wait has run out, so the products may not all have been waited for; neither tensor memory nor shared memory goes
        // before they are through (again with a limit).  Nobody waits any more: the flag is the same for all.
        if (warp == kQkWarp || warp == kPvWarp) {
            uint64_t *const bar = &bars.drained[warp - kQkWarp];
            if (elect_one()) tcgen05_commit(smem_u32(bar));
            __syncwarp();
            mbar_wait_bounded(smem_u32(bar), 0, a.wait_cycles);
        }
        __syncthreads();
    }
    if (warp == kPvWarp) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

// Queries as [T][Hq][D] bytes, boxes of a kv head's heads and a tile's queries.
bool make_query_map(CUtensorMap *map, const CachedAttnArgs &a, int queries) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)a.d, (cuuint64_t)a.Hq, (cuuint64_t)a.T};
    const cuuint64_t strides[2] = {(cuuint64_t)a.d, (cuuint64_t)a.Hq * a.d};
    const cuuint32_t box[3] = {(cuuint32_t)a.d, (cuuint32_t)a.group, (cuuint32_t)queries};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<int8_t *>(a.Q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              a.d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr size_t kMaxSmem = 219 * 1024;    // dynamic; the kernel's own arrays take up to 6 KB more

template <int D>
cudaError_t launch_typed(const CachedAttnArgs &a, cudaStream_t stream) {
    auto kernel = cross_short_kernel<D>;
    static std::atomic<bool> raised[64];
    cudaError_t e = raise_limits((const void *)kernel, (int)kMaxSmem, raised);
    int dev = 0, sms = 0;
    if (e == cudaSuccess) e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    ShortPlan p;
    p.queries = kTile / a.group;
    p.keys = a.max_kv <= 32 ? 32 : (a.max_kv + 31) / 32 * 32;
    const size_t fixed = 1024 + 2 * (size_t)kTile * D + 2 * (size_t)((p.keys + 127) / 128) * kTile * 128, kv = (size_t)p.keys * D;
    p.v_slots = fixed + 4 * kv <= kMaxSmem ? 2 : 1;
    const size_t smem = fixed + (2 + p.v_slots) * kv;
    // Tiles per chunk: the rounds of chunks that a CTA goes through, each as long as its tiles and about half a tile's time for the
    // chunk's own
    const int64_t pairs = (int64_t)a.B * a.Hkv, tiles = ((int64_t)a.max_q + p.queries - 1) / p.queries;
    int64_t best = -1;
    for (int64_t per = 1; per <= 64 && per <= tiles; ++per) {
        const int64_t chunks = pairs * ((tiles + per - 1) / per);
        if (chunks > 0x7fffffff - 1024) continue;
        const int64_t cost = (chunks + sms - 1) / sms * (2 * per + 1);
        if (best < 0 || cost < best) { best = cost; p.per_chunk = (int)per; }
    }
    if (best < 0) return cudaErrorInvalidConfiguration;
    p.chunks_per = (int)((tiles + p.per_chunk - 1) / p.per_chunk);
    p.chunks = (int)(pairs * p.chunks_per);
    CUtensorMap mq, mk, mv;
    if (!make_query_map(&mq, a, p.queries) || !make_states_map(&mk, a.k_pages, a.k_stride, a, p.keys) || !make_states_map(&mv, a.v_pages, a.v_stride, a, p.keys))
        return cudaErrorInvalidValue;
    kernel<<<p.chunks < sms ? p.chunks : sms, kThreads, smem, stream>>>(a, mq, mk, mv, p);
    return cudaGetLastError();
}

}  // namespace

bool cross_short_fits(const CachedAttnArgs &a) { return !a.key_range && a.max_kv <= kMaxKeys && a.group <= kTile; }

cudaError_t launch_cross_short(const CachedAttnArgs &a, cudaStream_t stream) {
    return a.d == 128 ? launch_typed<128>(a, stream) : launch_typed<64>(a, stream);
}

}  // namespace hccs
