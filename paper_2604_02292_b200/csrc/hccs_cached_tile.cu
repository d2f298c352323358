// HCCS attention over the int8 cache for several new tokens per sequence: trees of drafted tokens, chunks of a
// prompt.  A CTA owns 128 rows (query, head of the group) of one kv head and walks over blocks of 128 keys.
//
// The two contractions run on the tensor cores (tcgen05.mma kind::i8, accumulators in tensor memory), as in the
// fused attention kernel.  There is no probability pass: r = max(x + D - m, 0) fits seven bits, so
//     sum s V = F*sum V + S*sum r V
// needs only r, which leaves the accumulators by one clamp, one multiply-add and a byte pick per logit; F and S
// join at the end, where the sums are complete.  The clamp needs the row maximum first, so Q.K^T is computed
// twice: once for the maximum of the raw accumulators (the requantisation is monotone), once for r.
//
// sum V over the keys a row sees: over the blocks that every row sees whole it is the same for all rows, and a spare
// row of ones beside the rows' r (tiles of 127 rows, or any tile that is not full) brings it with the product that is
// computed anyway; over the others (the last ones, where a mask cuts) it is a contraction of its own with the 0/1 bytes
// of the mask in the place of r.  (With that second product in every block, a prompt chunk took 215 us instead of
// 184: tensor time, and the first product of the next block queued behind it.)
//
// Roles: sixteen row warps in two groups that take alternate blocks (two threads per row and group, 64 keys of a
// block each; TMEM lane = row), two warps that issue the TMA loads of alternate tiles (a box per page, or per 128
// keys of a larger one, a lane each), one thread that issues Q.K^T and one that issues the two products with V (and
// in the first pass, where there are none, every second Q.K^T).  K blocks of the first pass, then K and V blocks
// in turn, stream through one ring; load number x uses slot x % kSlots.
//
// Bound: the chain of a block, tensor product -> tensor memory -> registers -> r -> tensor product, in turns of two
// groups: tensor pipe and integer pipe are both half busy.  2048 new tokens on each of two caches of 8192 keys (16 query
// heads on 4 of 128), the caches in L2: 180 us, 0.40 of the int8 rate counting the formula's two products (inputs and caches
// new to L2: 196, 0.37); 8 trees of 48 on 8000 keys (32 heads on 8): 53 us.  Tried and slower or no faster: r (and Q) as operands in tensor memory (185 us), a
// third S buffer in the second pass (208), four groups (222), 64 columns per tensor-memory load (191), all sequences' longest
// tiles first (185; with caches beyond L2 up to half slower), one issuer for both products (263).
//
// Few rows and many keys: the key blocks of a row tile are split over the CTAs of a cluster, which exchange row
// maxima between the passes and sums at the end through distributed shared memory (exact integers: the split
// changes no bit).  Row warps whose 32 rows lie behind the tile's last row do nothing.
#include <cooperative_groups.h>

#include <type_traits>

#include "hccs_cached.cuh"
#include "hccs_tcgen05.cuh"

namespace hccs {

namespace {

namespace cg = cooperative_groups;

constexpr int kRowThreads = 512;
constexpr int kCopyWarp = 16, kCopyWarps = 2, kQkWarp = 18, kPvWarp = kQkWarp + 1;
constexpr int kThreads = 640;                    // 20 warps: 96 registers a thread
constexpr int kTile = 128;
constexpr int kPanelBytes = kTile * 128;         // 128 rows x 128 keys, 128-byte swizzle
constexpr int kMaxSlots = 12;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kIdescQK = instr_desc(1, 1, 0, 128, 128);

using Yes = std::true_type;
using No = std::false_type;

struct TileBarriers {
    uint64_t o_full;
    uint64_t drained[2];                // a given-up CTA: the products of either issuer are through
    uint64_t m_done;                    // every row thread has read its last S block of the first pass
    uint64_t full[kMaxSlots], free[kMaxSlots];
    uint64_t m_full[4], m_free[4];      // S blocks of the first pass (all of tensor memory holds four)
    uint64_t s_full[2], s_free[2];      // S blocks of the second: block kb in buffer kb & 1, group kb & 1
    uint64_t r_ready[2], r_free[2];     // r and mask panels of block kb in buffer kb & 1
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

template <int D> constexpr int kSlotsOf = D == 128 ? 8 : kMaxSlots;
template <int D> constexpr uint32_t kIdescPVOf = instr_desc(0, 1, 1, 128, D);   // r.V and mask.V: uint8 x int8, V MN-major

// CROSS: queries on an encoder's states.  A row sees keys [first, end) of its sequence, all of them where there are no key
// ranges; the blocks that every row of the tile sees whole come first, then the others (the order of blocks is free:
// the sums are exact).  2048 queries on each of two states of 6404 keys (32 heads on 8 of 128): 310 us, in runs among other work up to 346, 0.42
// to 0.38 of the int8 rate counting two products; 1001 queries on 2404 keys, twice, that see 601 of them or none (16 heads on 4): 31 us.
template <int D, bool CROSS>
__global__ void __launch_bounds__(kThreads, 1)
cached_tile_kernel(const __grid_constant__ CachedAttnArgs a, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, int split, int tile_rows) {
    // Q, K and V tiles are 128 rows of D bytes, swizzled over the whole row: K-major operands for Q and K, the
    // MN-major one for V as it is stored
    constexpr int kTileBytes = kTile * D;
    constexpr uint64_t kSwizzle = D == 128 ? kSwizzle128 : kSwizzle64;
    constexpr uint32_t kIdescPV = kIdescPVOf<D>;
    constexpr int kSlots = kSlotsOf<D>;
    static_assert(kSlots % 2 == 0 && kCopyWarps == 2, "a slot belongs to one copy warp, and in each pass to one issuer");
    constexpr uint32_t kTmemO = 256, kTmemW = kTmemO + D;      // S in columns 0..255 (0..511 in the first pass)
    constexpr int kCols = D / 4;                 // columns of O and W per row thread
    constexpr int kDump = D + 4;                 // row pitch of the joined sums, in words
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) TileBarriers bars;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag, any_bad;
    __shared__ int part_max[4][kTile], cta_max[kTile];
    __shared__ int part_sum[4][kTile], part_cnt[4][kTile];
    __shared__ int cta_sum[kTile], cta_cnt[kTile], vsum[D];

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(~0u, tid >> 5, 0);                        // (uniform in the compiler's eyes too)
    if constexpr (CROSS) previous_kernel_done();
    const int b = blockIdx.z, kvh = blockIdx.y;
    const int rank = (int)blockIdx.x % split;
    const int rt = (int)(gridDim.x / split - 1 - blockIdx.x / split);      // the tiles with the most keys first
    const SequenceAt seq = sequence_at<CROSS>(a, b);
    if (seq.cut && tid == 0 && blockIdx.x + blockIdx.y == 0) atomicOr(a.status, STATUS_BAD_LENGTH);
    const int queries = min(seq.nq, a.max_q);
    const int row0 = rt * tile_rows;
    const int vrows = min(tile_rows, queries * a.group - row0);
    if (vrows <= 0) return;                                                // the whole cluster
    const bool spare = vrows < kTile;                                      // row number vrows is all ones
    const int quarters = min((vrows + 32) >> 5, 4);                        // TMEM lane quarters with rows
    const int row_threads = quarters * 128;
    // key blocks of the tile (of its last query, where the rows are causal), and this CTA's share of them
    const int last_query = (row0 + vrows - 1) / a.group;
    const int n_tile = a.tree_mask ? seq.n : min(max(seq.prefix + last_query + 1, 0), seq.n);
    int first_any = 0, first_all = 0, end_any = n_tile, end_all = n_tile;  // CROSS: keys that some row sees, that all rows see
    if constexpr (CROSS) {
        if (a.key_range) {
            __shared__ int seen[4];
            if (tid == 0) { seen[0] = seq.n; seen[1] = 0; seen[2] = 0; seen[3] = seq.n; }
            __syncthreads();
            for (int q = row0 / a.group + tid; q <= last_query; q += kThreads) {
                const int2 r = range_of(a, seq, q);
                if (r.x < r.y) { atomicMin(&seen[0], r.x); atomicMax(&seen[2], r.y); }
                atomicMax(&seen[1], r.x);
                atomicMin(&seen[3], r.y);
            }
            __syncthreads();
            first_any = seen[0]; first_all = seen[1]; end_any = seen[2]; end_all = seen[3];
        }
    }
    const int blocks_from = CROSS ? min(first_any, end_any) / kTile : 0;
    const int blocks = CROSS && first_any >= end_any ? 0 : (end_any + kTile - 1) / kTile - blocks_from;
    const int per = (blocks + split - 1) / split;
    const int kb0 = blocks_from + min(rank * per, blocks), nb = min(min(rank * per, blocks) + per, blocks) - min(rank * per, blocks);
    // the leading blocks that every row sees whole (as long as no page is bad)
    const int seen_first = min(a.tree_mask ? seq.prefix : seq.prefix + row0 / a.group + 1, seq.n);
    const int32_t *table = CROSS ? nullptr : a.page_table + (int64_t)b * a.max_pages;
    volatile int *abortp = &abort_flag;

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *gen = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t s_q = base, s_ring = s_q + kTileBytes, s_r = s_ring + kSlots * kTileBytes, s_w = s_r + 2 * kPanelBytes;
    uint8_t *g_r = gen + (s_r - base), *g_w = gen + (s_w - base);

    if (tid == 0) {
        abort_flag = 0;
        any_bad = 0;
        mbar_init(smem_u32(&bars.o_full), 1);
        for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&bars.drained[i]), 1);
        mbar_init(smem_u32(&bars.m_done), row_threads);
        for (int i = 0; i < kSlots; ++i) { mbar_init(smem_u32(&bars.full[i]), 1); mbar_init(smem_u32(&bars.free[i]), 1); }
        for (int i = 0; i < 4; ++i) { mbar_init(smem_u32(&bars.m_full[i]), 1); mbar_init(smem_u32(&bars.m_free[i]), row_threads / 2); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bars.s_full[i]), 1);
            mbar_init(smem_u32(&bars.s_free[i]), row_threads / 2);
            mbar_init(smem_u32(&bars.r_ready[i]), row_threads / 2);
            mbar_init(smem_u32(&bars.r_free[i]), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kPvWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    __syncthreads();
    // (the copy warps are off to their loads; the others look at the pages and fetch Q first)
    constexpr int kOthers = kThreads - 32 * kCopyWarps;
    if (warp < kCopyWarp || warp >= kCopyWarp + kCopyWarps) {
        const int i0 = warp < kCopyWarp ? tid : tid - 32 * kCopyWarps;
        // pages outside the pools: a look at this CTA's part of the table tells whether the masks have to care
        if constexpr (!CROSS) {
            const int key_end = min((kb0 + nb) * kTile, seq.n);
            for (int p = (kb0 * kTile >> a.page_shift) + i0; (int64_t)p << a.page_shift < key_end; p += kOthers)
                if ((uint32_t)table[p] >= (uint32_t)a.num_pages) any_bad = 1;
        }
        // Q, swizzled by hand: the rows of a tile are (query, head) pairs, not a box of the tensor
        constexpr int kChunks = D / 16;
        for (int i = i0; i < kTile * kChunks; i += kOthers) {
            const int r = i / kChunks, chunk = i % kChunks;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < vrows) {
                const int row = row0 + r, q = row / a.group;
                v = *reinterpret_cast<const uint4 *>(a.Q + (((int64_t)seq.s0 + q) * a.Hq + kvh * a.group + (row - q * a.group)) * D + chunk * 16);
            }
            *reinterpret_cast<uint4 *>(gen + r * D + ((chunk ^ (D == 128 ? r & 7 : (r >> 1) & 3)) << 4)) = v;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("bar.sync 2, %0;" ::"n"(kOthers) : "memory");
    }
    tcgen05_fence_after();
    const uint32_t tmem = tmem_slot;
    const bool bad = any_bad != 0;
    if (bad && tid == 0) atomicOr(a.status, STATUS_BAD_PAGE);
    // whole blocks of this CTA's share, number full0 of it on: the first of the share, or CROSS, taken first all the same
    const int full0 = CROSS ? min(max((first_all + kTile - 1) / kTile - kb0, 0), nb) : 0;
    const int nfull = CROSS ? max(min(end_all / kTile - kb0, nb) - full0, 0) : bad ? 0 : min(max(seen_first / kTile - kb0, 0), nb);
    // the first key of block number kb in the order in which they are taken
    auto key_of = [&](int kb) -> int {
        if constexpr (CROSS) kb = kb < nfull ? full0 + kb : kb - nfull < full0 ? kb - nfull : kb;
        return (kb0 + kb) * kTile;
    };
    const int w0 = spare ? nfull : 0;                                      // first block whose mask.V is computed
    auto wait = [&](uint64_t *bar, uint32_t parity) { return warp_wait(smem_u32(bar), parity, abortp, a.status, a.wait_cycles); };

    if (warp >= kCopyWarp && warp < kCopyWarp + kCopyWarps) {
        // ===================================================== copies: load number x by warp x % kCopyWarps (a thread
        // gets through one TMA copy per several hundred cycles, the copies of different warps and lanes overlap)
        if (split > 1) cluster_arrive();
        const int box = CROSS ? kTile : min(1 << a.page_shift, kTile), boxes = kTile / box;
        const int loads = 3 * nb;
        bool ok = true;
        // lane l of `boxes` copies keys l * box ... of the block; keys that are not there, or whose page is not, are left
        // out (their masks are clear and what the slot held is finite).  The page of the next load is looked up early.
        auto block_of = [&](int x) { return x < nb ? x : (x - nb) >> 1; };
        auto page_of = [&](int x) -> int {
            if constexpr (CROSS) return lane == 0 ? 0 : -1;               // (a block that some row sees has keys)
            const int key = key_of(block_of(x)) + lane * box;
            int page = -1;
            if (lane < boxes && key < seq.n) page = __ldg(table + (key >> a.page_shift));
            return page;
        };
        const int x0 = warp - kCopyWarp;
        int page = x0 < loads ? page_of(x0) : -1, sent = -1;
        for (int x = x0; ok && x < loads; x += kCopyWarps) {
            const bool values = x >= nb && ((x - nb) & 1);
            const bool there = CROSS ? page == 0 : (uint32_t)page < (uint32_t)a.num_pages;
            const int count = __popc(__ballot_sync(~0u, there));
            const int next = x + kCopyWarps < loads ? page_of(x + kCopyWarps) : -1;
            if (x >= kSlots) ok = wait(&bars.free[x % kSlots], (x / kSlots - 1) & 1);
            if (!ok) break;
            const uint32_t bar = smem_u32(&bars.full[x % kSlots]);
            if (lane == 0) mbar_expect_tx(bar, (uint32_t)(count * box * D));
            __syncwarp();
            if (there) {
                const int key = key_of(block_of(x)) + lane * box;
                const uint32_t dst = s_ring + (x % kSlots) * kTileBytes + lane * box * D;
                // (keys behind the sequence's last are some other's, or zeros behind all of them; their masks are clear)
                if constexpr (CROSS) tma_load_3d(dst, values ? &map_v : &map_k, 0, kvh, seq.k0 + key, bar);
                else tma_load_3d(dst, values ? &map_v : &map_k, 0, key & ((1 << a.page_shift) - 1), page * a.Hkv + kvh, bar);
            }
            page = next;
            sent = x;
        }
        // (each slot's last copy has landed before the CTA may leave, whatever became of its readers; again with a limit)
        for (int x = max(x0, sent - kSlots + kCopyWarps); x <= sent; x += kCopyWarps)
            mbar_wait_bounded(smem_u32(&bars.full[x % kSlots]), (x / kSlots) & 1, a.wait_cycles);
    } else if (warp == kQkWarp || warp == kPvWarp) {
        // ===================================================== the products, issued by one thread of each warp.  The whole
        // warp walks through the loops and only the instructions themselves are the elected thread's: in a branch of one
        // lane the operands, which have to be uniform, cost about 100 cycles per product
        if (split > 1) cluster_arrive();
        if (nb > 0) {
            const int me = warp == kQkWarp ? 0 : 1;
            bool ok = true;
            auto wait = [&](uint64_t *bar, uint32_t parity) -> bool {
                return warp_wait(smem_u32(bar), parity, abortp, a.status, a.wait_cycles);
            };
            const uint64_t dq = smem_desc(s_q, 16, 8 * D, kSwizzle), dk = smem_desc(s_ring, 16, 8 * D, kSwizzle);
            const uint32_t dq_lo = (uint32_t)dq, dq_hi = (uint32_t)(dq >> 32), dk_lo = (uint32_t)dk, dk_hi = (uint32_t)(dk >> 32);
            auto qk = [&](int slot, uint32_t column, uint64_t *full) {
                tcgen05_fence_after();
                const uint32_t k_lo = dk_lo + ((uint32_t)(slot * kTileBytes) >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < D / 32; ++ks)
                        tcgen05_mma_i8(tmem + column, make_u64(dq_lo + 2 * ks, dq_hi), make_u64(k_lo + 2 * ks, dk_hi), kIdescQK, ks != 0);
                    tcgen05_commit(smem_u32(full));
                    tcgen05_commit(smem_u32(&bars.free[slot]));
                }
                __syncwarp();
            };
            // first pass: S = Q.K^T, the blocks in turn between the two threads
            for (int g = me; ok && g < nb; g += 2) {
                const int slot = g % kSlots, sb = g & 3;
                if (g >= 4) ok = wait(&bars.m_free[sb], ((g >> 2) - 1) & 1);
                if (ok) ok = wait(&bars.full[slot], (g / kSlots) & 1);
                if (ok) qk(slot, sb * 128, &bars.m_full[sb]);
            }
            // Between the passes buffers and slots change hands: tensor memory from S to O and W, a ring slot from one of
            // these threads to the other where nb is odd.  A wait by parity must not be two phases behind its barrier, so
            // both threads see the first pass finished (all its loads landed, all its products read) before they go on.
            if (ok) ok = wait(&bars.m_done, 0);
            if (me == 0) {
                // second pass: S again
                for (int kb = 0; ok && kb < nb; ++kb) {
                    const int x = nb + 2 * kb, slot = x % kSlots, sb = kb & 1;
                    if (kb >= 2) ok = wait(&bars.s_free[sb], ((kb >> 1) - 1) & 1);
                    if (ok) ok = wait(&bars.full[slot], (x / kSlots) & 1);
                    if (ok) qk(slot, sb * 128, &bars.s_full[sb]);
                }
            } else {
                // O += r.V and, where a mask cuts, W += mask.V
                const uint64_t dr = smem_desc(s_r, 16, 1024, kSwizzle128), dv = smem_desc(s_ring, 8 * D, 8 * D, kSwizzle);
                const uint32_t dr_lo = (uint32_t)dr, dr_hi = (uint32_t)(dr >> 32), dv_lo = (uint32_t)dv, dv_hi = (uint32_t)(dv >> 32);
                for (int kb = 0; ok && kb < nb; ++kb) {
                    const int x = nb + 2 * kb + 1, slot = x % kSlots, buf = kb & 1;
                    ok = wait(&bars.full[slot], (x / kSlots) & 1);
                    if (ok) ok = wait(&bars.r_ready[buf], (kb >> 1) & 1);
                    if (!ok) break;
                    tcgen05_fence_after();
                    const uint32_t v_lo = dv_lo + ((uint32_t)(slot * kTileBytes) >> 4), r_lo = dr_lo + (uint32_t)(buf * kPanelBytes >> 4);
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            tcgen05_mma_i8(tmem + kTmemO, make_u64(r_lo + 2 * ks, dr_hi), make_u64(v_lo + (ks * 32 * D >> 4), dv_hi), kIdescPV, (kb | ks) != 0);
                        if (kb >= w0) {
#pragma unroll
                            for (int ks = 0; ks < 4; ++ks)
                                tcgen05_mma_i8(tmem + kTmemW, make_u64(r_lo + (2 * kPanelBytes >> 4) + 2 * ks, dr_hi),
                                               make_u64(v_lo + (ks * 32 * D >> 4), dv_hi), kIdescPV, ((kb - w0) | ks) != 0);
                        }
                        tcgen05_commit(smem_u32(&bars.free[slot]));
                        tcgen05_commit(smem_u32(&bars.r_free[buf]));
                        if (kb == nb - 1) tcgen05_commit(smem_u32(&bars.o_full));
                    }
                    __syncwarp();
                }
            }
        }
        __syncwarp();
    } else {
        // ===================================================== row warps: threads t, t+128, t+256, t+384 own row t, the
        // first two the halves of the even blocks, the others those of the odd ones
        const int t = tid & (kTile - 1), grp = tid >> 7, group = grp >> 1, half = grp & 1;
        const bool active = (warp & 3) < quarters;
        cg::cluster_group cluster = cg::this_cluster();
        auto row_barrier = [&]() { asm volatile("bar.sync 1, %0;" ::"r"(row_threads) : "memory"); };
        const bool real = t < vrows;
        const int row = row0 + (real ? t : 0), qi = row / a.group, h = kvh * a.group + (row - qi * a.group);
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        bool ok = true;
        HeadEntry th;
        Requant rq;
        int M = 0;
        int rsum = 0, count = 0;
        int xmax = 0, kb;
        // which of keys 64 * half + 32 * part ... of block kb the thread's row sees
        const int2 range = !CROSS || !real ? make_int2(0, 0) : range_of(a, seq, qi);
        const int seen_all = !real ? 0 : CROSS ? range.y : min(a.tree_mask ? seq.prefix : seq.prefix + qi + 1, seq.n);
        const uint32_t *tree = a.tree_mask ? reinterpret_cast<const uint32_t *>(a.tree_mask) + ((int64_t)seq.s0 + qi) * a.tree_words : nullptr;
        auto mask_of = [&](int kb, int part) -> uint32_t {
            const int c0 = key_of(kb) + half * 64 + part * 32;
            uint32_t m = low_bits(seen_all - c0);
            if constexpr (CROSS) return m & ~low_bits(range.x - c0);
            if (tree && real && m != 0xffffffffu) {
                // new key number j0 + k sits at bit k; words beyond max_q's last are never read
                const int j0 = c0 - seq.prefix;
                uint32_t bits = 0;
                if (j0 > -32) {
                    const int w = j0 >> 5, s = j0 & 31;                     // (floor: w = -1 for negative j0)
                    const uint32_t lo = w >= 0 && w * 32 < a.max_q ? tree[w] & low_bits(a.max_q - w * 32) : 0u;
                    const uint32_t hi = (w + 1) * 32 < a.max_q ? tree[w + 1] & low_bits(a.max_q - (w + 1) * 32) : 0u;
                    bits = __funnelshift_r(lo, hi, s);
                }
                m |= bits & low_bits(seq.n - c0);
            }
            if (bad) {
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int key = c0 + 16 * g;
                    if (key >= seq.n || (uint32_t)table[key >> a.page_shift] >= (uint32_t)a.num_pages) m &= ~(0xffffu << (16 * g));
                }
            }
            return m;
        };
        if (active) {
            const int4 e = *reinterpret_cast<const int4 *>(a.table + h);
            th.B = e.x; th.S = e.y; th.D = e.z;
            M = a.mult[h];
            rq = make_requant(M, a.requant_shift);
            // ---- first pass: the largest accumulator
            int amax = kNone;
            auto first = [&](int kb, auto masked) {
                const int sb = kb & 3;
                ok = wait(&bars.m_full[sb], (kb >> 2) & 1);
                if (!ok) return;
                tcgen05_fence_after();
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t acc[32];
                    tmem_ld32(tmem + lane_addr + sb * 128 + half * 64 + part * 32, acc);
                    if (part == 1) {
                        tcgen05_fence_before();
                        mbar_arrive(smem_u32(&bars.m_free[sb]));
                    }
                    if constexpr (decltype(masked)::value) {
                        const uint32_t mask = mask_of(kb, part);
#pragma unroll
                        for (int i = 0; i < 32; ++i) acc[i] = (mask >> i) & 1 ? acc[i] : (uint32_t)kNone;
                    }
#pragma unroll
                    for (int i = 0; i < 32; i += 2) amax = __vimax3_s32(amax, (int)acc[i], (int)acc[i + 1]);
                }
            };
            kb = group;
            for (; ok && kb < nfull; kb += 2) first(kb, No{});
            for (; ok && kb < nb; kb += 2) first(kb, Yes{});
            mbar_arrive(smem_u32(&bars.m_done));
            part_max[grp][t] = amax;
            row_barrier();
            xmax = max(max(part_max[0][t], part_max[1][t]), max(part_max[2][t], part_max[3][t]));
        }
        if (split > 1) {
            if (active && grp == 0) cta_max[t] = xmax;
            cluster_arrive();
            cluster_wait();
            if (active)
                for (int r = 0; r < split; ++r) xmax = max(xmax, cluster.map_shared_rank(cta_max, r)[t]);
        }
        if (active) {
            xmax = (int)requant_top(rq, xmax) >> 24;
            // ---- second pass: with u = m - D, accumulators are clamped to [lo_u, hi], lo_u the smallest whose
            // logit reaches max(u, -128); then clamp(acc - lo_u, 0, hi - lo_u)*(M << k) + (((lo_u*M + R) << k) - (u << 24))
            // lies in [0, 2^31) and has r as its top byte
            const int u = xmax - th.D, sh = a.requant_shift, k = 24 - sh;
            const int lo = -rq.neg_lo, hi = lo + rq.span;
            const int64_t R = 1ll << (sh - 1);
            int lo_u = lo;
            if (M > 0) {      // ceil of a quotient below 2^33 by M < 2^13: exact through one fp64 division
                const double q = ceil((double)((int64_t)u * (1ll << sh) - R) / (double)M);
                lo_u = (int)fmin(fmax(q, (double)lo), (double)hi);
            }
            const int neg_lo = -lo_u, span = hi - lo_u;
            const uint32_t mk = rq.mk, ck = ((uint32_t)((int64_t)lo_u * M + R) << k) - ((uint32_t)u << 24);
            const int swz = t & 7;
            const uint32_t row_off = (uint32_t)((t >> 3) * 1024 + (t & 7) * 128);
            // r and mask panels of this group's blocks: buffer `group` of each
            uint8_t *pr = g_r + group * kPanelBytes + row_off, *pw = g_w + group * kPanelBytes + row_off;
            auto panel16 = [&](uint8_t *panel, int part, const uint32_t (&w)[8]) {      // 32 bytes of the thread's row
                const int c16 = 4 * half + 2 * part;
                *reinterpret_cast<uint4 *>(panel + ((c16 ^ swz) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4 *>(panel + (((c16 + 1) ^ swz) << 4)) = make_uint4(w[4], w[5], w[6], w[7]);
            };
            auto second = [&](int kb, auto masked) {
                ok = wait(&bars.s_full[group], (kb >> 1) & 1);
                if (!ok) return;
                tcgen05_fence_after();
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t acc[32];
                    tmem_ld32(tmem + lane_addr + group * 128 + half * 64 + part * 32, acc);
                    if (part == 1) {
                        tcgen05_fence_before();
                        mbar_arrive(smem_u32(&bars.s_free[group]));
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[i] = (uint32_t)__viaddmin_s32_relu((int)acc[i], neg_lo, span) * mk + ck;
                    uint32_t w[8], ones[8];
                    if constexpr (decltype(masked)::value) {
                        const uint32_t mask = mask_of(kb, part);
                        count += __popc(mask);
#pragma unroll
                        for (int g = 0; g < 8; ++g) ones[g] = (((mask >> (4 * g)) & 15u) * 0x00204081u) & 0x01010101u;
                    }
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        w[g] = __byte_perm(__byte_perm(acc[4 * g], acc[4 * g + 1], 0x0073), __byte_perm(acc[4 * g + 2], acc[4 * g + 3], 0x0073), 0x5410);
                        if constexpr (decltype(masked)::value) w[g] &= ones[g] * 255u;
                        rsum = (int)__dp4a(w[g], 0x01010101u, (uint32_t)rsum);
                    }
                    // the products of the buffer's previous block have read it
                    if (part == 0 && kb >= 2) {
                        ok = wait(&bars.r_free[group], ((kb >> 1) - 1) & 1);
                        if (!ok) return;
                    }
                    if (decltype(masked)::value || t != vrows) panel16(pr, part, w);     // (row vrows keeps its ones)
                    if constexpr (decltype(masked)::value) panel16(pw, part, ones);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(smem_u32(&bars.r_ready[group]));
            };
            kb = group;
            if (kb < nfull) {      // full blocks find the spare row, or else the mask panel, full of ones
                uint32_t ones[8];
#pragma unroll
                for (int g = 0; g < 8; ++g) ones[g] = 0x01010101u;
                if (!spare || t == vrows) {
                    panel16(spare ? pr : pw, 0, ones);
                    panel16(spare ? pr : pw, 1, ones);
                }
                count = 64 * ((nfull - group + 1) >> 1);
            }
            for (; ok && kb < nfull; kb += 2) second(kb, No{});
            for (; ok && kb < nb; kb += 2) second(kb, Yes{});
            part_sum[grp][t] = rsum;
            part_cnt[grp][t] = count;
            row_barrier();
            rsum = part_sum[0][t] + part_sum[1][t] + part_sum[2][t] + part_sum[3][t];
            count = part_cnt[0][t] + part_cnt[1][t] + part_cnt[2][t] + part_cnt[3][t];
            if (ok && nb > 0) ok = wait(&bars.o_full, 0);
            tcgen05_fence_after();
        }
        // ---- join
        const int64_t at0 = ((int64_t)seq.s0 * a.Hq + (int64_t)kvh * a.group) * D;
        if (split == 1) {
            if (active) {
                // the spare row's sums, for every row's thread of the same columns
                uint32_t o[kCols / 16][16];
#pragma unroll
                for (int part = 0; part < kCols / 16; ++part) {
                    if (nb > 0 && ok) {
                        tmem_ld16(tmem + lane_addr + kTmemO + grp * kCols + 16 * part, o[part]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[part][i] = 0u;
                    }
                    if (t == vrows) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) vsum[grp * kCols + 16 * part + i] = (int)o[part][i];
                    }
                }
                row_barrier();
                const int64_t F = th.B - th.S * th.D;
                const RowFactor f = row_factor(a, F * count + (int64_t)th.S * rsum, a.scale[h]);
                // the tile's rows as they are stored go through shared memory (the operands' place: every product is
                // complete), so that neighbouring lanes write neighbouring pieces of a row
                const bool wide = output_is_wide(a);
                const int pitch = D * (wide ? 4 : 2) + 16;
                uint8_t *const stage = gen + t * pitch + grp * kCols * (wide ? 4 : 2);
#pragma unroll
                for (int part = 0; part < kCols / 16; ++part) {
                    uint32_t w[16];
                    if (nb > w0 && ok) {
                        tmem_ld16(tmem + lane_addr + kTmemW + grp * kCols + 16 * part, w);
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) w[i] = 0u;
                    }
                    if (spare) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) w[i] += (uint32_t)vsum[grp * kCols + 16 * part + i];
                    }
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        int64_t num[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) num[i] = F * (int)w[4 * g + i] + (int64_t)th.S * (int)o[part][4 * g + i];
                        const uint4 v = output4(a, num, f);
                        if (wide) *reinterpret_cast<uint4 *>(stage + (16 * part + 4 * g) * 4) = v;
                        else *reinterpret_cast<uint2 *>(stage + (16 * part + 4 * g) * 2) = make_uint2(v.x, v.y);
                    }
                }
                row_barrier();
                const int pieces = D * (wide ? 4 : 2) / 16;
                const int me = (warp & 3) * 128 + grp * 32 + lane;        // of the row_threads that are active
                if (ok)
                    for (int i = me; i < vrows * pieces; i += row_threads) {
                        const int r = i / pieces, piece = i - r * pieces, rr = row0 + r, q = rr / a.group;
                        const int64_t at = at0 + ((int64_t)q * a.Hq + (rr - q * a.group)) * D;
                        reinterpret_cast<uint4 *>(static_cast<uint8_t *>(a.O) + at * (wide ? 4 : 2))[piece] =
                            *reinterpret_cast<const uint4 *>(gen + r * pitch + piece * 16);
                    }
            }
        } else {
            // the CTA's sums go to shared memory (the operands' place: every product is complete)
            int *dump_o = reinterpret_cast<int *>(gen), *dump_w = dump_o + kTile * kDump;
            if (active) {
#pragma unroll
                for (int part = 0; part < kCols / 8; ++part) {      // 16 columns of O, then of W
                    const bool which = part >= kCols / 16;
                    const int col = grp * kCols + 16 * (part % (kCols / 16));
                    uint32_t v[16];
                    if (nb > (which ? w0 : 0) && ok) {
                        tmem_ld16(tmem + lane_addr + (which ? kTmemW : kTmemO) + col, v);
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = 0u;
                    }
                    int *d = (which ? dump_w : dump_o) + t * kDump + col;
#pragma unroll
                    for (int g = 0; g < 4; ++g) *reinterpret_cast<uint4 *>(d + 4 * g) = make_uint4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
                }
                if (grp == 0) { cta_sum[t] = rsum; cta_cnt[t] = count; }
            }
            cluster_arrive();
            cluster_wait();
            // rows shared out over the cluster, four dims per thread and step
            for (int i = rank * kRowThreads + tid; i < vrows * (D / 4); i += split * kRowThreads) {
                const int r = i / (D / 4), dim = (i % (D / 4)) * 4;
                int o[4] = {0, 0, 0, 0}, w[4] = {0, 0, 0, 0}, rs = 0, cn = 0;
                for (int c = 0; c < split; ++c) {
                    const int4 ov = *reinterpret_cast<const int4 *>(cluster.map_shared_rank(dump_o, c) + r * kDump + dim);
                    int4 wv = *reinterpret_cast<const int4 *>(cluster.map_shared_rank(dump_w, c) + r * kDump + dim);
                    if (spare) {
                        const int4 sv = *reinterpret_cast<const int4 *>(cluster.map_shared_rank(dump_o, c) + vrows * kDump + dim);
                        wv.x += sv.x; wv.y += sv.y; wv.z += sv.z; wv.w += sv.w;
                    }
                    o[0] += ov.x; o[1] += ov.y; o[2] += ov.z; o[3] += ov.w;
                    w[0] += wv.x; w[1] += wv.y; w[2] += wv.z; w[3] += wv.w;
                    rs += cluster.map_shared_rank(cta_sum, c)[r];
                    cn += cluster.map_shared_rank(cta_cnt, c)[r];
                }
                const int rr = row0 + r, q = rr / a.group, hh = rr - q * a.group;
                const HeadEntry e = a.table[kvh * a.group + hh];
                const int64_t F = e.B - e.S * e.D;
                int64_t num[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) num[j] = F * w[j] + (int64_t)e.S * o[j];
                store_output4(a, at0 + ((int64_t)q * a.Hq + hh) * D + dim, num, row_factor(a, F * cn + (int64_t)e.S * rs, a.scale[kvh * a.group + hh]));
            }
            cluster_arrive();
            cluster_wait();
        }
    }
    if (split > 1 && warp >= kCopyWarp) {        // the other warps' part of the three cluster barriers
        cluster_wait();
        cluster_arrive();
        cluster_wait();
        cluster_arrive();
        cluster_wait();
    }
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

template <int D, bool CROSS>
cudaError_t launch_typed(const CachedAttnArgs &a, cudaStream_t stream) {
    const int64_t rows = (int64_t)a.max_q * a.group;
    // Tiles of 127 rows leave room for the row of ones; full ones are taken where a row less would mean a tile more,
    // unless there are many anyway (a second product per block costs a tile about 15 %).  CROSS, full ones instead: 2 x 2048 queries on
    // 6404 keys (32 heads on 8 of 128) 342 us instead of 310, 8 x 1024 on 1499 (8 heads of 128) 73.4 instead of 66.6; but 8 x 1024 of 16 heads of 64
    // on 577 keys 72 instead of 81, on 2404 141.5 instead of 145.5: the rule goes by the former.
    const int64_t tiles127 = (rows + kTile - 2) / (kTile - 1), tiles128 = (rows + kTile - 1) / kTile;
    const int tile_rows = tiles127 == tiles128 || tiles128 >= 8 ? kTile - 1 : kTile;
    const int row_tiles = (int)(tile_rows == kTile ? tiles128 : tiles127);
    const int blocks = (a.max_kv + kTile - 1) / kTile;
    const int64_t ctas = (int64_t)row_tiles * a.Hkv * a.B;
    constexpr size_t smem = 1024 + (size_t)(1 + kSlotsOf<D>) * kTile * D + 4 * kPanelBytes;
    static_assert(smem - 1024 >= 2 * sizeof(int) * kTile * (D + 4), "the joined sums fit the operands' place");
    auto kernel = cached_tile_kernel<D, CROSS>;
    static std::atomic<bool> raised[64];
    static Active known[64];
    const Active *active = nullptr;
    cudaError_t e = raise_limits((const void *)kernel, (int)smem, raised);
    if (e == cudaSuccess) e = active_clusters(kernel, kThreads, smem, known, &active);
    if (e != cudaSuccess) return e;
    // Cluster size: waves of as many CTAs as the device holds in clusters of that size, times the blocks each walks over, plus
    // about six blocks' time of set-up and join, ten with an exchange.  (One cache of 100000 keys, 8 kv heads, 8 new tokens: clusters of
    // sixteen, of which seven run at a time, 105 us; of eight 81.)
    int split = 1;
    int64_t best = -1;
    for (int s = 1; s <= kMaxSplit && (s == 1 || blocks >= 2 * s); s *= 2) {
        if (active->n[s] < 1) continue;
        const int64_t slots = (int64_t)active->n[s] * s;
        const int64_t cost = ((ctas * s + slots - 1) / slots) * ((blocks + s - 1) / s + (s > 1 ? 10 : 6));
        if (best < 0 || cost < best) { best = cost; split = s; }
    }
    if (best < 0) return cudaErrorInvalidConfiguration;
    if ((int64_t)row_tiles * split > 0x7fffffff) return cudaErrorInvalidValue;
    CUtensorMap mk, mv;
    if (CROSS ? !make_states_map(&mk, a.k_pages, a.k_stride, a, kTile) || !make_states_map(&mv, a.v_pages, a.v_stride, a, kTile)
              : !make_page_map(&mk, a.k_pages, a, kTile) || !make_page_map(&mv, a.v_pages, a, kTile))
        return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(row_tiles * split), (unsigned)a.Hkv, (unsigned)a.B);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)split;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CROSS ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, mk, mv, split, tile_rows);
}

}  // namespace

cudaError_t launch_cached_attention(const CachedAttnArgs &a, cudaStream_t stream, uint64_t *launches) {
    const cudaError_t e = a.max_q == 1 ? launch_cached_decode(a, stream)
                          : a.d == 128 ? launch_typed<128, false>(a, stream) : launch_typed<64, false>(a, stream);
    if (e == cudaSuccess && launches) ++*launches;
    return e;
}

cudaError_t launch_cross_attention(const CachedAttnArgs &a, cudaStream_t stream, uint64_t *launches) {
    // Up to sixteen rows of a kv head, all of which see the same keys, go through the kernel that is bound by HBM; sixteen is what its
    // products hold.  32 sequences of 16 queries (16 heads of 64), on 577, 1499, 4096 keys: 17.5, 29.0, 57.3 us, through the kernel for many 38.8,
    // 55.0, 95.1; on 77, 250: 12.2, 13.5, through the one for few keys 16.0, 16.1.  One sequence: 6.3 to 10.6, the others 7.1 to 13.1.
    // Then the kernel for few keys wherever it holds them (256: two stages of tensor memory): 8 x 4096 queries on 256 keys (16 heads of 64)
    // 53 us, through the one for many 246 (on 257: 262); 2 x 1000 (32 heads on 8 of 128) 16.3, 40.6 (44.4); 32 x 20 (8 heads of 64) 10.3,
    // 16.4 (17.9).
    const bool few = a.max_q == 1 || (!a.key_range && (int64_t)a.max_q * a.group <= 16);
    const cudaError_t e = few ? launch_cross_decode(a, stream) : cross_short_fits(a) ? launch_cross_short(a, stream)
                          : a.d == 128 ? launch_typed<128, true>(a, stream) : launch_typed<64, true>(a, stream);
    if (e == cudaSuccess && launches) ++*launches;
    return e;
}

}  // namespace hccs
