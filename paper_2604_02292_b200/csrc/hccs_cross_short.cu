// HCCS attention of many queries to few states (256 keys at most): the words of a prompt, the patches of an image.
//
// As in the kernel for longer states (hccs_cached_tile.cu) a CTA takes tiles of 128 rows, (query, head) pairs of one kv head, the two
// contractions run on the tensor cores, and with r = max(x + D - m, 0) <= 127
//     sum s V = F*sum V + S*sum r V,  Z = F*n + S*sum r,  F = B - S*D.
// All logits of a tile fit tensor memory here (128 rows x 256 columns of int32, twice), so Q.K^T is computed once and read twice, and
// K and V stay in shared memory for all tiles of a chunk.  sum V is the same for every row: a warp of its own adds V up once per
// chunk.  All sums fit int32: |sum r V| < 2^22, S < 2^7, F < 2^15, |sum V| <= 2^15.
//
// CTAs are persistent.  The tiles that the sequences really have are counted at the start and shared out evenly, in order, so a CTA
// walks through few (sequence, kv head) pairs: chunks of tiles with one K and V.  Stages, each with its part
// of tensor memory, a Q tile, a panel of r and its row warps, take the tiles in turn: while one waits for a product or
// stores its rows, the others have the integer pipe.  O takes columns of its own in the stage's part where the keys leave room,
// else those of S (all of whose logits have been read twice by then).
//
// Roles: sixteen row warps, a warp each for the copies, Q.K^T, r.V, and the sums of V.
//
// Bound: the chain of a tile (product, tensor memory, arithmetic, product, outputs), with five warps per scheduler to cover it: issue slots
// 52 to 61 % busy, tensor pipe 10 to 21 %.  8 x 4096 queries on 77 keys (16 heads of 64, fp16 out): 31 to 32 us, 3.2 TB/s of Q and O; 24 ragged
// texts of up to 700 on up to 256 keys (32 heads on 8 of 128, bf16 out): 45 us.  The kernel for longer states takes 226 and 176.
//
// Weak at sequences of few queries: a chunk's place is free again once all its rows are stored, and there are as many places as stages, so where a
// chunk is one tile the next one's copies start when a stage is through, in the open; all four quarters of a tile are computed and the whole
// box of Q is fetched, however few rows there are.  512 sequences of 20 queries on 100 keys (16 heads of 64): 185 to 189 us, 9 times the bytes'
// time; through the kernel for longer states 460.
#include "hccs_cached.cuh"
#include "hccs_tcgen05.cuh"

namespace hccs {

namespace {

constexpr int kRowWarps = 16, kCopyWarp = 16, kQkWarp = 17, kPvWarp = 18, kSumWarp = 19;
constexpr int kThreads = 640;                    // 20 warps: 96 registers a thread
constexpr int kTile = 128;
constexpr int kMaxStages = 4;
constexpr int kChunks = 4;                       // chunks that are known ahead
constexpr int kMaxKeys = 256;
constexpr uint32_t kTmemCols = 512;

constexpr uint32_t kIdescQK = instr_desc(1, 1, 0, 128, 0);                      // (the keys join at run time)
template <int D> constexpr uint32_t kIdescPVOf = instr_desc(0, 1, 1, 128, D);   // r.V: uint8 x int8, V MN-major

struct ShortBarriers {
    uint64_t q_full[kMaxStages], q_free[kMaxStages];               // a stage's Q tile
    uint64_t s_full[kMaxStages], s_free[kMaxStages];               // its logits
    uint64_t r_ready[kMaxStages], o_full[kMaxStages];
    uint64_t k_full[kChunks], k_free[kChunks], v_full[kChunks], v_free[kChunks];      // by chunk
    uint64_t sum_full[kChunks], sum_free[kChunks];     // sum V, by chunk
    uint64_t chunk_full[kChunks], chunk_free[kChunks];
    uint64_t met[kMaxStages];                    // the stage's row threads, twice per tile (WIDE)
    uint64_t drained[2];                         // a given-up CTA: the products of either issuer are through
};

// A chunk: tiles of one sequence and kv head.  The copy warp finds them, the others read them from shared memory.
struct Chunk {
    int tiles;                                   // 0: no more chunks
    int n, k0, kvh;                              // keys, the first one's place, kv head
    int q0, rows;                                // first query, rows from there to the sequence's end
};

struct ShortPlan {
    int keys;                                    // of the K and V tiles: a multiple of 32
    int k_shift, v_shift;                        // places for K and for V: 1 << shift, kChunks at most
    int queries;                                 // per tile
    int warp_queries;                            // whole ones among the 32 rows of a warp, or 0: its rows are cut by heads
};

__device__ __forceinline__ int tiles_of(const CachedAttnArgs &a, const SequenceAt &seq, const ShortPlan &plan) {
    return (min(seq.nq, a.max_q) + plan.queries - 1) / plan.queries;
}

// What a tile of a sequence costs, in parts: its rows' outputs and waits, and 16 keys a part (tiles of 256 and of 100 keys measure nearly
// alike, 3900 cycles for heads of 128).
__device__ __forceinline__ int tile_cost(const SequenceAt &seq) { return seq.n == 0 ? 4 : 24 + ((seq.n + 15) >> 4); }

// The chunks of a CTA, walked through by a warp: tiles are in the order (sequence, kv head, tile).  A lane holds one of 32
// neighbouring sequences, so that their lengths are read together and those without queries are skipped together.
struct Walk {
    int q0, q1, k0, kv, first;                   // this lane's sequence, number first + lane
    int b, kvh, tile;
    int64_t left;                                // cost of the tiles still to come (the last may go beyond)

    __device__ __forceinline__ void window(const CachedAttnArgs &a, int from) {
        const int mine = from + (int)(threadIdx.x & 31);
        first = from;
        q0 = q1 = k0 = kv = 0;
        if (mine < a.B) {
            q0 = __ldg(a.q_start + mine);
            q1 = __ldg(a.q_start + mine + 1);
            k0 = __ldg(a.k_start + mine);
            kv = __ldg(a.kv_len + mine);
        }
    }
    __device__ __forceinline__ Chunk next(const CachedAttnArgs &a, const ShortPlan &plan) {
        Chunk k = {0, 0, 0, 0, 0, 0};
        if (left <= 0) return k;
        for (;;) {
            const SequenceAt mine = cross_sequence(a, q0, q1, k0, kv);
            const uint32_t some = __ballot_sync(~0u, mine.nq > 0) & ~low_bits(b - first);
            if (some != 0) {
                const int from = __ffs(some) - 1;
                if (first + from != b) { b = first + from; kvh = 0; tile = 0; }
                break;
            }
            b = first + 32;
            kvh = tile = 0;
            if (b >= a.B) return k;
            window(a, b);
        }
        const int from = b - first;
        const SequenceAt seq = cross_sequence(a, __shfl_sync(~0u, q0, from), __shfl_sync(~0u, q1, from), __shfl_sync(~0u, k0, from), __shfl_sync(~0u, kv, from));
        k.n = seq.n;
        k.k0 = seq.k0;
        k.kvh = kvh;
        const int cost = tile_cost(seq);
        k.tiles = tiles_of(a, seq, plan) - tile;
        if ((int64_t)k.tiles * cost > left) k.tiles = (int)((left + cost - 1) / cost);       // (a division in the last chunk alone)
        k.q0 = seq.s0 + tile * plan.queries;
        k.rows = (min(seq.nq, a.max_q) - tile * plan.queries) * a.group;
        left -= (int64_t)k.tiles * cost;
        tile = 0;
        if (++kvh == a.Hkv) { kvh = 0; ++b; }
        return k;
    }
};

// Where a CTA's walk starts and how much it takes, found by one warp: CTAs share the cost evenly, and a tile goes to the one in whose
// part it begins.  A lane adds up its share of the sequences.
__device__ __forceinline__ void find_start(const CachedAttnArgs &a, const ShortPlan &plan, int *start, int64_t *left) {
    const int lane = threadIdx.x & 31, share = (a.B + 31) / 32, b0 = min(lane * share, a.B), b1 = min(b0 + share, a.B);
    auto cost_of = [&](const SequenceAt &seq) -> int64_t { return (int64_t)tiles_of(a, seq, plan) * tile_cost(seq) * a.Hkv; };
    int64_t mine = 0;
    bool cut = false;
#pragma unroll 4
    for (int b = b0; b < b1; ++b) {
        const SequenceAt seq = sequence_at<true>(a, b);
        mine += cost_of(seq);
        cut |= seq.cut;
    }
    if (cut && blockIdx.x == 0) atomicOr(a.status, STATUS_BAD_LENGTH);
    int64_t upto = mine;                         // of this lane's share and those before it
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(~0u, upto, o);
        if (lane >= o) upto += v;
    }
    const int64_t all = __shfl_sync(~0u, upto, 31), per = (all + gridDim.x - 1) / gridDim.x;
    const int64_t from = min(per * blockIdx.x, all), to = min(from + per, all);
    // the first tile that begins at `from` or behind it: a lane looks in its own share, the first one to have it counts
    int64_t before = upto - mine, begin = to;
    int first_b = 0, pair = 0, tile = 0;
    if (upto > from) {
        for (int b = b0; b < b1 && begin == to; ++b) {
            const SequenceAt seq = sequence_at<true>(a, b);
            const int tiles = tiles_of(a, seq, plan), cost = tile_cost(seq);
            const int64_t skip = (max(from - before, (int64_t)0) + cost - 1) / cost;      // tiles of this sequence
            if (skip < (int64_t)tiles * a.Hkv && before + skip * cost < to) {
                begin = before + skip * cost;
                first_b = b;
                pair = (int)(skip / tiles);
                tile = (int)(skip % tiles);
            }
            before += (int64_t)tiles * a.Hkv * cost;
        }
    }
    const uint32_t some = __ballot_sync(~0u, begin < to);
    if (lane == (some ? __ffs(some) - 1 : 0)) {
        start[0] = first_b;
        start[1] = pair;
        start[2] = tile;
        *left = to - begin;
    }
}

// Requantisation of a head (the rule and the fields of make_requant: a change to one is one to both) without fp64: a quotient of num = c * 2^(sh-1) - less by M is estimated in fp32, off by less than one
// where it is below 2^22, and put right by its remainder; beyond that it is cut to the accumulators' range.
struct HeadRequant {
    uint32_t mk, ck;
    int lo, hi, M, sh;
    float unit;                                  // 2^(sh-1) / M
};
__device__ __forceinline__ int whole_quotient(const HeadRequant &q, int c, int less) {      // floor((c * 2^(sh-1) - less) / M)
    int v = (int)floorf(fminf(fmaxf((float)c * q.unit, -0x1p22f), 0x1p22f));
    const int rest = (int)(((uint32_t)c << (q.sh - 1)) - (uint32_t)less - (uint32_t)v * (uint32_t)q.M);
    v += rest >= q.M ? 1 : rest < 0 ? -1 : 0;
    return min(max(v, -kAccLimit), kAccLimit);
}
__device__ __forceinline__ HeadRequant head_requant(int M, int sh) {
    HeadRequant q;
    q.M = M;
    q.sh = sh;
    q.unit = M > 0 ? (float)(1 << (sh - 1)) / (float)M : 0.0f;
    q.lo = M > 0 ? -whole_quotient(q, 257, 0) : -kAccLimit;
    q.hi = M > 0 ? whole_quotient(q, 255, 1) : kAccLimit;
    q.mk = (uint32_t)M << (24 - sh);
    q.ck = ((uint32_t)q.lo * (uint32_t)M + (1u << (sh - 1))) << (24 - sh);
    return q;
}

// N columns of tensor memory (load and wait in one statement)
__device__ __forceinline__ void tmem_ld(uint32_t at, uint32_t (&r)[16]) { tmem_ld16(at, r); }
__device__ __forceinline__ void tmem_ld(uint32_t at, uint32_t (&r)[32]) { tmem_ld32(at, r); }

// Two 16 x 16 blocks of bytes, their rows at the addresses of lanes 0..15 and 16..31, transposed: word 2m + i of lane l has
// rows 4 * (l % 4) .. + 3 of column l / 4 + 8i of block m.
__device__ __forceinline__ void ldmatrix_b8_trans(uint32_t row, uint32_t (&w)[4]) {
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(row) : "memory");
}
__device__ __forceinline__ int dp4a_s8(uint32_t a, uint32_t b, int c) { return __dp4a((int)a, (int)b, c); }

// Two values plus a constant, and two products with a factor.
__device__ __forceinline__ void add2(float &x, float &y, float by) {
    asm("{\n\t.reg .b64 v, w;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 w, {%2, %2};\n\tadd.rn.f32x2 v, v, w;\n\tmov.b64 {%0, %1}, v;\n\t}" : "+f"(x), "+f"(y) : "f"(by));
}
__device__ __forceinline__ void scale2(float &x, float &y, float by) {
    asm("{\n\t.reg .b64 v, w;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 w, {%2, %2};\n\tmul.rn.f32x2 v, v, w;\n\tmov.b64 {%0, %1}, v;\n\t}" : "+f"(x), "+f"(y) : "f"(by));
}

// WIDE: more than 128 keys: two stages, two threads per row.  Else four stages and a thread per row, which has nobody to wait for.
template <int D, int OUT, bool WIDE>
__global__ void __launch_bounds__(kThreads, 1)
cross_short_kernel(const __grid_constant__ CachedAttnArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_o, const ShortPlan plan) {
    constexpr int kTileBytes = kTile * D;
    constexpr int kStages = WIDE ? 2 : 4, kHalves = WIDE ? 2 : 1, kShift = WIDE ? 1 : 2;
    constexpr int kCols = (int)kTmemCols / kStages;                // tensor-memory columns of a stage
    constexpr int kStageThreads = 128 * kHalves, kDims = D / kHalves;
    constexpr uint64_t kSwizzle = D == 128 ? kSwizzle128 : kSwizzle64;
    constexpr uint32_t kIdescPV = kIdescPVOf<D>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) ShortBarriers bars;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ int part_max[kStages][kHalves][WIDE ? kTile : 1], part_sum[kStages][kHalves][WIDE ? kTile : 1];   // [stage][half][row]
    __shared__ __align__(16) int vsum[kChunks][D];
    __shared__ int start[3];                                       // of the walk: sequence, kv head, tile
    __shared__ int64_t count;
    __shared__ Chunk chunks[kChunks];
    __shared__ int row_at[kTile];                                  // where a row of a tile lies in O, in 16-byte pieces

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(~0u, tid >> 5, 0);                // (uniform in the compiler's eyes too)
    volatile int *abortp = &abort_flag;
    const int nk = plan.keys, kv_bytes = nk * D;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *gen = smem_raw + (base - smem_u32(smem_raw));
    const int panel_bytes = ((nk + 127) >> 7) * kTile * 128;       // r of a stage: 128 rows x 128 keys, 128-byte swizzle, once or twice
    const uint32_t s_q = base, s_k = s_q + kStages * kTileBytes, s_v = s_k + (kv_bytes << plan.k_shift), s_r = s_v + (kv_bytes << plan.v_shift);
    const uint32_t o_col = nk + D <= kCols ? kCols - D : 0;        // O's columns in its stage's part
    const bool apart = o_col != 0;
    const int k_mask = (1 << plan.k_shift) - 1, v_mask = (1 << plan.v_shift) - 1;

    if (warp == kCopyWarp && lane < 4) {
        const CUtensorMap *const map = lane == 0 ? &map_q : lane == 1 ? &map_k : lane == 2 ? &map_v : &map_o;
        asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
    }
    if (tid == 0) {
        abort_flag = 0;
        for (int i = 0; i < kStages; ++i) {
            mbar_init(smem_u32(&bars.q_full[i]), 1);
            mbar_init(smem_u32(&bars.q_free[i]), 1);
            mbar_init(smem_u32(&bars.s_full[i]), 1);
            mbar_init(smem_u32(&bars.s_free[i]), kStageThreads);
            mbar_init(smem_u32(&bars.r_ready[i]), kStageThreads);
            mbar_init(smem_u32(&bars.o_full[i]), 1);
            mbar_init(smem_u32(&bars.met[i]), kStageThreads);
        }
        for (int i = 0; i < kChunks; ++i) {
            mbar_init(smem_u32(&bars.sum_full[i]), 1);
            mbar_init(smem_u32(&bars.sum_free[i]), kRowWarps);
            mbar_init(smem_u32(&bars.chunk_full[i]), 1);
            mbar_init(smem_u32(&bars.chunk_free[i]), kRowWarps + 3);
        }
        for (int i = 0; i < kChunks; ++i) {
            mbar_init(smem_u32(&bars.k_full[i]), 1);
            mbar_init(smem_u32(&bars.k_free[i]), 1);
            mbar_init(smem_u32(&bars.v_full[i]), 1);
            mbar_init(smem_u32(&bars.v_free[i]), 2);               // the products and the sums
        }
        for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&bars.drained[i]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    constexpr bool kWide = OUT == HCCS_I32 || OUT == HCCS_F32;
    constexpr int kElem = kWide ? 4 : 2, kDimsAtATime = 64 / kElem;              // outputs of a thread in registers: 64 bytes
    // bytes of a row that a warp stages for its stores: a line of memory where the warp has one (with 64 everywhere, 24 ragged texts on
    // 256 patches took 56.3 us instead of 54.1)
    constexpr int kStageRow = kDims * kElem < 128 ? kDims * kElem : 128, kRowLanes = kStageRow / 16, kRowsAtATime = 32 / kRowLanes;
    if (tid < kTile) row_at[tid] = (tid / a.group * a.Hq + tid % a.group) * (D * kElem / 16);
    previous_kernel_done();
    if (warp == kCopyWarp) find_start(a, plan, start, &count);
    if (warp == kPvWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_slot;
    auto wait = [&](uint64_t *bar, uint32_t parity) -> bool { return warp_wait(smem_u32(bar), parity, abortp, a.status, a.wait_cycles); };

    // chunk number c, for the roles but the copies (false when a wait was given up), and that this warp is through with it
    auto chunk = [&](int c, Chunk &k) -> bool {
        const bool ok = wait(&bars.chunk_full[c % kChunks], (c / kChunks) & 1);
        if (ok) k = chunks[c % kChunks];
        return ok;
    };
    auto through = [&](int c) {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.chunk_free[c % kChunks]));
    };
    Chunk k = {};

    if (warp == kCopyWarp) {
        // ===================================================== copies: K and V of a chunk and the Q of its tiles, in the order in which they
        // are needed; tile number `it` of the CTA goes into stage it % kStages, chunk number kc into the places of K and V in turn
        int it = 0, kc = 0, sent_v = 0;
        bool ok = true;
        const uint32_t q_bytes = (uint32_t)(plan.queries * a.group * D);
        auto copy = [&](uint32_t dst, const CUtensorMap *map, int y, int z, uint64_t *full, uint32_t bytes) {
            if (lane == 0) {
                mbar_expect_tx(smem_u32(full), bytes);
                tma_load_3d(dst, map, 0, y, z, smem_u32(full));
            }
            __syncwarp();
        };
        auto keys = [&]() -> bool {
            const int ks = kc & k_mask, round = kc >> plan.k_shift;
            if (round >= 1 && !wait(&bars.k_free[ks], (round - 1) & 1)) return false;
            copy(s_k + ks * kv_bytes, &map_k, k.kvh, k.k0, &bars.k_full[ks], (uint32_t)kv_bytes);
            ++kc;
            return true;
        };
        auto values = [&]() -> bool {
            const int vs = sent_v & v_mask, round = sent_v >> plan.v_shift;
            if (round >= 1 && !wait(&bars.v_free[vs], (round - 1) & 1)) return false;
            copy(s_v + vs * kv_bytes, &map_v, k.kvh, k.k0, &bars.v_full[vs], (uint32_t)kv_bytes);
            ++sent_v;
            return true;
        };
        Walk walk;
        walk.b = start[0]; walk.kvh = start[1]; walk.tile = start[2]; walk.left = count;
        walk.window(a, walk.b);
        for (int c = 0; ok; ++c) {
            k = walk.next(a, plan);
            if (c >= kChunks) ok = wait(&bars.chunk_free[c % kChunks], (c / kChunks - 1) & 1);
            if (!ok) break;
            if (lane == 0) {
                chunks[c % kChunks] = k;
                mbar_arrive(smem_u32(&bars.chunk_full[c % kChunks]));
            }
            __syncwarp();
            if (k.tiles == 0) break;
            if (k.n == 0) continue;
            ok = keys();
            for (int t = 0; ok && t < k.tiles; ++t, ++it) {
                const int st = it & (kStages - 1);
                if (it >= kStages) ok = wait(&bars.q_free[st], ((it >> kShift) - 1) & 1);
                if (!ok) break;
                copy(s_q + st * kTileBytes, &map_q, k.kvh * a.group, k.q0 + t * plan.queries, &bars.q_full[st], q_bytes);
                if (t == 0) ok = values();
            }
        }
        // (the last copy into each place has landed before the CTA may leave, whatever became of its readers; again with a limit)
        for (int x = max(it - kStages, 0); x < it; ++x) mbar_wait_bounded(smem_u32(&bars.q_full[x & (kStages - 1)]), (x >> kShift) & 1, a.wait_cycles);
        for (int x = max(kc - 1 - k_mask, 0); x < kc; ++x) mbar_wait_bounded(smem_u32(&bars.k_full[x & k_mask]), (x >> plan.k_shift) & 1, a.wait_cycles);
        for (int x = max(sent_v - 1 - v_mask, 0); x < sent_v; ++x)
            mbar_wait_bounded(smem_u32(&bars.v_full[x & v_mask]), (x >> plan.v_shift) & 1, a.wait_cycles);
    } else if (warp == kQkWarp) {
        // ===================================================== S = Q.K^T (the whole warp walks, an elected thread issues)
        const uint64_t dq = smem_desc(s_q, 16, 8 * D, kSwizzle), dk = smem_desc(s_k, 16, 8 * D, kSwizzle);
        const uint32_t idesc = kIdescQK | (uint32_t)(nk >> 3) << 17;
        int it = 0, kc = 0;
        bool ok = true;
        for (int c = 0; ok && (ok = chunk(c, k)) && k.tiles > 0; ++c) {
            through(c);
            if (k.n == 0) continue;
            const int ks = kc & k_mask;
            ok = wait(&bars.k_full[ks], (kc >> plan.k_shift) & 1);
            const uint32_t k_lo = (uint32_t)dk + ((uint32_t)(ks * kv_bytes) >> 4);
            for (int t = 0; ok && t < k.tiles; ++t, ++it) {
                const int st = it & (kStages - 1);
                if (it >= kStages) ok = wait(&bars.s_free[st], ((it >> kShift) - 1) & 1);
                if (ok) ok = wait(&bars.q_full[st], (it >> kShift) & 1);
                if (!ok) break;
                tcgen05_fence_after();
                const uint32_t q_lo = (uint32_t)dq + ((uint32_t)(st * kTileBytes) >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int x = 0; x < D / 32; ++x)
                        tcgen05_mma_i8(tmem + st * kCols, make_u64(q_lo + 2 * x, (uint32_t)(dq >> 32)), make_u64(k_lo + 2 * x, (uint32_t)(dk >> 32)), idesc, x != 0);
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
        for (int c = 0; ok && (ok = chunk(c, k)) && k.tiles > 0; ++c) {
            through(c);
            if (k.n == 0) continue;
            const int vs = kc & v_mask, vround = kc >> plan.v_shift;
            ok = wait(&bars.v_full[vs], vround & 1);
            const uint32_t v_lo = (uint32_t)dv + ((uint32_t)(vs * kv_bytes) >> 4);
            for (int t = 0; ok && t < k.tiles; ++t, ++it) {
                const int st = it & (kStages - 1);
                ok = wait(&bars.r_ready[st], (it >> kShift) & 1);
                if (!ok) break;
                tcgen05_fence_after();
                const uint32_t r_lo = (uint32_t)dr + ((uint32_t)(st * panel_bytes) >> 4);
                if (elect_one()) {
                    for (int x = 0; x < nk / 32; ++x)
                        tcgen05_mma_i8(tmem + st * kCols + o_col, make_u64(r_lo + (x >> 2) * (kTile * 128 >> 4) + 2 * (x & 3), (uint32_t)(dr >> 32)),
                                       make_u64(v_lo + (x * 32 * D >> 4), (uint32_t)(dv >> 32)), kIdescPV, x != 0);
                    tcgen05_commit(smem_u32(&bars.o_full[st]));
                    if (t == k.tiles - 1) tcgen05_commit(smem_u32(&bars.v_free[vs]));
                }
                __syncwarp();
            }
            ++kc;
        }
    } else if (warp == kSumWarp) {
        // ===================================================== sum V.  32 keys of 16 dims at a time are loaded transposed: a word of lane l
        // holds four keys (those from 4 * (l % 4) on) of dim l / 4, the second one of dim l / 4 + 8, and so on for 16 keys more
        constexpr int kPieces = D / 16;
        const int col = lane >> 2;
        int kc = 0;
        bool ok = true;
        for (int c = 0; ok && (ok = chunk(c, k)) && k.tiles > 0; ++c) {
            through(c);
            if (k.n == 0) continue;
            const int vs = kc & v_mask, vround = kc >> plan.v_shift;
            if (kc >= kChunks) ok = wait(&bars.sum_free[kc % kChunks], (kc / kChunks - 1) & 1);
            if (ok) ok = wait(&bars.v_full[vs], vround & 1);
            if (!ok) break;
            const uint32_t v = s_v + vs * kv_bytes;
            int sum[kPieces][2];
#pragma unroll
            for (int p = 0; p < kPieces; ++p) sum[p][0] = sum[p][1] = 0;
            for (int r0 = 0; r0 < k.n; r0 += 32) {
                const int r = r0 + lane, first = r0 + (lane & 3) * 4;
                const uint32_t m0 = low_bits(8 * min(max(k.n - first, 0), 4)), m1 = low_bits(8 * min(max(k.n - first - 16, 0), 4));
#pragma unroll
                for (int p = 0; p < kPieces; ++p) {
                    uint32_t w[4];
                    ldmatrix_b8_trans(v + r * D + ((p ^ (D == 128 ? r & 7 : (r >> 1) & 3)) << 4), w);
                    sum[p][0] = dp4a_s8(w[0] & m0, 0x01010101u, dp4a_s8(w[2] & m1, 0x01010101u, sum[p][0]));
                    sum[p][1] = dp4a_s8(w[1] & m0, 0x01010101u, dp4a_s8(w[3] & m1, 0x01010101u, sum[p][1]));
                }
            }
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    sum[p][i] += __shfl_xor_sync(~0u, sum[p][i], 1);
                    sum[p][i] += __shfl_xor_sync(~0u, sum[p][i], 2);
                    if ((lane & 3) == 0) vsum[kc % kChunks][p * 16 + col + 8 * i] = sum[p][i];
                }
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_u32(&bars.sum_full[kc % kChunks]));
                mbar_arrive(smem_u32(&bars.v_free[vs]));
            }
            __syncwarp();
            ++kc;
        }
    } else {
        // ===================================================== row warps: thread t of a stage owns row t, or with t + 128 half of its
        // keys and dims
        const int stage = warp / (4 * kHalves), half = WIDE ? (warp >> 2) & 1 : 0, quarter = warp & 3, t = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16, s_at = tmem + lanes + stage * kCols, o_at = s_at + o_col + half * kDims;
        const int width = nk / kHalves, key0 = half * width;       // a multiple of 16, or 32
        uint8_t *const panel = gen + (s_r - base) + stage * panel_bytes;
        // where the warp stages its stores once the tile's products are through: WIDE, its share of the panel, which the others write again
        // behind the next barrier of the stage alone; else the place of its own rows, which nobody else writes
        uint8_t *const staged = panel + (WIDE ? (warp & 7) * (32 * kStageRow) : quarter * (32 * 128));
        // piece `piece` of the warp's row r: eight neighbouring rows' pieces lie on different banks
        auto staged_at = [&](int r, int piece) -> int { return r * kStageRow + ((piece ^ (kRowLanes == 8 ? r & 7 : (r >> 1) & 3)) << 4); };
        // the warp's copies have read what they store: its place may be written again
        auto stored = [&]() {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
        };
        // a barrier of the stage's row threads, given up like every other wait: the first of a tile, then the second
        auto meet = [&](uint32_t phase) -> bool {
            mbar_arrive(smem_u32(&bars.met[stage]));
            return wait(&bars.met[stage], phase);
        };
        int it = 0, kc = 0;
        bool ok = true;
        for (int c = 0; ok && (ok = chunk(c, k)) && k.tiles > 0; ++c) {
            // a lane of the stores takes piece lane % kRowLanes of rows lane / kRowLanes, + kRowsAtATime, ... of the warp's 32
            auto store_rows = [&](int tile, int at_dim, bool zeros) {
                const int there = min(k.rows - tile * plan.queries * a.group, plan.queries * a.group) - quarter * 32;
                if (!zeros && plan.warp_queries != 0 && there >= 32) {
                    // all 32 rows: one copy, which runs beside the next tile's first pass
                    if (lane == 0) {
                        tma_store_3d(&map_o, (half * kDims + at_dim) * kElem, k.kvh * a.group, k.q0 + tile * plan.queries + quarter * plan.warp_queries, smem_u32(staged));
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                    return;
                }
                const int r0 = lane / kRowLanes, piece = lane % kRowLanes;
                const int left = there - r0;
                uint4 *const out = reinterpret_cast<uint4 *>(static_cast<uint8_t *>(a.O) +
                    ((((int64_t)k.q0 + tile * plan.queries) * a.Hq + k.kvh * a.group) * D + half * kDims + at_dim) * kElem) + piece;
#pragma unroll
                for (int i = 0; i < kRowLanes; ++i) {
                    const int r = i * kRowsAtATime + r0;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (!zeros) v = *reinterpret_cast<const uint4 *>(staged + staged_at(r, piece));
                    if (i * kRowsAtATime < left) out[row_at[quarter * 32 + r]] = v;
                }
            };
            if (k.n == 0) {                                        // nothing to see: zeros
                for (int x = stage; x < k.tiles; x += kStages)
                    for (int dim = 0; dim < kDims; dim += kStageRow / kElem) store_rows(x, dim, true);
                through(c);
                continue;
            }
            // A stage without a tile in this chunk only says so.  (A row warp is through with a chunk when it has said so, and nobody is kChunks
            // chunks ahead of it: no warp speaks for a later use of a place before all have for this one.  With heads looked up and sums waited
            // for by all stages in all chunks, 24 ragged texts on 256 patches took 49.5 us instead of 47.4.)
            auto sums_read = [&]() {
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars.sum_free[kc % kChunks]));
                ++kc;
                through(c);
            };
            if (((stage - it) & (kStages - 1)) >= k.tiles) {
                it += k.tiles;
                sums_read();
                continue;
            }
            const int h = k.kvh * a.group + t % a.group;
            const int4 e = *reinterpret_cast<const int4 *>(a.table + h);
            const HeadRequant rq = head_requant(a.mult[h], a.requant_shift);
            const int F = e.x - e.y * e.z, n = k.n;
            const float scale = a.scale[h];
            const int mine = min(max(n - key0, 0), width), whole = mine & ~31;      // keys of this thread's that there are
            bool sums = false;                                     // sum V of the chunk has been waited for
            for (int x = 0; x < k.tiles; ++x, ++it) {
                if ((it & (kStages - 1)) != stage) continue;
                const uint32_t phase = (it >> kShift) & 1;
                // ---- the largest accumulator
                ok = wait(&bars.s_full[stage], phase);
                if (!ok) break;
                tcgen05_fence_after();
                int amax = kNone;
#pragma unroll 1
                for (int i = 0; i < whole; i += 32) {
                    uint32_t acc[32];
                    tmem_ld32(s_at + key0 + i, acc);
#pragma unroll
                    for (int j = 0; j < 32; j += 2) amax = __vimax3_s32(amax, (int)acc[j], (int)acc[j + 1]);
                }
#pragma unroll 1
                for (int i = whole; i < mine; i += 16) {
                    uint32_t acc[16];
                    tmem_ld16(s_at + key0 + i, acc);
#pragma unroll
                    for (int j = 0; j < 16; ++j) amax = max(amax, i + j < mine ? (int)acc[j] : kNone);
                }
                stored();
                if constexpr (WIDE) {
                    part_max[stage][half][t] = amax;
                    ok = meet(0);
                    if (!ok) break;
                    amax = max(amax, part_max[stage][half ^ 1][t]);
                }
                // ---- r: with u = m - D, accumulators are clamped to [lo_u, hi], lo_u the smallest whose logit reaches max(u, -128); then
                // clamp(acc - lo_u, 0, hi - lo_u)*(M << shl) + (((lo_u*M + R) << shl) - (u << 24)) has r as its top byte
                const int u = ((int)((uint32_t)__viaddmin_s32_relu(amax, -rq.lo, rq.hi - rq.lo) * rq.mk + rq.ck) >> 24) - e.z;
                // the smallest accumulator with acc*M >= u*2^sh - R
                const int lo_u = rq.M > 0 ? min(max(whole_quotient(rq, 2 * u - 1, 1) + 1, rq.lo), rq.hi) : rq.lo;
                const int neg_lo = -lo_u, span = rq.hi - lo_u;
                const uint32_t mk = rq.mk, ck = (((uint32_t)lo_u * (uint32_t)rq.M + (1u << (rq.sh - 1))) << (24 - rq.sh)) - ((uint32_t)u << 24);
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
#pragma unroll 1
                for (int i = 0; i < whole; i += 32) {
                    uint32_t acc[32], w[8];
                    tmem_ld32(s_at + key0 + i, acc);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        w[j] = bytes4(acc + 4 * j);
                        rsum = (int)__dp4a(w[j], 0x01010101u, (uint32_t)rsum);
                    }
                    put16(key0 + i, w);
                    put16(key0 + i + 16, w + 4);
                }
#pragma unroll 1
                for (int i = whole; i < mine; i += 16) {
                    uint32_t acc[16], w[4];
                    tmem_ld16(s_at + key0 + i, acc);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        w[j] = bytes4(acc + 4 * j) & low_bits(8 * min(max(mine - i - 4 * j, 0), 4));
                        rsum = (int)__dp4a(w[j], 0x01010101u, (uint32_t)rsum);
                    }
                    put16(key0 + i, w);
                }
                for (int i = (mine + 15) & ~15; i < width; i += 16) {
                    const uint32_t w[4] = {0u, 0u, 0u, 0u};
                    put16(key0 + i, w);
                }
                tcgen05_fence_before();
                if (apart) mbar_arrive(smem_u32(&bars.s_free[stage]));
                if constexpr (WIDE) part_sum[stage][half][t] = rsum;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(smem_u32(&bars.r_ready[stage]));
                if constexpr (WIDE) {
                    ok = meet(1);
                    if (!ok) break;
                    rsum += part_sum[stage][half ^ 1][t];
                }
                const RowFactor f = row_factor(a, (int64_t)F * n + (int64_t)e.y * rsum, scale);
                if (!sums) {
                    ok = wait(&bars.sum_full[kc % kChunks], (kc / kChunks) & 1);
                    sums = true;
                }
                if (ok) ok = wait(&bars.o_full[stage], phase);
                if (!ok) break;
                tcgen05_fence_after();
                // ---- the rows' outputs, 64 bytes of each at a time, through the warp's part of the panel, from which neighbouring lanes store a row.
                // Sums below 2^22 (ordinary tables) become floats by their place in the mantissa of 1.5 * 2^23, which the products' addend has in
                // it already; their product with rho is a whole number below 2^24, so exact.  (A converter has a quarter of the other
                // pipes' rate: with it 24 ragged texts on 256 patches, leading-bit reciprocal, took 57 us.)
                const bool small = OUT != HCCS_I32 && __all_sync(~0u, F * n + e.y * rsum < 32768 && f.unit == 1.0f);
                const int whole_rho = a.recip == HCCS_RECIP_REAL ? 1 : f.rho;
                const float rho = (float)whole_rho;
                const int by_r = e.y * (small ? 1 : whole_rho), by_v = F * (small ? 1 : whole_rho);
                const uint32_t magic = small ? 0x4b400000u : 0u;
                auto pack = [&](uint32_t (&o)[kDimsAtATime], int i, float v, float w) {
                    if constexpr (OUT == HCCS_F32) {
                        o[i] = __float_as_uint(v);
                        o[i + 1] = __float_as_uint(w);
                    } else if constexpr (OUT == HCCS_BF16) {
                        const __nv_bfloat162 b2 = __floats2bfloat162_rn(v, w);
                        o[i >> 1] = *reinterpret_cast<const uint32_t *>(&b2);
                    } else {
                        const __half2 h2 = __floats2half2_rn(v, w);
                        o[i >> 1] = *reinterpret_cast<const uint32_t *>(&h2);
                    }
                };
#pragma unroll 1
                for (int y = 0; y < kDims / kDimsAtATime; ++y) {
                    if (y > 0 && (y * 4) % kRowLanes == 0) stored();
                    uint32_t o[kDimsAtATime];
                    tmem_ld(o_at + y * kDimsAtATime, o);
#pragma unroll
                    for (int i = 0; i < kDimsAtATime; i += 4) {
                        const int4 vs = *reinterpret_cast<const int4 *>(&vsum[kc % kChunks][half * kDims + y * kDimsAtATime + i]);
                        o[i] = (uint32_t)by_r * o[i] + ((uint32_t)by_v * (uint32_t)vs.x + magic);
                        o[i + 1] = (uint32_t)by_r * o[i + 1] + ((uint32_t)by_v * (uint32_t)vs.y + magic);
                        o[i + 2] = (uint32_t)by_r * o[i + 2] + ((uint32_t)by_v * (uint32_t)vs.z + magic);
                        o[i + 3] = (uint32_t)by_r * o[i + 3] + ((uint32_t)by_v * (uint32_t)vs.w + magic);
                    }
                    if constexpr (OUT != HCCS_I32) {
                        if (small) {
#pragma unroll
                            for (int i = 0; i < kDimsAtATime; i += 2) {
                                float v = __uint_as_float(o[i]), w = __uint_as_float(o[i + 1]);
                                add2(v, w, -12582912.0f);
                                scale2(v, w, rho);
                                scale2(v, w, f.scale);
                                pack(o, i, v, w);
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < kDimsAtATime; i += 2) pack(o, i, (float)(int)o[i] * f.scale * f.unit, (float)(int)o[i + 1] * f.scale * f.unit);
                        }
                    }
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        *reinterpret_cast<uint4 *>(staged + (staged_at(lane, 0) ^ (((y * 4 + p) % kRowLanes) << 4))) = make_uint4(o[4 * p], o[4 * p + 1], o[4 * p + 2], o[4 * p + 3]);
                    if (y == kDims / kDimsAtATime - 1) {
                        tcgen05_fence_before();
                        if (!apart) mbar_arrive(smem_u32(&bars.s_free[stage]));
                    }
                    if ((y * 4 + 4) % kRowLanes == 0) {
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        store_rows(x, (y + 1) * kDimsAtATime - kStageRow / kElem, false);
                        __syncwarp();
                    }
                }
            }
            sums_read();
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
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

// Queries, or outputs, as [T][Hq][row bytes], boxes of `inner` bytes of a kv head's heads and some queries.
bool make_rows_map(CUtensorMap *map, const void *rows, int row_bytes, int inner, const CachedAttnArgs &a, int queries) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)row_bytes, (cuuint64_t)a.Hq, (cuuint64_t)a.T};
    const cuuint64_t strides[2] = {(cuuint64_t)row_bytes, (cuuint64_t)a.Hq * row_bytes};
    const cuuint32_t box[3] = {(cuuint32_t)inner, (cuuint32_t)a.group, (cuuint32_t)queries};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void *>(rows), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              inner == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr size_t kMaxSmem = 219 * 1024;    // dynamic; the kernel's own arrays take up to 7 KB more

template <int D, int OUT, bool WIDE>
cudaError_t launch_typed(const CachedAttnArgs &a, cudaStream_t stream) {
    auto kernel = cross_short_kernel<D, OUT, WIDE>;
    constexpr int kStages = WIDE ? 2 : 4;
    static std::atomic<bool> raised[64];
    cudaError_t e = raise_limits((const void *)kernel, (int)kMaxSmem, raised);
    int dev = 0, sms = 0;
    if (e == cudaSuccess) e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    ShortPlan p;
    p.queries = kTile / a.group;
    p.keys = a.max_kv <= 32 ? 32 : (a.max_kv + 31) / 32 * 32;
    const size_t fixed = 1024 + kStages * ((size_t)kTile * D + (size_t)((p.keys + 127) / 128) * kTile * 128), kv = (size_t)p.keys * D;
    // Four chunks on their way where there is room: sequences of few queries are chunks of one tile, and V's place is taken until the tile's
    // last product
    p.k_shift = fixed + 8 * kv <= kMaxSmem ? 2 : 1;
    p.v_shift = p.k_shift == 2 ? 2 : fixed + 4 * kv <= kMaxSmem ? 1 : 0;
    const size_t smem = fixed + (kv << p.k_shift) + (kv << p.v_shift);
    // (a warp's rows are whole queries where the heads of a kv head divide 32; the map of the outputs is not used otherwise)
    p.warp_queries = 32 % a.group == 0 ? 32 / a.group : 0;
    constexpr int kElem = OUT == HCCS_I32 || OUT == HCCS_F32 ? 4 : 2, kRow = (WIDE ? D / 2 : D) * kElem;
    CUtensorMap mq, mk, mv, mo;
    if (!make_rows_map(&mq, a.Q, D, D, a, p.queries) || !make_rows_map(&mo, a.O, D * kElem, kRow < 128 ? kRow : 128, a, p.warp_queries ? p.warp_queries : 1) || !make_states_map(&mk, a.k_pages, a.k_stride, a, p.keys) || !make_states_map(&mv, a.v_pages, a.v_stride, a, p.keys))
        return cudaErrorInvalidValue;
    const int64_t most = (int64_t)a.B * a.Hkv * (((int64_t)a.max_q + p.queries - 1) / p.queries);      // tiles
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(most < sms ? most : sms));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, mq, mk, mv, mo, p);
}

template <int D, bool WIDE>
cudaError_t launch_keys(const CachedAttnArgs &a, cudaStream_t stream) {
    switch (a.out_type) {
        case HCCS_I32: return launch_typed<D, HCCS_I32, WIDE>(a, stream);
        case HCCS_F32: return launch_typed<D, HCCS_F32, WIDE>(a, stream);
        case HCCS_BF16: return launch_typed<D, HCCS_BF16, WIDE>(a, stream);
        default: return launch_typed<D, HCCS_F16, WIDE>(a, stream);
    }
}

template <int D>
cudaError_t launch_head_dim(const CachedAttnArgs &a, cudaStream_t stream) {
    return a.max_kv > 128 ? launch_keys<D, true>(a, stream) : launch_keys<D, false>(a, stream);
}

}  // namespace

bool cross_short_fits(const CachedAttnArgs &a) { return !a.key_range && a.max_kv <= kMaxKeys && a.group <= kTile; }

cudaError_t launch_cross_short(const CachedAttnArgs &a, cudaStream_t stream) {
    return a.d == 128 ? launch_head_dim<128>(a, stream) : launch_head_dim<64>(a, stream);
}

}  // namespace hccs
