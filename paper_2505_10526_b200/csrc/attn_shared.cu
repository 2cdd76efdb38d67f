// Verify attention of sequences whose contexts begin with the same positions (massv_verify_attn_shared).
//
// softmax over positions [0, L + j] is the merge of softmax over a shared prefix [0, s) and over the rest: with m the maximum,
// l the sum and O the weighted values of each part relative to its m,
//   out = sum_i O_i 2^(m_i - M) / sum_i l_i 2^(m_i - M),   M = max m_i.
// The prefix is read once per group: the rows of all its sequences stand together, so that what was a stream of bytes per sequence
// becomes a matrix product of hundreds to thousands of rows with the prefix; the rest is read per sequence.  Both run in
// one kernel on tcgen05, in blocks of 128 positions:
//
//   S[128, 128] = Q[128 rows, d] K_block^T          Q and K in shared memory as TMA writes them, S in tensor memory
//   P           = 2^(S scale log2 e - reference)    one row per thread; bf16, back into the columns of S
//   O[128, d]  += P[128, 128] V_block               P read from tensor memory, V from shared memory
//
// PREFIX items: a tile is as many whole (sequence, block row) pairs of a KV head's G query heads as fit 128 rows.  At head_dim 64 and
// 128 a CTA works on two tiles at once, so that one tile's products run under the other's exponentials; both share each K and V
// block; each tile's products are issued by a warp of its own, 64 positions at a time, so that a tile's next scores are made while its
// softmax is at the other half.  At 256 the accumulator leaves room for one, whose scores are double buffered instead.  Every position is
// seen by every row.
// TAIL items: the positions of one sequence behind the prefix, block rows included (appended here), for its G * R <= 64 rows.  The
// blocks of all tails of a CTA form one pipeline across items (the next item's queries have a buffer of their own): the scores run two
// blocks ahead of the weights, and where there is room for two accumulators the blocks alternate between them.
//
// Warps 0 and 3 copy K and V (TMA), each into a ring of its own; warp 1 issues the products, for a second tile warp 2 does, which in tails
// patches the block's own K rows into the blocks that hold their positions and stores them to their page slots, as the last warp does
// with V's; four warps per tile make the softmax.
//
// All items form one line, a block costing what its kind costs (below), cut into equal ranges for a persistent grid of one CTA per
// SM: prefix items, which the tensor cores bound, and tails, which memory bounds, are at work at the same time.  What a CTA has
// of an item is a piece (O, m, l); attn_shared_merge_kernel adds the pieces of every row up, in order.
//
// What bounds it: a two-tile block at head_dim 128 is 2,560 cycles of products (64 for each 128 x 128 x 16 with V; 48 instead of 32 for one of 64
// scores, whose operands shared memory cannot deliver faster) and 2,048 of exponentials, and takes about 3,300: products,
// copies and tensor-memory traffic share one shared memory.  At 64 the products are 1,280 cycles and the exponentials, as many as before, are
// the floor (1.1 PFLOP/s).  At 256 one tile's products (2,048) and softmax take turns.  Kernel alone, 64 sequences of 6 rows: prefixes (28 / 4
// heads of 64 and of 128 behind 16,384 positions, 16 / 8 of 256 behind 8,192) at 430, 770 and 445 TFLOP/s; tails (28 / 4 of 64 and of 128,
// 2,000 positions each, 16 / 8 of 256, 1,000) at 2.4, 3.7 and 5.3 TB/s of K and V: a block's chain of scores, softmax and product is
// exposed with two blocks in flight, the more the fewer bytes a block has.
#include "kernels.cuh"
#include "ptx.cuh"
#include "umma.cuh"

namespace massv {

namespace {

constexpr int kTileRows = 128;
constexpr int kPagesPerBlock = kPrefixBlock / kPageSize;
constexpr float kRescaleThreshold = 8.f;   // log2 units a row's maximum may outgrow its reference by

// Cost of a block: products of two tiles, of one, of a tail; and what an item costs beside its blocks (queries, write-out).  Set by
// measurement: equal ranges should take equal time (calls back to back on the same inputs: 64 sequences of 28 heads of 128 in three groups, prefixes
// up to 16,384: 129 us, with 7 for two tiles and 8 for a tail 137; 31 of 16 heads of 256, two groups up to 4,111: 62 us, with 7 for one tile 64).
// One set serves all head dimensions; it was not fitted to 64, nor to calls of mostly tails.
constexpr int kCostTwo = 8, kCostOne = 6, kCostTail = 7, kCostPrefixItem = 8, kCostTailItem = 5;
constexpr int kCostMost = kCostTwo + kCostPrefixItem;

// Blocks of an item that begins at `start`: block 0 there, block k > 0 at start + item + k * block.  The first block that begins at or
// behind position f of the line (n or more: none).
__device__ __forceinline__ int first_block(int f, int start, int block, int item) {
    return f <= start ? 0 : max(1, (f - start - item + block - 1) / block);
}
__device__ __forceinline__ int block_begin(int k, int start, int block, int item) { return k == 0 ? start : start + item + k * block; }

template <int D>
struct SharedCfg {
    static constexpr int kTiles = D == 256 ? 1 : 2;           // query tiles of a CTA
    static constexpr int kParts = D == 256 ? 2 : 1;           // ring entries of a K block (halves of d) and of a V block (halves of the positions)
    static constexpr int kNCH = D / 64;
    static constexpr int kQTile = kTileRows * D * 2;
    static constexpr int kEntry = kPrefixBlock * D * 2 / kParts;
    static constexpr int kEntries = D == 64 ? 4 : 2;         // of each ring
    static constexpr int kBoxes = kPagesPerBlock * kNCH / kParts;      // 16-position x 64-element boxes of an entry
    static constexpr int kSmem = kTiles * kQTile + 2 * kEntries * kEntry + 1024;      // and the line (line_ints)
    static constexpr int kThreads = 160 + kTiles * 128;
    static constexpr uint32_t kTmemCols = 512;
    static constexpr uint32_t kTmemO = 2 * kPrefixBlock;      // two score buffers, then the accumulators
    static constexpr int kMaxSmem = kSmem + (kSharedMaxBatch + 1 + 5 * (kMaxGroups + 1)) * 4;
    static_assert(kBoxes <= 32 && kTmemO + kTiles * D <= kTmemCols && kMaxSmem <= 226 * 1024, "fits");
};

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// 32 columns of this warp's 32 lanes: register c is column c of the thread's row.
__device__ __forceinline__ void tmem_ld_row32(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_row16(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_st_row16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), "r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
        "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
template <int N>
__device__ __forceinline__ void tmem_ld_wait(uint32_t (&r)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+r"(r[j]));       // no use may move ahead of the wait
}

// Where a piece is kept: slots of the CTAs' cut items (two each), slots of prefix items that one CTA has all of, slots of such tails.
// The number of rows of the pieces ahead of it, and how many it has itself.  A piece's values are [d / 4][rows] groups of four
// columns, its references (log2 units) and sums [rows] pairs.
__device__ __forceinline__ long long piece_rows(const SharedAttnParams& p, int slot, int x, int& n_rows) {
    const SharedAttnSlots& s = p.slots;
    const int item = -1 - slot;
    long long rows;
    n_rows = kTileRows;
    if (slot >= 0) rows = ((long long)slot * s.tiles + x) * kTileRows;
    else if (item < s.prefix_items) rows = ((long long)(s.cut + item) * s.tiles + x) * kTileRows;
    else {
        n_rows = s.tail_rows;
        rows = (long long)(s.cut + s.prefix_items) * s.tiles * kTileRows + ((long long)(item - s.prefix_items) * s.tiles + x) * n_rows;
    }
    if (!MASSV_IN_BOUNDS(rows + n_rows, (long long)s.rows() + 1, p.a.dev_status)) rows = 0;
    return rows;
}

// ---- the line of work, in shared memory: what every role finds its pieces by
struct Line {
    const int* gs;        // [n_groups + 1] first sequence of each group (all sequences in group 0 with no blocks where the groups are none)
    const int* gcost;     // [n_groups + 1] cost of the prefix items of groups 0 .. g-1
    const int* gitem;     // [n_groups + 1] their number
    const int* gblocks;   // [n_groups] blocks of the shared prefix
    const int* gsrc;      // [n_groups] the sequence whose page table is read for it
    const int* tail;      // [B + 1] cost of the tails of sequences 0 .. b-1, per KV head
    int n_groups, B;
};
__device__ __forceinline__ int find_last(const int* cum, int n, int u) {       // the largest i < n with cum[i] <= u
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cum[mid] <= u) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// A run of blocks of one item.
struct Run {
    int tail;            // (truth value)
    int head, seq;       // seq: whose page table is read
    int blk0;            // first (sequence, block row) pair of the rows
    int n_rows[2];       // query rows of each tile
    int pos0;            // position of the first block
    int n;               // blocks; 0 behind the last run
    int L;               // tail: committed length
    int slot;            // slot of its piece: >= 0 one of the CTA's two, else -1 - item for an item that the CTA has all of (prefix items, then tails)
};

constexpr int kRunQueue = 8;

template <int D>
__global__ void __launch_bounds__(SharedCfg<D>::kThreads, 1)
attn_shared_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_q,
                   const __grid_constant__ CUtensorMap map_qt, const SharedAttnParams p) {
    using Cfg = SharedCfg<D>;
    constexpr int E = Cfg::kEntries, NT = Cfg::kTiles, PARTS = Cfg::kParts, NCH = Cfg::kNCH;
    constexpr int UPR = D / 8;             // 16-byte units per K/V row
    extern __shared__ uint8_t smem_raw[];
    // rings: K's entries, then V's
    __shared__ __align__(8) uint64_t ready_bar[2 * E], empty_bar[2 * E];
    __shared__ __align__(8) uint64_t landed_bar[2 * E];                // the bytes of an entry that still needs patching
    __shared__ __align__(8) uint64_t q_ready_bar[2], q_free_bar[2];   // by query buffer: a prefix item has both, tails take turns
    __shared__ __align__(8) uint64_t s_full_bar[2][2], p_full_bar[2][2];      // by score buffer; of the first and the second 64 positions
    __shared__ __align__(8) uint64_t o_full_bar[2], o_free_bar[2];     // by tile
    __shared__ __align__(8) uint64_t pv_done_bar;                      // one tile: O is up to date
    __shared__ __align__(8) uint64_t pv_half_bar[2];                   // by accumulator: it has the first 64 positions of a block
    __shared__ __align__(8) uint64_t two_done_bar;                     // the second tile's products of all prefix items are done (one phase)
    __shared__ __align__(8) uint64_t run_ready_bar[kRunQueue], run_free_bar[kRunQueue];      // the runs, worked out by the K warp for all
    __shared__ Run s_runs[kRunQueue];
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int R = p.a.R, B = p.a.B;
    const int G = p.a.Hq / p.a.Hkv, nb = kTileRows / G, tile_rows = nb * G;
    // barriers, one thread each (45 initialisations by one thread take 1,100 cycles)
    {
        struct { uint64_t* bar; int n, arrivals; } const kinds[] = {
            {ready_bar, 2 * E, 1}, {empty_bar, 2 * E, NT}, {landed_bar, 2 * E, 1}, {q_ready_bar, 2, 1}, {q_free_bar, 2, NT}, {&s_full_bar[0][0], 4, 1}, {&p_full_bar[0][0], 4, 4},
            {o_full_bar, 2, 1}, {o_free_bar, 2, 4}, {&pv_done_bar, 1, 1}, {pv_half_bar, 2, 1}, {&two_done_bar, 1, 1}, {run_ready_bar, kRunQueue, 1},
            {run_free_bar, kRunQueue, 4 + 4 * NT}};                   // V, two helpers, products, softmax
        int at = threadIdx.x;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(kinds) / sizeof(kinds[0])); ++i) {
            if (at >= 0 && at < kinds[i].n) mbar_init(kinds[i].bar + at, kinds[i].arrivals);
            at -= kinds[i].n;
        }
        if (threadIdx.x == 0) abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(Cfg::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* q_smem = smem;                                            // [tile][d / 64][128 rows][128 B], swizzled
    // Where a tail's queries go: a tile's place each, or (one tile) the two halves of its rows.  A product of 128 rows from the
    // second half on reads 64 rows of what stands behind it: rows nobody takes.
    constexpr int kQTurn = NT == 2 ? Cfg::kQTile : 64 * 128;
    uint8_t* ring_smem = q_smem + NT * Cfg::kQTile;
    int* gs = reinterpret_cast<int*>(ring_smem + 2 * E * Cfg::kEntry);
    int *gcost = gs + p.n_groups + 1, *gitem = gcost + p.n_groups + 1, *gblocks = gitem + p.n_groups + 1, *gsrc = gblocks + p.n_groups, *tail = gsrc + p.n_groups;
    const Line ln{gs, gcost, gitem, gblocks, gsrc, tail, p.n_groups, B};
    // rows past the last pair of a tile are never copied
    for (int i = threadIdx.x; i < NT * NCH * (kTileRows - tile_rows) * 8; i += blockDim.x) {
        const int per = (kTileRows - tile_rows) * 8, region = i / per, k = i - region * per;
        *reinterpret_cast<uint4*>(q_smem + region * (kTileRows * 128) + tile_rows * 128 + k * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    pdl_wait();

    // ---- groups: the least length of the members and their number (gcost, gitem for the moment), the first sequence
    auto fits = [&](int L) { return has_room(L, R, p.a.max_pages); };
    bool bad_here = false;
    {
        // (the first round's loads are all asked for before any is used)
        const int t = threadIdx.x, n = p.n_groups;
        const int L0 = t < B ? p.a.seq_lens[t] : 0, g0 = t <= n ? p.group_start[t] : 0, g1 = t < n ? p.group_start[t + 1] : 0, sh = t < n ? p.shared_lens[t] : 0;
        if (t <= n) gs[t] = g0;
        if (t < n) { gcost[t] = 0x7fffffff; gitem[t] = 0; gsrc[t] = 0x7fffffff; gblocks[t] = sh; }
        bad_here = (t == 0 && g0 != 0) || (t == n && g0 != B) || (t < n && g0 > g1);
        if (t < B) tail[t + 1] = L0;
        for (int b = t + blockDim.x; b < B; b += blockDim.x) tail[b + 1] = p.a.seq_lens[b];
    }
    const bool bad = __syncthreads_or(bad_here) != 0;      // (at most 256 groups: one round)
    if (bad) {                              // one group that shares nothing
        for (int i = threadIdx.x; i <= p.n_groups; i += blockDim.x) { gs[i] = i == 0 ? 0 : B; if (i < p.n_groups) gblocks[i] = 0; }
        __syncthreads();
    }
    for (int b = threadIdx.x; b < B; b += blockDim.x) {
        const int L = tail[b + 1], g = find_last(gs, p.n_groups, b);
        if (!fits(L)) continue;
        atomicMin(&gcost[g], L);
        atomicMin(&gsrc[g], b);
        atomicAdd(&gitem[g], 1);
    }
    __syncthreads();
    {
        // whole blocks that every member has committed; a sequence alone shares nothing
        const int i = threadIdx.x;
        int items = 0, cost = 0;
        if (i < p.n_groups) {
            const int blocks = gitem[i] < 2 ? 0 : max(0, min(gblocks[i], gcost[i])) / kPrefixBlock;
            const int pairs = (gs[i + 1] - gs[i]) * R, tiles = (pairs + nb - 1) / nb;
            gblocks[i] = blocks;
            items = blocks > 0 ? (tiles + NT - 1) / NT * p.a.Hkv : 0;
            cost = items * (blocks * (NT == 2 && tiles > 1 ? kCostTwo : kCostOne) + kCostPrefixItem);
        }
        __syncthreads();
        if (i < p.n_groups) { gitem[i + 1] = items; gcost[i + 1] = cost; }
        if (i == 0) { gcost[0] = 0; gitem[0] = 0; tail[0] = 0; }
    }
    for (int b = threadIdx.x; b < B; b += blockDim.x) {
        const int L = tail[b + 1];
        const bool ok = fits(L);
        if (!ok && blockIdx.x == 0) set_status(p.a.dev_status, MASSV_ERR_CAPACITY);
        tail[b + 1] = ok ? ((L + R + kPrefixBlock - 1) / kPrefixBlock - gblocks[find_last(gs, p.n_groups, b)]) * kCostTail + kCostTailItem : 0;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0 || warp == 2 || warp == 3) {      // running sums of cum[1 .. n], one warp each, 32 at a time
        int* cum = warp == 0 ? gcost : warp == 2 ? gitem : tail;
        const int n = warp == 3 ? B : p.n_groups;
        int run = 0;
        for (int i0 = 1; i0 <= n; i0 += 32) {
            const int i = i0 + lane;
            int incl = i <= n ? cum[i] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            if (i <= n) cum[i] = run + incl;
            run += __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    __syncthreads();
    const int tails0 = gcost[p.n_groups];                              // where the tails begin on the line
    const int total = tails0 + tail[B] * p.a.Hkv;
    const int per = max(kCostMost, (total + (int)gridDim.x - 1) / (int)gridDim.x);       // (no block is longer than a range)
    if (blockIdx.x == 0) {
        if (threadIdx.x == 0) {
            p.meta[0] = per; p.meta[1] = tails0;
            if (bad) set_status(p.a.dev_status, MASSV_ERR_INVALID_ARG);
        }
        for (int b = threadIdx.x; b < B; b += blockDim.x) {
            const int g = find_last(gs, p.n_groups, b);
            p.seqs[b] = make_int4(tail[b], (tail[b + 1] - tail[b] - kCostTailItem) / kCostTail, (b - gs[g]) * R, gblocks[g]);
            p.seq_groups[b] = make_int4(gcost[g], gitem[g], NT == 2 && (gs[g + 1] - gs[g]) * R > nb ? kCostTwo : kCostOne, 0);
        }
    }

    // ---- this CTA's range: the blocks that begin in it
    const int f_begin = min((long long)total, (long long)blockIdx.x * per), f_end = min((long long)total, (long long)f_begin + per);
    // The blocks at or behind f of the item that position f of the line lies in (or of the next one), and f behind them.
    auto next_run = [&](int& f, Run& r) -> bool {
        while (f < f_end) {
            int start, n_all, cost, extra, item;
            if (f < tails0) {
                const int g = find_last(ln.gcost, ln.n_groups, f), pairs = (ln.gs[g + 1] - ln.gs[g]) * R;
                cost = NT == 2 && pairs > nb ? kCostTwo : kCostOne;
                extra = kCostPrefixItem;
                n_all = ln.gblocks[g];
                const int length = n_all * cost + extra, k = (f - ln.gcost[g]) / length, tile = k / p.a.Hkv, done = tile * nb * NT;
                start = ln.gcost[g] + k * length;
                item = ln.gitem[g] + k;
                r.tail = 0;
                r.head = k - tile * p.a.Hkv;
                r.seq = ln.gsrc[g];
                r.blk0 = ln.gs[g] * R + done;
                r.n_rows[0] = min(nb, pairs - done) * G;
                r.n_rows[1] = NT == 2 ? max(0, min(nb, pairs - done - nb)) * G : 0;
                r.pos0 = 0;
                r.L = 0;
            } else {
                const int u = f - tails0, b = find_last(ln.tail, B, u / p.a.Hkv), length = ln.tail[b + 1] - ln.tail[b];      // (head after head)
                cost = kCostTail;
                extra = kCostTailItem;
                n_all = (length - extra) / cost;
                r.head = (u - ln.tail[b] * p.a.Hkv) / length;
                start = tails0 + ln.tail[b] * p.a.Hkv + r.head * length;
                item = p.slots.prefix_items + b * p.a.Hkv + r.head;
                r.tail = 1;
                r.seq = b;
                r.blk0 = b * R;
                r.n_rows[0] = r.n_rows[1] = R * G;
                r.pos0 = ln.gblocks[find_last(ln.gs, ln.n_groups, b)] * kPrefixBlock;
                r.L = p.a.seq_lens[b];
            }
            const int k0 = first_block(f, start, cost, extra), k1 = min(n_all, first_block(f_end, start, cost, extra));
            f = k1 == n_all ? start + extra + n_all * cost : f_end;
            if (k0 >= k1) continue;         // the item's last block begins ahead of the range
            r.pos0 += k0 * kPrefixBlock;
            r.n = k1 - k0;
            // an item that began in an earlier CTA's range has slot 0, one that runs on into the next has slot 1
            r.slot = k0 == 0 && k1 == n_all ? -1 - item : (int)blockIdx.x * 2 + (k0 > 0 ? 0 : 1);
            return true;
        }
        r.n = 0;
        return false;
    };

    constexpr uint32_t tmem_base = 0;                                  // all 512 columns are this CTA's: they begin at 0
    volatile int* abort_ptr = &abort_flag;
    // Run i of the queue; n 0 where there is none (or a wait gave up).  keep: the caller reads it again.
    auto take_run = [&](int i, Run& r, bool keep) -> bool {
        const bool ok = mbar_wait_warp(&run_ready_bar[i % kRunQueue], (uint32_t)(i / kRunQueue) & 1u, abort_ptr);
        r = s_runs[i % kRunQueue];
        if (!ok) r.n = 0;
        __syncwarp();
        if (!keep && lane == 0) mbar_arrive(&run_free_bar[i % kRunQueue]);
        return r.n > 0;
    };

    // ------------------------------------------------ products of prefix items on two tiles: warp 1 issues the first tile's, warp 2 the second's
    // (A wait takes 200 cycles in these warps even where there is nothing to wait for, since the products keep shared memory busy: one warp for
    // both tiles is at it all the time and no faster.)  The whole warp runs this code, so that addresses and descriptors stay warp-uniform;
    // one elected lane issues.
    const uint32_t lead = elect_one();
    const uint32_t q_lo = umma_desc_lo(smem_u32(q_smem)), k_lo0 = umma_desc_lo(smem_u32(ring_smem));
    const uint32_t v_lo0 = (((smem_u32(ring_smem) + E * Cfg::kEntry) & 0x3FFFFu) >> 4) | ((uint32_t)((kPrefixBlock / PARTS * 128) >> 4) << 16);
    constexpr uint32_t idesc_pv = umma_idesc_bf16(kTileRows, D, true);
    Run pr;
    int p_run = 0, p_blk = 0, p_two = 0, p_blk_two = 0;                // prefix items so far, their blocks; of these on two tiles
    bool p_any = false;
    if (warp == 1 || (NT == 2 && warp == 2)) p_any = take_run(0, pr, true);
    if constexpr (NT == 2) {
        if (warp == 1 || warp == 2) {
            const int x = warp - 1;
            bool ok = true;
            auto wait = [&](uint64_t* bar, uint32_t parity) { if (!mbar_wait_warp(bar, parity, abort_ptr)) ok = false; };
            for (; ok && p_any && !pr.tail; p_any = take_run(++p_run, pr, true)) {
                if (lane == 0) mbar_arrive(&run_free_bar[p_run % kRunQueue]);
                const int n = pr.n, tau = x ? p_blk_two : p_blk, use = x ? p_two : p_run;
                const bool two = pr.n_rows[1] > 0;
                if (x == 1 && !two) {
                    // One tile: the second tile's warp still sees every phase of the barriers and gives back what it has no use for.  (Passing the
                    // run by, it could reach the next one while this one's copies are in flight, and a wait for the next phase, which has
                    // the parity of the phase before this one, would pass at once.)
                    wait(&q_ready_bar[0], (uint32_t)p_run & 1u);
                    if (lane == 0) mbar_arrive(&q_free_bar[0]);
                    for (int b = p_blk; b < p_blk + n && ok; ++b) {
#pragma unroll
                        for (int ring = 0; ring < 2 * E; ring += E) {
                            wait(&ready_bar[ring + b % E], (uint32_t)(b / E) & 1u);
                            if (lane == 0) mbar_arrive(&empty_bar[ring + b % E]);
                        }
                    }
                } else {
                    wait(&q_ready_bar[0], (uint32_t)p_run & 1u);
                    for (int t = -1; t < n && ok; ++t) {
                        // 64 positions at a time: the weights of block t times V, then, over what they left, the scores of block t + 1.  So the
                        // scores that a tile's softmax takes next are made while it is at the other half.
                        const int kb = p_blk + t + 1, vb = p_blk + t;
                        // (the three in one: their latencies overlap)
                        if (t == 0) wait(&o_free_bar[x], (uint32_t)(use & 1) ^ 1u);
                        uint64_t *const k_ready = &ready_bar[kb % E], *const v_ready = &ready_bar[E + vb % E];
                        const uint32_t k_lap = (uint32_t)(kb / E) & 1u, v_lap = (uint32_t)(vb / E) & 1u, p_lap = (uint32_t)(tau + t) & 1u;
                        if (t < 0) wait(k_ready, k_lap);
                        else if (!mbar_wait_warp3(v_ready, v_lap, t + 1 < n ? k_ready : v_ready, t + 1 < n ? k_lap : v_lap, &p_full_bar[x][0], p_lap, abort_ptr)) ok = false;
                        const uint32_t k_lo = k_lo0 + (uint32_t)(kb % E * (Cfg::kEntry >> 4)), v_lo = v_lo0 + (uint32_t)(vb % E * (Cfg::kEntry >> 4));
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const uint32_t s_tmem = tmem_base + (uint32_t)(x * kPrefixBlock + half * (kPrefixBlock / 2));
                            if (t >= 0) {
                                if (half == 1) wait(&p_full_bar[x][1], p_lap);
                                if (!ok) break;
                                tc_fence_after();
#pragma unroll
                                for (int ks = 0; ks < kPrefixBlock / 32; ++ks)
                                    umma_bf16_ts_lead(lead, tmem_base + Cfg::kTmemO + (uint32_t)(x * D), s_tmem + (uint32_t)(ks * 8),
                                                      v_lo + (uint32_t)((half * (kPrefixBlock / 2 * 128) + ks * 2048) >> 4), idesc_pv, t == 0 && half == 0 && ks == 0 ? 0u : 1u);
                                if (half == 0) umma_commit_lead(lead, &pv_half_bar[x]);
                            }
                            if (!ok) break;
                            if (t + 1 < n) {
                                tc_fence_after();
#pragma unroll
                                for (int kk = 0; kk < D / 16; ++kk)
                                    umma_bf16_lead(lead, s_tmem, q_lo + (uint32_t)((x * Cfg::kQTile + (kk >> 2) * (kTileRows * 128) + (kk & 3) * 32) >> 4),
                                                   k_lo + (uint32_t)((half * (kPrefixBlock / 2 * 128) + (kk >> 2) * (kPrefixBlock * 128) + (kk & 3) * 32) >> 4),
                                                   umma_idesc_bf16(kTileRows, kPrefixBlock / 2, false), kk == 0 ? 0u : 1u);
                                umma_commit_lead(lead, &s_full_bar[x][half]);
                            } else if (half == 1) {
                                umma_commit_lead(lead, &o_full_bar[x]);
                            }
                        }
                        if (!ok) break;
                        if (t >= 0) umma_commit_lead(lead, &empty_bar[E + vb % E]);
                        if (t + 1 < n) umma_commit_lead(lead, &empty_bar[kb % E]);
                        if (t + 2 == n) umma_commit_lead(lead, &q_free_bar[0]);
                    }
                }
                p_blk += n;
                if (two) { p_blk_two += n; ++p_two; }
            }
            if (x == 1 && p_two > 0) umma_commit_lead(lead, &two_done_bar);
            if (!ok) p_any = false;
        }
    }

    if (warp == 0 || warp == 3) {
        // ------------------------------------------------ copies: K (and the queries) by warp 0, V by warp 3
        const bool is_v = warp == 3;
        uint64_t policy;
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
        // This lane's 16-position x 64-element box of an entry: K parts are halves of d, V parts halves of the positions.
        const int groups = is_v ? NCH : NCH / PARTS, pages = Cfg::kBoxes / groups;
        const int c = lane % groups, pg = lane / groups, box = c * (pages * kPageSize * 128) + pg * 2048;
        const CUtensorMap* map = is_v ? &map_v : &map_k;
        uint8_t* ring = ring_smem + (is_v ? E * Cfg::kEntry : 0);
        uint64_t *ready = ready_bar + (is_v ? E : 0), *landed = landed_bar + (is_v ? E : 0), *empty = empty_bar + (is_v ? E : 0);
        int f = f_begin, e = 0, turn = 0;          // ring entry; tails so far
        uint32_t lap = 1;                          // parity to wait for: an entry's first use does not wait
        int q_uses[2] = {0, 0};
        bool ok = true;
        Run r;
        for (int run = 0; ok; ++run) {
            if (is_v) {
                if (!take_run(run, r, false)) break;
            } else {
                if (run >= kRunQueue && !mbar_wait_warp(&run_free_bar[run % kRunQueue], (uint32_t)(run / kRunQueue - 1) & 1u, abort_ptr)) break;
                const bool any = next_run(f, r);
                if (lane == 0) {
                    s_runs[run % kRunQueue] = r;
                    mbar_arrive(&run_ready_bar[run % kRunQueue]);
                }
                __syncwarp();
                if (!any) break;
            }
            if (!is_v) {
                const int buf = r.tail ? turn++ & 1 : 0, used = buf ? q_uses[1]++ : q_uses[0]++;
                if (used > 0 && !mbar_wait_warp(&q_free_bar[buf], (uint32_t)(used - 1) & 1u, abort_ptr)) break;
                const int tiles = !r.tail && r.n_rows[1] > 0 ? 2 : 1;
                if (lane == 0) mbar_expect_tx(&q_ready_bar[buf], (uint32_t)(tiles * (r.tail ? R * G : tile_rows) * D * 2));
                __syncwarp();
                if (lane < tiles * NCH) {
                    const int x = lane / NCH, dc = lane % NCH;
                    uint8_t* dst = q_smem + dc * (kTileRows * 128);
                    if (r.tail) tma_load_3d(dst + buf * kQTurn, &map_qt, dc * 64, r.head * G, r.blk0, &q_ready_bar[buf], policy);
                    else tma_load_3d(dst + x * Cfg::kQTile, &map_q, dc * 64, r.head * G, r.blk0 + x * nb, &q_ready_bar[buf], policy);
                }
            }
            // page ids travel in registers: lane l holds page 32 * group + l of the run, four blocks to a group
            const int32_t* pt = p.a.page_table + (size_t)r.seq * p.a.max_pages + r.pos0 / kPageSize;
            const int end = r.tail ? min(r.L + R - r.pos0, r.n * kPrefixBlock) : r.n * kPrefixBlock;      // positions of the run
            const int n_pages = (end + kPageSize - 1) / kPageSize;
            int pid_cur = lane < n_pages ? pt[lane] : 0, pid_next = 32 + lane < n_pages ? pt[32 + lane] : 0;
            for (int t = 0; t < r.n && ok; ++t) {
                if (t > 0 && t % 4 == 0) {
                    pid_cur = pid_next;
                    const int nxt = (t / 4 + 1) * 32 + lane;
                    pid_next = nxt < n_pages ? pt[nxt] : 0;
                }
                const bool patch = r.tail && r.pos0 + (t + 1) * kPrefixBlock > r.L;
                const int have = min(kPagesPerBlock, n_pages - t * kPagesPerBlock);        // pages of the block that hold positions
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                    const int page0 = is_v ? part * pages : 0, n_pg = max(0, min(pages, have - page0));
                    int pid = __shfl_sync(0xffffffffu, pid_cur, (t % 4) * kPagesPerBlock + (page0 + pg) % kPagesPerBlock);
                    if (!mbar_wait_warp(&empty[e], lap, abort_ptr)) { ok = false; break; }
                    uint64_t* bar = patch ? &landed[e] : &ready[e];
                    if (lane == 0) mbar_expect_tx(bar, (uint32_t)(n_pg * groups * 2048));
                    __syncwarp();
                    if (lane < Cfg::kBoxes && pg < n_pg) {
                        if (pid < 0 || pid >= p.a.num_pages) { set_status(p.a.dev_status, MASSV_ERR_CAPACITY); pid = 0; }
                        tma_load_2d(ring + e * Cfg::kEntry + box, map, (is_v ? c : part * groups + c) * 64, (pid * p.a.Hkv + r.head) * kPageSize, bar, policy);
                    }
                    if (++e == E) { e = 0; lap ^= 1u; }
                }
            }
        }
        if (lane == 0 && *abort_ptr) {
            for (int i = 0; i < 64; ++i) __nanosleep(2000);            // let copies in flight land
        }
    } else if (warp == 2 || warp == 4 + 4 * NT) {
        // ------------------------------------------------ helpers: the block's own rows, and what lies behind the last position
        const bool is_v = warp != 2;
        uint32_t landed_phase = 0;       // bit e: parity of the next completion of landed_bar[e]
        int it = p_blk;                  // entries of the ring so far (the K warp comes from the prefix items)
        bool ok = true;
        // Block t of a run, entry by entry.
        auto patch = [&](const Run& r, int t) {
            const int start = r.pos0 + t * kPrefixBlock, end = r.L + R;
            const int32_t* pt = p.a.page_table + (size_t)r.seq * p.a.max_pages;
            const __nv_bfloat16* src = is_v ? p.a.v_new : p.a.k_new;
            __nv_bfloat16* pool = is_v ? p.a.v_pages : p.a.k_pages;
            for (int part = 0; part < PARTS; ++part, ++it) {
                const int e = it % E + (is_v ? E : 0);
                // the entry's positions and 16-byte units of a row: K parts are halves of d, V parts halves of the positions
                constexpr int kVRows = kPrefixBlock / PARTS, kKUnits = UPR / PARTS;
                const int row0 = is_v ? part * kVRows : 0, n_row = is_v ? kVRows : kPrefixBlock, u0 = is_v ? 0 : part * kKUnits, n_u = is_v ? UPR : kKUnits;
                const int first = max(r.L, start + row0), last = min(end, start + row0 + n_row);      // new positions inside
                uint8_t* dst = ring_smem + (size_t)e * Cfg::kEntry;
                auto at = [&](int row, int u) { const int w = row - row0; return dst + (u / 8) * (n_row * 128) + w * 128 + (((u % 8) ^ (w & 7)) << 4); };
                // what comes from memory is asked for ahead of the wait
                constexpr int PRE = 4;
                const int n_units = max(0, last - first) * n_u;
                uint4 val[PRE];
                int pid[PRE];
#pragma unroll
                for (int k = 0; k < PRE; ++k) {
                    const int idx = k * 32 + lane;
                    if (idx < n_units) {
                        const int pos = first + idx / n_u, u = u0 + idx % n_u;
                        val[k] = *reinterpret_cast<const uint4*>(src + (((size_t)r.seq * R + (pos - r.L)) * p.a.Hkv + r.head) * D + u * 8);
                        pid[k] = pt[pos / kPageSize];
                    }
                }
                if (!mbar_wait_warp(&landed_bar[e], (landed_phase >> e) & 1u, abort_ptr)) { ok = false; return; }
                landed_phase ^= 1u << e;
                auto put = [&](int idx, const uint4& x, int page) {
                    const int pos = first + idx / n_u, u = u0 + idx % n_u;
                    *reinterpret_cast<uint4*>(at(pos - start, u - u0)) = x;
                    if (page >= 0 && page < p.a.num_pages)
                        *reinterpret_cast<uint4*>(pool + (((size_t)page * p.a.Hkv + r.head) * kPageSize + (pos % kPageSize)) * D + u * 8) = x;
                };
#pragma unroll
                for (int k = 0; k < PRE; ++k)
                    if (k * 32 + lane < n_units) put(k * 32 + lane, val[k], pid[k]);
                for (int idx = PRE * 32 + lane; idx < n_units; idx += 32) {
                    const int pos = first + idx / n_u, u = u0 + idx % n_u;
                    put(idx, *reinterpret_cast<const uint4*>(src + (((size_t)r.seq * R + (pos - r.L)) * p.a.Hkv + r.head) * D + u * 8), pt[pos / kPageSize]);
                }
                if (is_v) {
                    // positions past the end have weight zero, but zero times a stale NaN would still poison P V
                    const int z0 = max(row0, end - start), n_zero = row0 + n_row - z0;
                    for (int idx = lane; idx < n_zero * UPR; idx += 32) *reinterpret_cast<uint4*>(at(z0 + idx / UPR, idx % UPR)) = make_uint4(0u, 0u, 0u, 0u);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&ready_bar[e]);
            }
        };
        Run r = pr;
        int run = p_run;
        if (is_v || NT == 1) p_any = take_run(0, r, true);
        for (; ok && p_any; p_any = take_run(++run, r, true)) {
            if (lane == 0) mbar_arrive(&run_free_bar[run % kRunQueue]);
            const int t0 = r.tail ? min(r.n, max(0, r.L - r.pos0) / kPrefixBlock) : r.n;       // the first block with a position not in the cache
            it += t0 * PARTS;
            for (int t = t0; t < r.n && ok; ++t) patch(r, t);
        }
    } else if (warp == 1) {
        // ------------------------------------------------ products of everything else: one pipeline over all blocks
        constexpr uint32_t idesc_qk = umma_idesc_bf16(kTileRows, kPrefixBlock, false);
        bool ok = true;
        int ek = p_blk % E, ev = ek;                                   // ring entries
        // parities of the next waits
        uint32_t lap_k = (uint32_t)(p_blk / E) & 1u, lap_v = lap_k, s_lap[2] = {(uint32_t)p_blk & 1u, (uint32_t)p_blk_two & 1u}, q_lap[2] = {NT == 2 ? (uint32_t)p_run & 1u : 0u, 0u},
                 o_lap[2] = {(uint32_t)(p_run & 1) ^ 1u, (uint32_t)(p_two & 1) ^ 1u};
        auto wait = [&](uint64_t* bar, uint32_t parity) { if (!mbar_wait_warp(bar, parity, abort_ptr)) ok = false; };
        // S[buf] = Q K^T over `part`'s share of d; the queries q_off bytes into their place
        auto qk = [&](uint32_t q_off, int buf, int part) {
            tc_fence_after();
            const uint32_t k_lo = k_lo0 + (uint32_t)(ek * (Cfg::kEntry >> 4)), a0 = q_lo + (q_off >> 4), d_tmem = tmem_base + (uint32_t)(buf * kPrefixBlock);
#pragma unroll
            for (int kk = 0; kk < D / 16 / PARTS; ++kk) {
                const int dc = part * (NCH / PARTS) + (kk >> 2);
                umma_bf16_lead(lead, d_tmem, a0 + (uint32_t)((dc * (kTileRows * 128) + (kk & 3) * 32) >> 4),
                               k_lo + (uint32_t)(((kk >> 2) * (kPrefixBlock * 128) + (kk & 3) * 32) >> 4), idesc_qk, kk == 0 && part == 0 ? 0u : 1u);
            }
        };
        // O_x (+)= P[buf] V over one half of the positions
        auto pv = [&](int x, int buf, int half, bool first) {
            tc_fence_after();
            const uint32_t v_lo = v_lo0 + (uint32_t)(ev * (Cfg::kEntry >> 4) + (PARTS == 1 ? half * (kPrefixBlock / 2 * 128 >> 4) : 0));
            const uint32_t d_tmem = tmem_base + Cfg::kTmemO + (uint32_t)(x * D), a0 = tmem_base + (uint32_t)(buf * kPrefixBlock + half * (kPrefixBlock / 2));
#pragma unroll
            for (int ks = 0; ks < kPrefixBlock / 32; ++ks)
                umma_bf16_ts_lead(lead, d_tmem, a0 + (uint32_t)(ks * 8), v_lo + (uint32_t)((ks * 2048) >> 4), idesc_pv, ks == 0 && first ? 0u : 1u);
        };
        auto give = [&](uint64_t* bar) { umma_commit_lead(lead, bar); if (NT == 2 && lane == 0) mbar_arrive(bar); };      // (for both issuers)
        auto k_done = [&]() { give(&empty_bar[ek]); if (++ek == E) { ek = 0; lap_k ^= 1u; } };
        auto v_done = [&]() { give(&empty_bar[E + ev]); if (++ev == E) { ev = 0; lap_v ^= 1u; } };
        // (blocks of the scores and of the products: run, block within, blocks of the run)
        // A block's scores go over the P of two blocks before, behind the product that read it.
        Run kr = pr, vr = pr;
        int k_run = p_run, k_t = 0, v_run = p_run, v_t = 0;
        bool any = p_any, have_v = any;
        // The second tile's products are another warp's.  (That warp may be an item behind: a parity of o_full_bar[1] could be an older phase's.)
        if (any && p_two > 0) wait(&two_done_bar, 0u);
        int turn = 0, n_s = 0, n_p = 0;                               // tails so far (scores), blocks so far
        while (have_v && ok) {
            if (any && n_s < n_p + 2) {
                const int qb = kr.tail ? turn & 1 : 0, buf = n_s++ & 1;
                if (k_t == 0) { wait(&q_ready_bar[qb], qb ? q_lap[1] : q_lap[0]); if (qb) q_lap[1] ^= 1u; else q_lap[0] ^= 1u; }
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                    wait(&ready_bar[ek], lap_k);
                    if (!ok) break;
                    qk((uint32_t)(qb * kQTurn), buf, part);
                    k_done();
                }
                if (!ok) break;
                umma_commit_lead(lead, &s_full_bar[buf][0]);
                if (++k_t == kr.n) {
                    give(&q_free_bar[qb]);
                    if (kr.tail) ++turn;
                    any = take_run(++k_run, kr, true);
                    k_t = 0;
                }
                continue;
            }
            const int buf = n_p++ & 1, x = NT == 2 ? buf : 0;
            const bool first = NT == 2 ? v_t < 2 : v_t == 0, last = NT == 2 ? v_t >= vr.n - 2 : v_t == vr.n - 1;      // of this accumulator
            const uint32_t lap = buf ? s_lap[1] : s_lap[0];
            if (buf) s_lap[1] ^= 1u; else s_lap[0] ^= 1u;
            if (first) { wait(&o_free_bar[x], x ? o_lap[1] : o_lap[0]); if (x) o_lap[1] ^= 1u; else o_lap[0] ^= 1u; }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                // (a wait for both halves of the weights would be one for ever: the second may wait for the first's product)
                uint64_t* const p_bar = &p_full_bar[buf][half];
                if (half == 0 || PARTS == 2) { if (!mbar_wait_warp3(p_bar, lap, &ready_bar[E + ev], lap_v, p_bar, lap, abort_ptr)) ok = false; }
                else wait(p_bar, lap);
                if (!ok) break;
                pv(x, buf, half, first && half == 0);
                if (half == 0) umma_commit_lead(lead, &pv_half_bar[x]);
                if (half == 1 || PARTS == 2) v_done();
            }
            if (!ok) break;
            if (NT == 1) umma_commit_lead(lead, &pv_done_bar);
            if (last) umma_commit_lead(lead, &o_full_bar[x]);
            if (++v_t == vr.n) {
                if (lane == 0) mbar_arrive(&run_free_bar[v_run % kRunQueue]);
                have_v = take_run(++v_run, vr, true);
                v_t = 0;
            }
        }
    } else if (warp >= 4) {
        // ------------------------------------------------ softmax: a row per thread
        const int x = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tmem_o = tmem_base + Cfg::kTmemO + (uint32_t)(x * D) + lane_base;
        const float scale_log2 = p.a.scale * 1.4426950408889634f;
        bool ok = true;
        int tau = 0, uses = 0;
        int at = 0;                                                    // blocks of the pipeline ahead of this run
        Run r;
        for (int run = 0; ok && take_run(run, r, false); ++run) {
            const bool halves = NT == 2 && !r.tail;                    // the scores come 64 positions at a time
            const bool alone = r.tail && NT == 2;                      // every second block is this accumulator's
            const int turn = alone ? (at & 1) ^ x : x;                 // its first block; the place of its piece
            if (alone) at += r.n;
            if (alone ? turn >= r.n : r.n_rows[x] == 0) continue;
            const bool some = (warp & 3) * 32 < r.n_rows[x];           // this warp has rows
            const int j = min(row / G, R - 1);                         // tail: block row
            float ref = -INFINITY, l_run = 0.f;
            for (int t = alone ? turn : 0; t < r.n && ok; t += alone ? 2 : 1, ++tau) {
                const int buf = NT == 2 ? x : tau & 1;
                const uint32_t parity = (uint32_t)(NT == 2 ? tau : tau >> 1) & 1u;
                if (NT == 1 && !mbar_wait_warp(&s_full_bar[buf][0], parity, abort_ptr)) { ok = false; break; }
                tc_fence_after();
                if (some) {
                    const uint32_t tmem_s = tmem_base + lane_base + (uint32_t)(buf * kPrefixBlock);
                    const int start = r.pos0 + t * kPrefixBlock;
                    const int seen = r.tail && start + kPrefixBlock > r.L + 1 ? r.L + j - start : kPrefixBlock;      // the last column this row sees
                    const uint64_t scale2 = pack2(scale_log2, scale_log2);
                    uint64_t part[4] = {0, 0, 0, 0};                   // sums of pairs
                    // 64 columns at a time: the product with V of the first half runs under the second's exponentials, and the code is half as
                    // long (a CTA waits for its first blocks' instructions one by one).
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) {
                        if (NT == 2 && (h == 0 || halves)) {
                            if (!mbar_wait_warp(&s_full_bar[buf][h], parity, abort_ptr)) { ok = false; break; }
                            tc_fence_after();
                        }
                        uint32_t s[64];
                        tmem_ld_row32(tmem_s + (uint32_t)(h * 64), s);
                        tmem_ld_row32(tmem_s + (uint32_t)(h * 64 + 32), s + 32);
                        tmem_ld_wait(s);
                        if (seen < kPrefixBlock) {
#pragma unroll
                            for (int c = 0; c < 64; ++c) s[c] = h * 64 + c > seen ? 0xff800000u : s[c];
                        }
                        float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int c = 0; c < 64; c += 2) m4[(c >> 1) & 3] = max3(m4[(c >> 1) & 3], __uint_as_float(s[c]), __uint_as_float(s[c + 1]));
                        const float mx = max3(fmaxf(m4[0], m4[1]), m4[2], m4[3]) * scale_log2;        // (the scale is positive)
                        // The reference moves when the row's maximum has outgrown it by the threshold (and when it is first set); O and l follow it.
                        if (__any_sync(0xffffffffu, mx > ref + kRescaleThreshold)) {
                            const bool moved = mx > ref + kRescaleThreshold;
                            const float factor = moved && ref != -INFINITY ? exp2f(ref - mx) : 1.f;
                            ref = moved ? mx : ref;
                            if (__any_sync(0xffffffffu, factor != 1.f)) {
                                // O has to be up to date: with the block's first half where this is its second, else with the block before (scores
                                // in halves: those of this block's second half stand behind it; a tail with two accumulators: this block's do)
                                // (one tile: the block before comes first in both, since its product may not have begun when this block's scores
                                // are there, and the parity of pv_half_bar would be that of a phase before)
                                if (NT == 1 && !mbar_wait_warp(&pv_done_bar, (uint32_t)(tau - 1) & 1u, abort_ptr)) ok = false;
                                if (h == 1 && !mbar_wait_warp(&pv_half_bar[x], (uint32_t)tau & 1u, abort_ptr)) ok = false;
                                if (h == 0 && halves && !mbar_wait_warp(&s_full_bar[x][1], parity, abort_ptr)) ok = false;
                                if (!ok) break;
                                tc_fence_after();
#pragma unroll 1
                                for (int c0 = 0; c0 < D; c0 += 16) {
                                    uint32_t o[16];
                                    tmem_ld_row16(tmem_o + (uint32_t)c0, o);
                                    tmem_ld_wait(o);
#pragma unroll
                                    for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * factor);
                                    tmem_st_row16(tmem_o + (uint32_t)c0, o);
                                }
                                l_run *= factor;
                                const uint64_t factor2 = pack2(factor, factor);
#pragma unroll
                                for (int k = 0; k < 4; ++k) part[k] = fma2(part[k], factor2, 0);
                            }
                        }
                        const float neg = ref == -INFINITY ? 0.f : -ref;
                        const uint64_t neg2 = pack2(neg, neg);
#pragma unroll
                        for (int c0 = 0; c0 < 64; c0 += 32) {
                            uint32_t pk[16];
#pragma unroll
                            for (int c = 0; c < 16; ++c) {
                                const float2 e = unpack2(fma2(pack2(__uint_as_float(s[c0 + 2 * c]), __uint_as_float(s[c0 + 2 * c + 1])), scale2, neg2));
                                const float p0 = ex2_ftz(e.x), p1 = ex2_ftz(e.y);
                                part[c & 3] = add2(part[c & 3], pack2(p0, p1));
                                pk[c] = bf16x2(p0, p1);
                            }
                            tmem_st_row16(tmem_s + (uint32_t)(h * 64 + c0 / 2), pk);       // (over columns that have been read: P is half as wide as S)
                        }
                        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&p_full_bar[buf][h]);
                    }
                    if (!ok) break;
                    const float2 sum = unpack2(add2(add2(part[0], part[1]), add2(part[2], part[3])));
                    l_run += sum.x + sum.y;
                } else {
                    for (int h = 0; h < 2; ++h) {
                        if (NT == 2 && (h == 0 || halves) && !mbar_wait_warp(&s_full_bar[buf][h], parity, abort_ptr)) { ok = false; break; }
                        tc_fence_after();
                        tc_fence_before();
                        if (lane == 0) mbar_arrive(&p_full_bar[buf][h]);
                    }
                }
            }
            if (!ok || !mbar_wait_warp(&o_full_bar[x], (uint32_t)uses & 1u, abort_ptr)) { ok = false; break; }
            ++uses;
            tc_fence_after();
            if (some) {
                // ---- the piece
                int stride;
                const long long base = piece_rows(p, r.slot, turn, stride);
                float4* dst = reinterpret_cast<float4*>(p.part_o) + base * (D / 4) + row;
                const bool live = row < r.n_rows[x];
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 32) {
                    uint32_t o[32];
                    tmem_ld_row32(tmem_o + (uint32_t)c0, o);
                    tmem_ld_wait(o);
                    if (live) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4)
                            dst[(size_t)((c0 + k) / 4) * stride] = make_float4(__uint_as_float(o[k]), __uint_as_float(o[k + 1]), __uint_as_float(o[k + 2]), __uint_as_float(o[k + 3]));
                    }
                }
                if (live) reinterpret_cast<float2*>(p.part_ml)[base + row] = make_float2(ref, l_run);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&o_free_bar[x]);
        }
    }

    pdl_trigger();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(Cfg::kTmemCols) : "memory");
    }
    if (threadIdx.x == 0 && abort_flag) set_status(p.a.dev_status, MASSV_ERR_TIMEOUT);
}

// Pieces of a row added up.  A unit is eight columns of one query row of a (sequence, KV head) pair, rows side by side.  A thread goes through
// its unit's pieces four at a time, all their loads in flight together, with a running maximum; where there are few units, eight threads
// share one, each taking every eighth four: few units means that one prefix is cut into many pieces (whole calls, one thread to a unit against
// eight: 2 sequences behind 16,384 positions 30.3 and 22.1 us; 8 behind 2,048 25.0 and 27.5, 16 behind 2,304 28.6 and 35.4, 64 behind three long prefixes
// 128 and 170).  The order of the sums is fixed.
template <int SHARE>
__global__ void __launch_bounds__(SHARE == 1 ? 128 : 256) attn_shared_merge_kernel(const SharedAttnParams p) {
    constexpr int kUnits = SHARE == 1 ? 128 : 256 / SHARE;             // of a CTA
    __shared__ float s_red[SHARE == 1 ? 1 : 10][SHARE == 1 ? 1 : 256];
    const int h = blockIdx.x % p.a.Hkv, b = blockIdx.x / p.a.Hkv, D = p.a.d, R = p.a.R;
    const int G = p.a.Hq / p.a.Hkv, rows = G * R, nb = kTileRows / G, share = threadIdx.x / kUnits;
    const int unit = blockIdx.y * kUnits + threadIdx.x % kUnits, c8 = unit / rows, row = unit - c8 * rows;
    const SharedAttnSlots& sl = p.slots;
    const int j = row / G, hh = row - j * G;
    pdl_wait();
    pdl_trigger();
    const int4 seq = p.seqs[b], grp = p.seq_groups[b];
    const int per = p.meta[0], tails0 = p.meta[1];
    if (seq.y <= 0) return;                            // a sequence without room
    const bool live = c8 * 8 < D;
    // An item's pieces: consecutive CTAs of the kernel above; alone in one, it has a slot of its own.
    struct Pieces { int start, c0, c1, item; };
    auto pieces_of = [&](int start, int blocks, int cost, int extra, int item) { return Pieces{start, start / per, block_begin(blocks - 1, start, cost, extra) / per, item}; };
    auto slot_of = [&](const Pieces& q, int c) { return q.c0 == q.c1 ? -1 - q.item : c * 2 + (q.start < c * per ? 0 : 1); };
    const Pieces tl = pieces_of(tails0 + seq.x * p.a.Hkv + h * (seq.y * kCostTail + kCostTailItem), seq.y, kCostTail, kCostTailItem, sl.prefix_items + b * p.a.Hkv + h);
    const int pair = seq.z + j, tile = pair / nb, at_prefix = (pair - tile * nb) * G + hh, tiles = sl.tiles;
    Pieces pf{0, 0, -1, 0};
    if (seq.w > 0) {
        const int k = tile / tiles * p.a.Hkv + h;
        pf = pieces_of(grp.x + k * (seq.w * grp.z + kCostPrefixItem), seq.w, grp.z, kCostPrefixItem, grp.y + k);
    }
    const int n_prefix = pf.c1 - pf.c0 + 1, n_pieces = live ? n_prefix + (tl.c1 - tl.c0 + 1) * tiles : 0;
    const float4* po = reinterpret_cast<const float4*>(p.part_o);
    const float2* pml = reinterpret_cast<const float2*>(p.part_ml);
    float M = -INFINITY, sum = 0.f, acc[8] = {};
    for (int first = share * 4; first < n_pieces; first += 4 * SHARE) {
        float2 ml[4];
        float4 u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = first + i;
            ml[i] = make_float2(-INFINITY, 0.f);
            u[i] = v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            int slot = 0, x = tile & (tiles - 1), at = at_prefix;
            bool have = k < n_pieces;
            if (k < n_prefix) {
                slot = slot_of(pf, pf.c0 + k);
            } else if (have) {
                // a tail's piece is in two accumulators where it has more than one block
                const int w = k - n_prefix, c = tl.c0 + w / tiles;
                x = w & (tiles - 1);
                slot = slot_of(tl, c);
                at = row;
                if (x > 0) have = min(seq.y, first_block((c + 1) * per, tl.start, kCostTail, kCostTailItem)) - first_block(c * per, tl.start, kCostTail, kCostTailItem) > 1;
            }
            if (have) {
                int stride;
                const long long base = piece_rows(p, slot, x, stride);
                ml[i] = pml[base + at];
                const float4* o = po + base * (D / 4) + (long long)(2 * c8) * stride + at;
                u[i] = o[0];
                v[i] = o[stride];
            }
        }
        const float m = fmaxf(M, fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)));
        const float keep = M == -INFINITY ? 0.f : exp2f(M - m);
        M = m;
        sum *= keep;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] *= keep;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float w = ml[i].x == -INFINITY ? 0.f : exp2f(ml[i].x - m);       // (a row may see nothing of a piece)
            sum += ml[i].y * w;
            acc[0] += u[i].x * w; acc[1] += u[i].y * w; acc[2] += u[i].z * w; acc[3] += u[i].w * w;
            acc[4] += v[i].x * w; acc[5] += v[i].y * w; acc[6] += v[i].z * w; acc[7] += v[i].w * w;
        }
    }
    if constexpr (SHARE > 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s_red[i][threadIdx.x] = acc[i];
        s_red[8][threadIdx.x] = sum;
        s_red[9][threadIdx.x] = M;
        __syncthreads();
        if (share != 0) return;
        for (int g = 1; g < SHARE; ++g) M = fmaxf(M, s_red[9][g * kUnits + threadIdx.x]);
        const float own = s_red[9][threadIdx.x] == -INFINITY ? 0.f : exp2f(s_red[9][threadIdx.x] - M);
        sum *= own;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] *= own;
        for (int g = 1; g < SHARE; ++g) {
            const int from = g * kUnits + threadIdx.x;
            const float w = s_red[9][from] == -INFINITY ? 0.f : exp2f(s_red[9][from] - M);
            sum += s_red[8][from] * w;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += s_red[i][from] * w;
        }
    }
    if (!live) return;
    const float inv = 1.f / sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] *= inv;
    const size_t out = ((size_t)b * R + j) * p.a.Hq + h * G + hh;
    *reinterpret_cast<uint4*>(p.a.out + out * D + c8 * 8) = make_uint4(bf16x2(acc[0], acc[1]), bf16x2(acc[2], acc[3]), bf16x2(acc[4], acc[5]), bf16x2(acc[6], acc[7]));
    if (p.a.out_f32) {
        float4* f = reinterpret_cast<float4*>(p.a.out_f32 + out * D + c8 * 8);
        f[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        f[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
    }
    if (p.a.lse && c8 == 0) p.a.lse[out] = (M + log2f(sum)) * 0.6931471805599453f;
}

template <int D>
cudaError_t launch(const SharedAttnParams& p, cudaStream_t stream) {
    using Cfg = SharedCfg<D>;
    const int G = p.a.Hq / p.a.Hkv;
    CUtensorMap mk, mv, mq, mqt;
    const uint64_t rows_total = (uint64_t)p.a.num_pages * p.a.Hkv * kPageSize;
    if (!make_tensor_map_bf16_2d(&mk, p.a.k_pages, rows_total, D, kPageSize) || !make_tensor_map_bf16_2d(&mv, p.a.v_pages, rows_total, D, kPageSize) ||
        !make_tensor_map_bf16_heads(&mq, p.a.q, (uint64_t)p.a.B * p.a.R, (uint64_t)p.a.Hq, D, (uint32_t)(kTileRows / G), (uint32_t)G) ||
        !make_tensor_map_bf16_heads(&mqt, p.a.q, (uint64_t)p.a.B * p.a.R, (uint64_t)p.a.Hq, D, (uint32_t)p.a.R, (uint32_t)G))
        return cudaErrorInvalidValue;
    cudaError_t e = cudaFuncSetAttribute(attn_shared_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kMaxSmem);
    if (e != cudaSuccess) return e;
    int ctas = device_sm_count();
    if (ctas > kSharedMaxCtas) ctas = kSharedMaxCtas;
    const size_t smem = Cfg::kSmem + (size_t)(p.a.B + 1 + 5 * (p.n_groups + 1)) * 4;
    e = launch_pdl(attn_shared_kernel<D>, dim3(ctas), dim3(Cfg::kThreads), smem, stream, mk, mv, mq, mqt, p);
    if (e != cudaSuccess) return e;
    const int pairs = p.a.B * p.a.Hkv, units = G * p.a.R * (D / 8);
    // eight threads to a unit as long as that gives every SM no more than 512 threads
    if ((long)pairs * units * 8 > 512L * ctas) return launch_pdl(attn_shared_merge_kernel<1>, dim3(pairs, (units + 127) / 128), dim3(128), 0, stream, p);
    return launch_pdl(attn_shared_merge_kernel<8>, dim3(pairs, (units + 31) / 32), dim3(256), 0, stream, p);
}

}  // namespace

SharedAttnSlots shared_attn_slots(int B, int R, int Hq, int Hkv, int d, int n_groups) {
    SharedAttnSlots s;
    const int G = Hq / Hkv, nb = kTileRows / G;
    const long pairs = (long)B * R;
    s.tiles = d == 256 ? 1 : 2;
    s.tail_rows = (G * R + 7) / 8 * 8;
    s.prefix_items = (int)(((pairs + (long)nb * s.tiles - 1) / ((long)nb * s.tiles) + n_groups) * Hkv);
    s.cut = 2 * kSharedMaxCtas;
    s.tails = B * Hkv;
    return s;
}

cudaError_t launch_shared_attn(const SharedAttnParams& p, cudaStream_t stream) {
    const TimingHooks& hooks = timing_hooks();
    if (hooks.attn_start && cudaEventRecord(hooks.attn_start, stream) != cudaSuccess) return cudaGetLastError();
    cudaError_t e;
    switch (p.a.d) {
        case 64: e = launch<64>(p, stream); break;
        case 128: e = launch<128>(p, stream); break;
        case 256: e = launch<256>(p, stream); break;
        default: return cudaErrorInvalidValue;
    }
    if (e != cudaSuccess) return e;
    if (hooks.attn_stop && cudaEventRecord(hooks.attn_stop, stream) != cudaSuccess) return cudaGetLastError();
    count_launches(2);
    return cudaGetLastError();
}

}  // namespace massv
