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
// block.  At 256 the accumulator leaves room for one, whose scores are double buffered instead.  Every position is seen by every row.
// TAIL items: the positions of one sequence behind the prefix, block rows included (appended here), for its G * R <= 64 rows.  With room
// for two tiles, even and odd blocks go to one accumulator each, which keeps two blocks in flight.
//
// Warp 0 copies (TMA), one thread of warp 1 issues the products, warp 2 patches the block's own K/V rows into the blocks that hold their
// positions and stores them to their page slots, four warps per tile make the softmax.
//
// All items form one line, a block costing what its kind costs (below), cut into equal ranges for a persistent grid of one CTA per
// SM: prefix items, which the tensor cores bound, and tails, which memory bounds, are at work at the same time.  What a CTA has
// of an item is a piece (O, m, l); attn_shared_merge_kernel adds the pieces of every row up, in order.
#include "kernels.cuh"
#include "ptx.cuh"
#include "umma.cuh"

namespace massv {

namespace {

constexpr int kTileRows = 128;
constexpr int kPagesPerBlock = kPrefixBlock / kPageSize;
constexpr float kRescaleThreshold = 8.f;   // log2 units a row's maximum may outgrow its reference by

// Cost of a block: products of two tiles, of one, of a tail.
constexpr int kCostTwo = 8, kCostOne = 5, kCostTail = 4;

template <int D>
struct SharedCfg {
    static constexpr int kTiles = D == 256 ? 1 : 2;           // query tiles of a CTA
    static constexpr int kParts = D == 256 ? 2 : 1;           // ring entries of a K block (halves of d) and of a V block (halves of the positions)
    static constexpr int kNCH = D / 64;
    static constexpr int kQTile = kTileRows * D * 2;
    static constexpr int kEntry = kPrefixBlock * D * 2 / kParts;
    static constexpr int kEntries = D == 64 ? 8 : 4;
    static constexpr int kBoxes = kPagesPerBlock * kNCH / kParts;      // 16-position x 64-element boxes of an entry
    static constexpr int kSmem = kTiles * kQTile + kEntries * kEntry + 1024;      // and the line (line_ints)
    static constexpr int kThreads = 128 + kTiles * 128;
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
template <int N>
__device__ __forceinline__ void tmem_ld_wait(uint32_t (&r)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+r"(r[j]));       // no use may move ahead of the wait
}
__device__ __forceinline__ void tmem_st_row32(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
        "r"(r[31])
        : "memory");
}

// Where a piece is kept: slots of the CTAs' cut items (two each), slots of prefix items that one CTA has all of, slots of such tails.
struct Piece {
    float4* o;            // [d / 4][stride rows]: unit c4 * stride + row holds four columns of a row
    float2* ml;           // [stride rows]: reference (log2 units) and sum
    int stride;
};
__device__ __forceinline__ Piece piece_at(const SharedAttnParams& p, int slot, int x, int D) {
    const SharedAttnSlots& s = p.slots;
    const int big = s.cut + s.prefix_items, item = -1 - slot;
    size_t rows;                                                       // rows of the pieces ahead of it
    Piece r;
    r.stride = kTileRows;
    if (slot >= 0) rows = ((size_t)slot * s.tiles + x) * kTileRows;
    else if (item < s.prefix_items) rows = ((size_t)(s.cut + item) * s.tiles + x) * kTileRows;
    else {
        rows = (size_t)big * s.tiles * kTileRows + ((size_t)(item - s.prefix_items) * s.tiles + x) * s.tail_rows;
        r.stride = s.tail_rows;
    }
    if (!MASSV_IN_BOUNDS(rows + r.stride, (long long)s.rows() + 1, p.a.dev_status)) rows = 0;
    r.o = reinterpret_cast<float4*>(p.part_o) + rows * (D / 4);
    r.ml = reinterpret_cast<float2*>(p.part_ml) + rows;
    return r;
}

// ---- the line of work, in shared memory: what every role finds its pieces by
struct Line {
    const int* gs;        // [n_groups + 1] first sequence of each group (all sequences in group 0 with no blocks where the groups are none)
    const int* gcost;     // [n_groups + 1] cost of the prefix items of groups 0 .. g-1
    const int* gitem;     // [n_groups + 1] their number
    const int* gblocks;   // [n_groups] blocks of the shared prefix
    const int* gsrc;      // [n_groups] the sequence whose page table is read for it
    const int* tail;      // [B + 1] tail blocks of sequences 0 .. b-1, per KV head
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
    bool tail;
    int head, seq;       // seq: whose page table is read
    int blk0;            // first (sequence, block row) pair of the rows
    int n_rows[2];       // query rows of each tile
    int pos0;            // position of the first block
    int n;               // blocks
    int L;               // tail: committed length
    int slot;            // slot of its piece: >= 0 one of the CTA's two, else -1 - item for an item that the CTA has all of (prefix items, then tails)
};

template <int D>
__global__ void __launch_bounds__(SharedCfg<D>::kThreads, 1)
attn_shared_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_q,
                   const SharedAttnParams p) {
    using Cfg = SharedCfg<D>;
    constexpr int E = Cfg::kEntries, NT = Cfg::kTiles, PARTS = Cfg::kParts, NCH = Cfg::kNCH;
    constexpr int UPR = D / 8;             // 16-byte units per K/V row
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t ready_bar[E], empty_bar[E];
    __shared__ __align__(8) uint64_t landed_bar[E];                    // the bytes of an entry that still needs patching
    __shared__ __align__(8) uint64_t q_ready_bar, q_free_bar;
    __shared__ __align__(8) uint64_t s_full_bar[2], p_full_bar[2];     // by score buffer
    __shared__ __align__(8) uint64_t o_full_bar[2], o_free_bar[2];     // by tile
    __shared__ __align__(8) uint64_t pv_done_bar;                      // one tile: O is up to date
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag, s_bad;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int R = p.a.R, B = p.a.B, cap = p.a.max_pages * kPageSize;
    const int G = p.a.Hq / p.a.Hkv, nb = kTileRows / G, tile_rows = nb * G;
    if (threadIdx.x == 0) {
        for (int e = 0; e < E; ++e) { mbar_init(&ready_bar[e], 1); mbar_init(&empty_bar[e], 1); mbar_init(&landed_bar[e], 1); }
        mbar_init(&q_ready_bar, 1); mbar_init(&q_free_bar, 1); mbar_init(&pv_done_bar, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&s_full_bar[i], 1); mbar_init(&p_full_bar[i], 4); mbar_init(&o_full_bar[i], 1); mbar_init(&o_free_bar[i], 4); }
        abort_flag = 0;
        s_bad = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(Cfg::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* q_smem = smem + E * Cfg::kEntry;                          // [tile][d / 64][128 rows][128 B], swizzled
    int* gs = reinterpret_cast<int*>(q_smem + NT * Cfg::kQTile);
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
    auto fits = [&](int L) { return L >= 0 && L + R <= cap; };
    for (int i = threadIdx.x; i <= p.n_groups; i += blockDim.x) {
        const int lo = p.group_start[i];
        gs[i] = lo;
        if (i < p.n_groups) { gcost[i] = 0x7fffffff; gitem[i] = 0; gsrc[i] = 0x7fffffff; gblocks[i] = p.shared_lens[i]; }
        if ((i == 0 && lo != 0) || (i == p.n_groups && lo != B) || (i < p.n_groups && lo > p.group_start[i + 1])) s_bad = 1;
    }
    for (int b = threadIdx.x; b < B; b += blockDim.x) tail[b + 1] = p.a.seq_lens[b];
    __syncthreads();
    const bool bad = s_bad != 0;
    if (bad)                                // one group that shares nothing
        for (int i = threadIdx.x; i <= p.n_groups; i += blockDim.x) { gs[i] = i == 0 ? 0 : B; if (i < p.n_groups) gblocks[i] = 0; }
    __syncthreads();
    for (int b = threadIdx.x; b < B; b += blockDim.x) {
        const int L = tail[b + 1], g = find_last(gs, p.n_groups, b);
        if (!fits(L)) continue;
        atomicMin(&gcost[g], L);
        atomicMin(&gsrc[g], b);
        atomicAdd(&gitem[g], 1);
    }
    __syncthreads();
    // whole blocks that every member has committed; a sequence alone shares nothing
    for (int i0 = 0; i0 < p.n_groups; i0 += blockDim.x) {              // (one round: at most 256 groups)
        const int i = i0 + threadIdx.x;
        if (i < p.n_groups) gblocks[i] = gitem[i] < 2 ? 0 : max(0, min(gblocks[i], gcost[i])) / kPrefixBlock;
    }
    __syncthreads();
    for (int b = threadIdx.x; b < B; b += blockDim.x) {
        const int L = tail[b + 1];
        const bool ok = fits(L);
        if (!ok && blockIdx.x == 0) set_status(p.a.dev_status, MASSV_ERR_CAPACITY);
        tail[b + 1] = ok ? (L + R + kPrefixBlock - 1) / kPrefixBlock - gblocks[find_last(gs, p.n_groups, b)] : 0;
    }
    for (int i = threadIdx.x; i < p.n_groups; i += blockDim.x) {
        const int pairs = (gs[i + 1] - gs[i]) * R, tiles = (pairs + nb - 1) / nb, items = gblocks[i] > 0 ? (tiles + NT - 1) / NT * p.a.Hkv : 0;
        gitem[i + 1] = items;
        gcost[i + 1] = items * gblocks[i] * (NT == 2 && tiles > 1 ? kCostTwo : kCostOne);
    }
    if (threadIdx.x == 0) { gcost[0] = 0; gitem[0] = 0; tail[0] = 0; }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    auto scan = [&](int* cum, int n) {      // cum[1 .. n] to their running sums, by one warp
        const int per = (n + 31) / 32, i0 = min(n, lane * per), i1 = min(n, i0 + per);
        int local = 0;
        for (int i = i0; i < i1; ++i) local += cum[i + 1];
        int incl = local;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        int run = incl - local;
        for (int i = i0; i < i1; ++i) { run += cum[i + 1]; cum[i + 1] = run; }
    };
    if (warp == 0) scan(gcost, p.n_groups);
    else if (warp == 2) scan(gitem, p.n_groups);
    else if (warp == 3) scan(tail, B);
    __syncthreads();
    const int tails0 = gcost[p.n_groups];                              // where the tails begin on the line
    const int total = tails0 + tail[B] * p.a.Hkv * kCostTail;
    const int per = max(kCostTwo, (total + (int)gridDim.x - 1) / (int)gridDim.x);        // (no block is longer than a range)
    if (blockIdx.x == 0) {
        if (threadIdx.x == 0) {
            p.meta[0] = per; p.meta[1] = tails0;
            if (bad) set_status(p.a.dev_status, MASSV_ERR_INVALID_ARG);
        }
        for (int b = threadIdx.x; b < B; b += blockDim.x) {
            const int g = find_last(gs, p.n_groups, b);
            p.seqs[b] = make_int4(tail[b], tail[b + 1] - tail[b], (b - gs[g]) * R, gblocks[g]);
            p.seq_groups[b] = make_int4(gcost[g], gitem[g], NT == 2 && (gs[g + 1] - gs[g]) * R > nb ? kCostTwo : kCostOne, 0);
        }
    }

    // ---- this CTA's range: the blocks that begin in it
    const int f_begin = min((long long)total, (long long)blockIdx.x * per), f_end = min((long long)total, (long long)f_begin + per);
    int f = f_begin;
    // The item that position f of the line lies in, and the run of its blocks that begin at or behind f and inside the range.
    auto next_run = [&](Run& r) -> bool {
        while (f < f_end) {
            int start, n_all, cost, item;
            if (f < tails0) {
                const int g = find_last(ln.gcost, ln.n_groups, f), pairs = (ln.gs[g + 1] - ln.gs[g]) * R;
                cost = NT == 2 && pairs > nb ? kCostTwo : kCostOne;
                n_all = ln.gblocks[g];
                const int k = (f - ln.gcost[g]) / (n_all * cost), tile = k / p.a.Hkv, done = tile * nb * NT;
                start = ln.gcost[g] + k * n_all * cost;
                item = ln.gitem[g] + k;
                r.tail = false;
                r.head = k - tile * p.a.Hkv;
                r.seq = ln.gsrc[g];
                r.blk0 = ln.gs[g] * R + done;
                r.n_rows[0] = min(nb, pairs - done) * G;
                r.n_rows[1] = NT == 2 ? max(0, min(nb, pairs - done - nb)) * G : 0;
                r.pos0 = 0;
            } else {
                const int u = (f - tails0) / kCostTail, b = find_last(ln.tail, B, u / p.a.Hkv);      // (blocks of a sequence: n per head, head after head)
                cost = kCostTail;
                n_all = ln.tail[b + 1] - ln.tail[b];
                r.head = (u - ln.tail[b] * p.a.Hkv) / n_all;
                start = tails0 + (ln.tail[b] * p.a.Hkv + r.head * n_all) * kCostTail;
                item = p.slots.prefix_items + b * p.a.Hkv + r.head;
                r.tail = true;
                r.seq = b;
                r.blk0 = b * R;
                r.n_rows[0] = r.n_rows[1] = R * G;
                r.pos0 = ln.gblocks[find_last(ln.gs, ln.n_groups, b)] * kPrefixBlock;
            }
            const int k0 = (f - start + cost - 1) / cost, k1 = min(n_all, (f_end - start + cost - 1) / cost);
            f = start + k1 * cost;
            if (k0 >= k1) continue;         // the item's last block begins ahead of the range
            r.pos0 += k0 * kPrefixBlock;
            r.n = k1 - k0;
            // an item that began in an earlier CTA's range has slot 0, one that runs on into the next has slot 1
            r.slot = k0 == 0 && k1 == n_all ? -1 - item : (int)blockIdx.x * 2 + (k0 > 0 ? 0 : 1);
            r.L = r.tail ? p.a.seq_lens[r.seq] : 0;
            if (r.tail && (NT == 1 || r.n < 2)) r.n_rows[1] = 0;
            return true;
        }
        return false;
    };
    // Entries of the ring are filled in the order in which the products take them.  Two tiles on one prefix: K0 V0 K1 V1 ...; otherwise
    // the scores run a block ahead: K0 K1 V0 K2 V1 ... V(n-1).
    auto decode = [&](const Run& r, int i, int& t, int& is_v) {
        if (NT == 2 && !r.tail) { t = i >> 1; is_v = i & 1; }
        else if (i == 0) { t = 0; is_v = 0; }
        else if (i == 2 * r.n - 1) { t = r.n - 1; is_v = 1; }
        else if (i & 1) { t = (i + 1) >> 1; is_v = 0; }
        else { t = (i >> 1) - 1; is_v = 1; }
    };

    const uint32_t tmem_base = tmem_base_slot;
    volatile int* abort_ptr = &abort_flag;
    Run r;
    if (warp == 0) {
        // ------------------------------------------------ copies
        uint64_t policy;
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
        int it = 0;                      // entries filled so far
        bool ok = true;
        for (int run = 0; ok && next_run(r); ++run) {
            if (run >= 1) {
                int fr = 0;
                if (lane == 0) fr = mbar_wait(&q_free_bar, (uint32_t)(run - 1) & 1u, abort_ptr) ? 1 : 0;
                if (!__shfl_sync(0xffffffffu, fr, 0)) { ok = false; break; }
            }
            const int tiles = !r.tail && r.n_rows[1] > 0 ? 2 : 1;      // (a tail's two accumulators have the same rows)
            if (lane == 0) mbar_expect_tx(&q_ready_bar, (uint32_t)(tiles * tile_rows * D * 2));
            __syncwarp();
            if (lane < tiles * NCH) {
                const int x = lane / NCH, dc = lane % NCH;
                tma_load_3d(q_smem + x * Cfg::kQTile + dc * (kTileRows * 128), &map_q, dc * 64, r.head * G, r.blk0 + x * nb, &q_ready_bar, policy);
            }
            // page ids travel in registers: lane l holds page 32 * group + l of the run, four blocks to a group
            const int32_t* pt = p.a.page_table + (size_t)r.seq * p.a.max_pages + r.pos0 / kPageSize;
            const int end = r.tail ? min(r.L + R - r.pos0, r.n * kPrefixBlock) : r.n * kPrefixBlock;      // positions of the run
            const int n_pages = (end + kPageSize - 1) / kPageSize;
            int pid_prev = 0, pid_cur = lane < n_pages ? pt[lane] : 0, pid_next = 32 + lane < n_pages ? pt[32 + lane] : 0, grp = 0;
            for (int i = 0; i < 2 * r.n && ok; ++i) {
                int t, is_v;
                decode(r, i, t, is_v);
                if (t / 4 > grp) {       // only a K block can be the first of a new group
                    grp = t / 4;
                    pid_prev = pid_cur; pid_cur = pid_next;
                    const int nxt = (grp + 1) * 32 + lane;
                    pid_next = nxt < n_pages ? pt[nxt] : 0;
                }
                const int held = t / 4 == grp ? pid_cur : pid_prev;
                const bool patch = r.tail && r.pos0 + (t + 1) * kPrefixBlock > r.L;
                const int have = min(kPagesPerBlock, n_pages - t * kPagesPerBlock);        // pages of the block that hold positions
                for (int part = 0; part < PARTS; ++part, ++it) {
                    const int e = it % E;
                    int freed = 0;
                    if (lane == 0) freed = mbar_wait(&empty_bar[e], (((uint32_t)(it / E)) & 1u) ^ 1u, abort_ptr) ? 1 : 0;
                    if (!__shfl_sync(0xffffffffu, freed, 0)) { ok = false; break; }
                    // K parts are halves of d, V parts halves of the positions
                    const int groups = is_v ? NCH : NCH / PARTS, pages = Cfg::kBoxes / groups;
                    const int c = lane % groups, pg = lane / groups;
                    const int dc = is_v ? c : part * groups + c, page0 = is_v ? part * pages : 0;
                    const int n_pg = max(0, min(pages, have - page0));
                    uint64_t* bar = patch ? &landed_bar[e] : &ready_bar[e];
                    if (lane == 0) mbar_expect_tx(bar, (uint32_t)(n_pg * groups * 2048));
                    __syncwarp();
                    int pid = __shfl_sync(0xffffffffu, held, (t % 4) * kPagesPerBlock + (page0 + pg) % kPagesPerBlock);
                    if (lane < Cfg::kBoxes && pg < n_pg) {
                        if (pid < 0 || pid >= p.a.num_pages) { set_status(p.a.dev_status, MASSV_ERR_CAPACITY); pid = 0; }
                        tma_load_2d(smem + (size_t)e * Cfg::kEntry + c * (pages * kPageSize * 128) + pg * 2048, is_v ? &map_v : &map_k, dc * 64,
                                    (pid * p.a.Hkv + r.head) * kPageSize, bar, policy);
                    }
                }
            }
        }
        if (lane == 0 && *abort_ptr) {
            for (int i = 0; i < 64; ++i) __nanosleep(2000);            // let copies in flight land
        }
    } else if (warp == 2) {
        // ------------------------------------------------ helper: the block's own rows, and what lies behind the last position
        uint32_t landed_phase = 0;       // bit e: parity of the next completion of landed_bar[e]
        int it0 = 0;                     // entries of earlier runs
        bool ok = true;
        for (; ok && next_run(r); it0 += 2 * r.n * PARTS) {
            if (!r.tail || r.pos0 + r.n * kPrefixBlock <= r.L) continue;
            const int t_first = max(0, r.L - r.pos0) / kPrefixBlock, end = r.L + R;
            const int32_t* pt = p.a.page_table + (size_t)r.seq * p.a.max_pages;
            for (int i = 0; i < 2 * r.n && ok; ++i) {
                int t, is_v;
                decode(r, i, t, is_v);
                if (t < t_first) continue;
                const int start = r.pos0 + t * kPrefixBlock;
                const __nv_bfloat16* src = is_v ? p.a.v_new : p.a.k_new;
                __nv_bfloat16* pool = is_v ? p.a.v_pages : p.a.k_pages;
                for (int part = 0; part < PARTS; ++part) {
                    const int e = (it0 + i * PARTS + part) % E;
                    // the entry's positions and 16-byte units of a row: K parts are halves of d, V parts halves of the positions
                    constexpr int kVRows = kPrefixBlock / PARTS, kKUnits = UPR / PARTS;
                    const int row0 = is_v ? part * kVRows : 0, n_row = is_v ? kVRows : kPrefixBlock, u0 = is_v ? 0 : part * kKUnits, n_u = is_v ? UPR : kKUnits;
                    const int first = max(r.L, start + row0), last = min(end, start + row0 + n_row);      // new positions inside
                    uint8_t* dst = smem + (size_t)e * Cfg::kEntry;
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
                    if (!mbar_wait_warp(&landed_bar[e], (landed_phase >> e) & 1u, abort_ptr)) { ok = false; break; }
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
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------ products
        if (lane == 0) {
            constexpr uint32_t idesc_qk = umma_idesc_bf16(kTileRows, kPrefixBlock, false);
            constexpr uint32_t idesc_pv = umma_idesc_bf16(kTileRows, D, true);
            constexpr int kVRegion = kPrefixBlock / PARTS * 128;
            const uint32_t q_lo = umma_desc_lo(smem_u32(q_smem)), ring = smem_u32(smem);
            bool ok = true;
            int it = 0;                              // ring entries taken so far
            int tau[2] = {0, 0}, runs[2] = {0, 0};   // blocks by score buffer, runs by tile so far
            auto entry_ready = [&](int i) { if (ok && !mbar_wait(&ready_bar[i % E], ((uint32_t)(i / E)) & 1u, abort_ptr)) ok = false; };
            // S[buf] = Q_x K^T over `part`'s share of d
            auto qk = [&](int x, int buf, int i, int part) {
                tc_fence_after();
                const uint32_t k_lo = umma_desc_lo(ring + (uint32_t)(i % E) * Cfg::kEntry), d_tmem = tmem_base + (uint32_t)(buf * kPrefixBlock);
#pragma unroll
                for (int kk = 0; kk < D / 16 / PARTS; ++kk) {
                    const int dc = part * (NCH / PARTS) + (kk >> 2);
                    const uint32_t a = q_lo + (uint32_t)((x * Cfg::kQTile + dc * (kTileRows * 128) + (kk & 3) * 32) >> 4);
                    const uint32_t bb = k_lo + (uint32_t)(((kk >> 2) * (kPrefixBlock * 128) + (kk & 3) * 32) >> 4);
                    if (kk == 0 && part == 0) umma_bf16<false>(d_tmem, a, bb, idesc_qk);
                    else umma_bf16<true>(d_tmem, a, bb, idesc_qk);
                }
            };
            // O_x (+)= P[buf] V over `part`'s share of the positions
            auto pv = [&](int x, int buf, int i, int part, bool first) {
                tc_fence_after();
                const uint32_t v_lo = (((ring + (uint32_t)(i % E) * Cfg::kEntry) & 0x3FFFFu) >> 4) | ((uint32_t)(kVRegion >> 4) << 16);
                const uint32_t d_tmem = tmem_base + Cfg::kTmemO + (uint32_t)(x * D), a0 = tmem_base + (uint32_t)(buf * kPrefixBlock);
#pragma unroll
                for (int ks = 0; ks < kPrefixBlock / 16 / PARTS; ++ks) {
                    const uint32_t a = a0 + (uint32_t)((part * (kPrefixBlock / 16 / PARTS) + ks) * 8), bb = v_lo + (uint32_t)((ks * 2048) >> 4);
                    if (ks == 0 && part == 0 && first) umma_bf16_ts<false>(d_tmem, a, bb, idesc_pv);
                    else umma_bf16_ts<true>(d_tmem, a, bb, idesc_pv);
                }
            };
            auto weights_ready = [&](int buf, int count) { if (ok && !mbar_wait(&p_full_bar[buf], (uint32_t)count & 1u, abort_ptr)) ok = false; };
            auto o_drained = [&](int x) { if (ok && runs[x] > 0 && !mbar_wait(&o_free_bar[x], (uint32_t)(runs[x] - 1) & 1u, abort_ptr)) ok = false; };
            for (int run = 0; ok && next_run(r); ++run) {
                const int n = r.n;
                const bool two = r.n_rows[1] > 0;
                if (!mbar_wait(&q_ready_bar, (uint32_t)run & 1u, abort_ptr)) { ok = false; break; }
                if (NT == 2 && !r.tail) {
                    entry_ready(it);
                    if (!ok) break;
                    qk(0, 0, it, 0); umma_commit(&s_full_bar[0]);
                    if (two) { qk(1, 1, it, 0); umma_commit(&s_full_bar[1]); }
                    umma_commit(&empty_bar[it % E]);
                    if (n == 1) umma_commit(&q_free_bar);
                    ++it;
                    for (int t = 0; t < n && ok; ++t) {
                        const int iv = it, ik = it + 1;               // V of this block, K of the next
                        const bool more = t + 1 < n;
                        it += more ? 2 : 1;
                        entry_ready(iv);
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            if (x == 1 && !two) break;
                            weights_ready(x, tau[x] + t);
                            if (t == 0) o_drained(x);
                            if (!ok) break;
                            pv(x, x, iv, 0, t == 0);
                            if (x == (two ? 1 : 0)) umma_commit(&empty_bar[iv % E]);
                            if (more) {
                                if (x == 0) { entry_ready(ik); if (!ok) break; }
                                qk(x, x, ik, 0);                       // over this tile's P, behind the product that read it
                                umma_commit(&s_full_bar[x]);
                            } else {
                                umma_commit(&o_full_bar[x]);
                            }
                        }
                        if (ok && more) {
                            umma_commit(&empty_bar[ik % E]);
                            if (t + 2 == n) umma_commit(&q_free_bar);
                        }
                    }
                    tau[0] += n; runs[0] += 1;
                    if (two) { tau[1] += n; runs[1] += 1; }
                } else {
                    // Scores ahead of the weights: block t's buffer takes the scores of block t + 2 behind the product that read its P.  One
                    // accumulator (head_dim 256), or even and odd blocks with one each, by buffer; buffers alternate from run to run where there is
                    // one accumulator, and start at 0 where there are two.
                    const int b0 = NT == 1 ? tau[0] & 1 : 0;
                    int done[2] = {0, 0};                              // blocks of this run by score buffer (two accumulators)
                    auto scores = [&](int t) {
                        const int buf = (b0 + t) & 1;
#pragma unroll
                        for (int part = 0; part < PARTS; ++part, ++it) {
                            entry_ready(it);
                            if (!ok) return;
                            qk(0, buf, it, part);
                            umma_commit(&empty_bar[it % E]);
                        }
                        umma_commit(&s_full_bar[buf]);
                        if (t == n - 1) umma_commit(&q_free_bar);
                    };
                    scores(0);
                    if (ok && n > 1) scores(1);
                    for (int t = 0; t < n && ok; ++t) {
                        const int buf = (b0 + t) & 1, x = NT == 1 ? 0 : buf;
                        weights_ready(buf, NT == 1 ? (tau[0] + t) >> 1 : tau[buf] + done[buf]);
                        if (NT == 1 ? t == 0 : t < 2) o_drained(x);
#pragma unroll
                        for (int part = 0; part < PARTS; ++part, ++it) {
                            entry_ready(it);
                            if (!ok) break;
                            pv(x, buf, it, part, NT == 1 ? t == 0 : t < 2);
                            umma_commit(&empty_bar[it % E]);
                        }
                        if (!ok) break;
                        ++done[buf];
                        if (NT == 1) umma_commit(&pv_done_bar);
                        if (NT == 1 ? t == n - 1 : t >= n - 2) umma_commit(&o_full_bar[x]);
                        if (t + 2 < n) scores(t + 2);
                    }
                    if (NT == 1) { tau[0] += n; runs[0] += 1; }
                    else { tau[0] += done[0]; tau[1] += done[1]; runs[0] += 1; if (n > 1) runs[1] += 1; }
                }
            }
        }
    } else if (warp >= 4) {
        // ------------------------------------------------ softmax: a row per thread
        const int x = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tmem_o = tmem_base + Cfg::kTmemO + (uint32_t)(x * D) + lane_base;
        const float scale_log2 = p.a.scale * 1.4426950408889634f;
        bool ok = true;
        int tau = 0, runs = 0;
        while (ok && next_run(r)) {
            if (r.n_rows[x] == 0) continue;
            const bool alone = r.tail && NT == 2;                      // every second block is this tile's
            const bool some = (warp & 3) * 32 < r.n_rows[x];           // this warp has rows
            const int j = min(row / G, R - 1);                         // tail: block row
            float ref = -INFINITY, l_run = 0.f;
            for (int t = alone ? x : 0; t < r.n && ok; t += alone ? 2 : 1, ++tau) {
                const int buf = NT == 2 ? x : tau & 1;
                const uint32_t parity = (uint32_t)(NT == 2 ? tau : tau >> 1) & 1u;
                if (!mbar_wait_warp(&s_full_bar[buf], parity, abort_ptr)) { ok = false; break; }
                tc_fence_after();
                if (some) {
                    const uint32_t tmem_s = tmem_base + lane_base + (uint32_t)(buf * kPrefixBlock);
                    uint32_t s[kPrefixBlock];
#pragma unroll
                    for (int c = 0; c < kPrefixBlock; c += 32) tmem_ld_row32(tmem_s + (uint32_t)c, s + c);
                    tmem_ld_wait(s);
                    const int start = r.pos0 + t * kPrefixBlock;
                    if (r.tail && start + kPrefixBlock > r.L + 1) {    // a position ahead of some row, or past the end
                        const int seen = r.L + j - start;              // the last column this row sees
#pragma unroll
                        for (int c = 0; c < kPrefixBlock; ++c) s[c] = c > seen ? 0xff800000u : s[c];
                    }
                    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < kPrefixBlock; c += 2) m4[(c >> 1) & 3] = fmaxf(m4[(c >> 1) & 3], fmaxf(__uint_as_float(s[c]), __uint_as_float(s[c + 1])));
                    const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * scale_log2;        // (the scale is positive)
                    // The reference moves when the row's maximum has outgrown it by the threshold; O and l follow it.
                    float factor = 1.f;
                    bool moved = false;
                    if (ref == -INFINITY) ref = mx;
                    else if (mx > ref + kRescaleThreshold) { factor = exp2f(ref - mx); ref = mx; moved = true; }
                    if (__any_sync(0xffffffffu, moved)) {
                        // (two accumulators: the scores stand behind the product before them, so O is up to date)
                        if (NT == 1 && !mbar_wait_warp(&pv_done_bar, (uint32_t)(tau - 1) & 1u, abort_ptr)) { ok = false; break; }
                        tc_fence_after();
#pragma unroll 1
                        for (int c0 = 0; c0 < D; c0 += 32) {
                            uint32_t o[32];
                            tmem_ld_row32(tmem_o + (uint32_t)c0, o);
                            tmem_ld_wait(o);
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * factor);
                            tmem_st_row32(tmem_o + (uint32_t)c0, o);
                        }
                        l_run *= factor;
                    }
                    const float neg = ref == -INFINITY ? 0.f : -ref;
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t pk[32];
#pragma unroll
                        for (int c = 0; c < 32; ++c) {
                            const float p0 = ex2_ftz(fmaf(__uint_as_float(s[h * 64 + 2 * c]), scale_log2, neg));
                            const float p1 = ex2_ftz(fmaf(__uint_as_float(s[h * 64 + 2 * c + 1]), scale_log2, neg));
                            part[c & 3] += p0 + p1;
                            pk[c] = bf16x2(p0, p1);
                        }
                        tmem_st_row32(tmem_s + (uint32_t)(h * 32), pk);
                    }
                    l_run += (part[0] + part[1]) + (part[2] + part[3]);
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full_bar[buf]);
            }
            if (!ok || !mbar_wait_warp(&o_full_bar[x], (uint32_t)runs & 1u, abort_ptr)) { ok = false; break; }
            ++runs;
            tc_fence_after();
            if (some) {
                // ---- the piece
                const Piece pc = piece_at(p, r.slot, x, D);
                const bool live = row < r.n_rows[x];
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 32) {
                    uint32_t o[32];
                    tmem_ld_row32(tmem_o + (uint32_t)c0, o);
                    tmem_ld_wait(o);
                    if (live) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4)
                            pc.o[(size_t)((c0 + k) / 4) * pc.stride + row] =
                                make_float4(__uint_as_float(o[k]), __uint_as_float(o[k + 1]), __uint_as_float(o[k + 2]), __uint_as_float(o[k + 3]));
                    }
                }
                if (live) pc.ml[row] = make_float2(ref, l_run);
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

// Pieces of a row added up.  CTA (sequence and KV head, part of its units): a unit is eight columns of one row, rows side by side.
constexpr int kMergeThreads = 128;
__global__ void __launch_bounds__(kMergeThreads) attn_shared_merge_kernel(const SharedAttnParams p, int tiles_per_item) {
    const int h = blockIdx.x % p.a.Hkv, b = blockIdx.x / p.a.Hkv, D = p.a.d, R = p.a.R;
    const int G = p.a.Hq / p.a.Hkv, rows = G * R, nb = kTileRows / G;
    const int unit = blockIdx.y * kMergeThreads + threadIdx.x, row = unit % rows, c8 = unit / rows;
    pdl_wait();
    pdl_trigger();
    const int4 seq = p.seqs[b], grp = p.seq_groups[b];
    const int per = p.meta[0], tails0 = p.meta[1];
    if (seq.y == 0 || c8 * 8 >= D) return;                             // skipped; past the last unit
    // An item's pieces: consecutive CTAs of the kernel above; alone in one, it has a slot of its own.
    struct Pieces { int start, blocks, cost, c0, c1, item; };
    auto pieces_of = [&](int start, int blocks, int cost, int item) {
        return Pieces{start, blocks, cost, start / per, (start + (blocks - 1) * cost) / per, item};
    };
    auto slot_of = [&](const Pieces& q, int c) { return q.c0 == q.c1 ? -1 - q.item : c * 2 + (q.start < c * per ? 0 : 1); };
    const Pieces tl = pieces_of(tails0 + (seq.x * p.a.Hkv + h * seq.y) * kCostTail, seq.y, kCostTail, p.slots.prefix_items + b * p.a.Hkv + h);
    const int pair = seq.z + row / G, tile = pair / nb, k = tile / tiles_per_item * p.a.Hkv + h;
    const int prow = (pair - tile * nb) * G + row % G, px = tile % tiles_per_item;
    Pieces pf{0, 0, 1, 0, -1, 0};
    if (seq.w > 0) pf = pieces_of(grp.x + k * seq.w * grp.z, seq.w, grp.z, grp.y + k);
    // a tail's piece is in two accumulators where it has more than one block
    auto tail_tiles = [&](int c) {
        const long long lo = max(0LL, (long long)c * per - tl.start), hi = (long long)(c + 1) * per - tl.start;
        const int k0 = (int)((lo + kCostTail - 1) / kCostTail), k1 = (int)min((long long)tl.blocks, (hi + kCostTail - 1) / kCostTail);
        return min(tiles_per_item, k1 - k0);
    };
    float m = -INFINITY;
    for (int c = pf.c0; c <= pf.c1; ++c) m = fmaxf(m, piece_at(p, slot_of(pf, c), px, D).ml[prow].x);
    for (int c = tl.c0; c <= tl.c1; ++c)
        for (int x = 0; x < tail_tiles(c); ++x) m = fmaxf(m, piece_at(p, slot_of(tl, c), x, D).ml[row].x);
    float sum = 0.f, acc[8] = {};
    auto add = [&](const Piece& pc, int at) {
        const float2 ml = pc.ml[at];
        const float4 u = pc.o[(size_t)(2 * c8) * pc.stride + at], v = pc.o[(size_t)(2 * c8 + 1) * pc.stride + at];
        const float w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - m);     // (a row that sees nothing of the piece)
        sum += ml.y * w;
        acc[0] += u.x * w; acc[1] += u.y * w; acc[2] += u.z * w; acc[3] += u.w * w;
        acc[4] += v.x * w; acc[5] += v.y * w; acc[6] += v.z * w; acc[7] += v.w * w;
    };
#pragma unroll 4
    for (int c = pf.c0; c <= pf.c1; ++c) add(piece_at(p, slot_of(pf, c), px, D), prow);
    for (int c = tl.c0; c <= tl.c1; ++c)
        for (int x = 0; x < tail_tiles(c); ++x) add(piece_at(p, slot_of(tl, c), x, D), row);
    const float inv = 1.f / sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] *= inv;
    const size_t out = ((size_t)b * R + row / G) * p.a.Hq + h * G + row % G;
    *reinterpret_cast<uint4*>(p.a.out + out * D + c8 * 8) = make_uint4(bf16x2(acc[0], acc[1]), bf16x2(acc[2], acc[3]), bf16x2(acc[4], acc[5]), bf16x2(acc[6], acc[7]));
    if (p.a.out_f32) {
        float4* f = reinterpret_cast<float4*>(p.a.out_f32 + out * D + c8 * 8);
        f[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        f[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
    }
    if (p.a.lse && c8 == 0) p.a.lse[out] = (m + log2f(sum)) * 0.6931471805599453f;
}

template <int D>
cudaError_t launch(const SharedAttnParams& p, cudaStream_t stream) {
    using Cfg = SharedCfg<D>;
    const int G = p.a.Hq / p.a.Hkv;
    CUtensorMap mk, mv, mq;
    const uint64_t rows_total = (uint64_t)p.a.num_pages * p.a.Hkv * kPageSize;
    if (!make_tensor_map_bf16_2d(&mk, p.a.k_pages, rows_total, D, kPageSize) || !make_tensor_map_bf16_2d(&mv, p.a.v_pages, rows_total, D, kPageSize) ||
        !make_tensor_map_bf16_heads(&mq, p.a.q, (uint64_t)p.a.B * p.a.R, (uint64_t)p.a.Hq, D, (uint32_t)(kTileRows / G), (uint32_t)G))
        return cudaErrorInvalidValue;
    cudaError_t e = cudaFuncSetAttribute(attn_shared_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kMaxSmem);
    if (e != cudaSuccess) return e;
    int ctas = device_sm_count();
    if (ctas > kSharedMaxCtas) ctas = kSharedMaxCtas;
    const size_t smem = Cfg::kSmem + (size_t)(p.a.B + 1 + 5 * (p.n_groups + 1)) * 4;
    e = launch_pdl(attn_shared_kernel<D>, dim3(ctas), dim3(Cfg::kThreads), smem, stream, mk, mv, mq, p);
    if (e != cudaSuccess) return e;
    const int units = G * p.a.R * (D / 8);
    return launch_pdl(attn_shared_merge_kernel, dim3(p.a.B * p.a.Hkv, (units + kMergeThreads - 1) / kMergeThreads), dim3(kMergeThreads), 0, stream, p, Cfg::kTiles);
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
